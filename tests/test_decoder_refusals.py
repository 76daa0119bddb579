"""What attention over triangles and shared prefixes, the weights of cached positions and eviction refuse on the host, without a device."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def api():
    from paper_2609_24802_b200 import build
    build.build_library()
    from paper_2609_24802_b200 import api
    return api


REF = ctypes.byref
BIG = 1 << 40


def heads(api, dtype=1, h=4, hk=2, D=64, scale=1.0, q=(256, 64), key=(128, 64), value=(128, 64), go=(256, 64)):
    s = api._Stride
    return api._Heads(dtype, h, hk, D, scale, s(*q), s(*key), s(*value), s(*go))


def dense(api, n_seg=2, n_q=10, n_kv=20, q=256, kv=256, mask=0):
    return api._Dense(q, kv, mask, n_seg, n_q, n_kv)


def pages(api, key=256, value=256, table=256, lens=256, n_seg=2, n_pages=8, page_size=16, table_stride=4, max_pages=4, page_stride=2048, slot=128, head=64):
    return api._Pages(key, value, table, lens, n_seg, n_pages, page_size, table_stride, max_pages, page_stride, slot, head)


def weights(api, data=512, seg=200, head=100, length=64):
    return api._Weights(data, seg, head, length)


BAD_HEADS = [(dict(dtype=0), 2), (dict(dtype=3), 1), (dict(h=0), 1), (dict(hk=0), 1), (dict(h=5), 1), (dict(D=0), 1), (dict(D=60), 2), (dict(D=136), 2),
             (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1)]
BAD_PAGES = [dict(page_size=0), dict(n_pages=-1), dict(max_pages=-1), dict(table_stride=-1), dict(slot=100), dict(page_stride=-8), dict(head=4), dict(n_seg=-1),
             dict(key=None), dict(table=None), dict(lens=None), dict(table=258)]


def test_triangle(api):
    L = api.load_library()

    def forward(g, h, q=256, k=256, v=256, out=256, lse=256, ws=256, size=BIG):
        return L.tiga_apply_triangular_attention(REF(g), REF(h), q, k, v, out, lse, ws, size, None)

    def backward(g, h, q=256, k=256, v=256, out=256, lse=256, go=256, gq=256, gk=256, gv=256, ws=256, size=BIG):
        return L.tiga_apply_triangular_attention_backward(REF(g), REF(h), q, k, v, out, lse, go, gq, gk, gv, ws, size, None)
    h = heads(api)
    for bad, status in BAD_HEADS:
        assert forward(dense(api), heads(api, **bad)) == status and backward(dense(api), heads(api, **bad)) == status
        assert L.tiga_triangular_attention_workspace_bytes(REF(dense(api)), REF(heads(api, **bad)), 1) == 0
    for bad, status in ((dict(n_q=-1), 1), (dict(n_seg=-1), 1), (dict(n_q=1 << 31), 2), (dict(n_seg=1 << 25), 2), (dict(n_kv=(1 << 31) - 100), 2), (dict(q=0), 1), (dict(kv=258), 1)):
        assert forward(dense(api, **bad), h) == status and backward(dense(api, **bad), h) == status, bad
    for name in ("q", "k", "v", "out"):
        assert forward(dense(api), h, **{name: None}) == 1 and forward(dense(api), h, **{name: 264}) == 1
    for name in ("q", "k", "v", "out", "lse", "go"):
        assert backward(dense(api), h, **{name: None}) == 1
    for bad in (dict(q=(-256, 64)), dict(key=(128, 4)), dict(value=(100, 64))):
        assert forward(dense(api), heads(api, **bad)) == 1
    assert backward(dense(api), heads(api, go=(256, 60))) == 1
    assert forward(dense(api), h, ws=None) == 3 and forward(dense(api), h, size=16) == 3 and backward(dense(api), h, size=16) == 3
    assert forward(dense(api, n_q=0), h) == 0 and forward(dense(api, n_seg=0), h) == 0 and backward(dense(api), h, gq=None, gk=None, gv=None) == 0


def test_shared_prefixes(api):
    L, h = api.load_library(), heads(api)

    def call(c=None, g=(256, 256, 1), hh=h, q=256, start=256, n=10, out=256, lse=256, ws=256, size=BIG):
        return L.tiga_apply_shared_attention(REF(c or pages(api)), REF(hh), REF(api._Prefixes(*g)), q, start, n, 1, out, lse, ws, size, None)
    for bad, status in BAD_HEADS:
        assert call(hh=heads(api, **bad)) == status
    for bad in BAD_PAGES + [dict(value=264)]:
        assert call(pages(api, **bad)) == 1, bad
    for bad in ((None, 256, 1), (256, None, 1), (258, 256, 1), (256, 257, 1), (256, 256, -1)):
        assert call(g=bad) == 1, bad
    assert call(g=(256, 256, 1 << 24)) == 2 and call(g=(256, None, 0), size=8) == 3
    assert call(q=None) == 1 and call(start=None) == 1 and call(out=264) == 1 and call(lse=260) == 1 and call(n=-1) == 1
    assert call(size=8) == 3 and call(ws=None) == 3 and call(ws=264) == 3 and call(n=0) == 0 and call(pages(api, n_seg=0)) == 0
    assert L.tiga_shared_attention_workspace_bytes(REF(pages(api)), REF(h), REF(api._Prefixes(256, 256, -1)), 10) == 0
    # the states of rows take room as far as their groups may share, however many rows there are
    sizes = [L.tiga_shared_attention_workspace_bytes(REF(pages(api)), REF(h), REF(api._Prefixes(256, 256, 1)), n) for n in (10, 1000, 100000)]
    assert 0 < sizes[0] < sizes[1] == sizes[2]


def test_weights(api):
    L, h = api.load_library(), heads(api)

    def call(c=None, hh=h, q=256, start=256, n=10, lse=256, before=None, w=None, ws=256, size=BIG):
        w = w or weights(api)
        return L.tiga_paged_attention_weights(REF(c or pages(api)), REF(hh), q, start, n, lse, 1, None if before is None else REF(before), REF(w), ws, size, None)
    for bad, status in BAD_HEADS:
        assert call(hh=heads(api, **bad)) == status
    for bad in BAD_PAGES:
        assert call(pages(api, **bad)) == 1, bad
    for bad in (dict(data=None), dict(data=520), dict(seg=-1), dict(head=-1), dict(length=-1), dict(head=63), dict(seg=100), dict(seg=163), dict(seg=0)):
        assert call(w=weights(api, **bad)) == 1, bad
    assert call(w=weights(api, seg=64, head=200), size=8) == 3              # sequences in a head, heads one behind the other
    for bad in (dict(data=None), dict(data=520), dict(length=63), dict(data=512, seg=300), dict(data=512, head=64)):
        assert call(before=weights(api, **bad)) == 1, bad
    assert call(before=weights(api), size=8) == 3 and call(before=weights(api, data=1 << 20, seg=0, head=0), size=8) == 3
    assert call(q=None) == 1 and call(start=None) == 1 and call(lse=None) == 1 and call(lse=260) == 1 and call(n=-1) == 1 and call(hh=heads(api, q=(256, 4))) == 1
    assert call(size=8) == 3 and call(ws=None) == 3
    assert call(pages(api, n_seg=0)) == 0 and call(w=weights(api, length=0)) == 0 and call(pages(api, max_pages=0, table=None)) == 0
    assert L.tiga_paged_weights_workspace_bytes(REF(pages(api)), REF(heads(api, D=60)), 10) == 0


def test_eviction(api):
    L, h = api.load_library(), heads(api)

    def call(c=None, to=None, hh=h, w=None, keep=32, recent=4, tw=None, lens=1024, kept=256):
        return L.tiga_paged_evict(REF(c or pages(api)), REF(to or pages(api, lens=None)), REF(hh), REF(w or weights(api)), keep, recent, None if tw is None else REF(tw), lens, kept, None)
    for bad, status in BAD_HEADS:
        assert call(hh=heads(api, **bad)) == status
    for bad in BAD_PAGES + [dict(value=264)]:
        assert call(pages(api, **bad)) == 1, bad
    for bad in BAD_PAGES + [dict(value=264), dict(n_seg=3), dict(max_pages=1), dict(slot=0), dict(head=0), dict(page_stride=0)]:
        if "lens" not in bad:
            assert call(to=pages(api, **bad)) == 1, bad
    for bad in (dict(keep=0), dict(keep=-1), dict(recent=-1), dict(recent=33), dict(keep=65), dict(lens=None), dict(lens=1026), dict(lens=256), dict(kept=None), dict(kept=258)):
        assert call(**bad) == 1, bad
    for bad in (dict(data=None), dict(data=520), dict(seg=-1), dict(length=-1)):
        assert call(w=weights(api, **bad)) == 1, bad
    for bad in (dict(data=None), dict(data=520), dict(data=512), dict(data=4096, seg=100), dict(data=4096, head=10)):
        assert call(tw=weights(api, **bad)) == 1, bad
    assert call(pages(api, n_seg=0), pages(api, n_seg=0)) == 0


def test_descriptors_and_arrays_in_python(api):
    start = torch.tensor([0, 4], dtype=torch.int32)
    x = torch.zeros(4, 2, 64, dtype=torch.float16)
    assert api.TriangularRelation(start).kv_start is start
    for bad in (lambda: api.TriangularRelation(start, start[:1]), lambda: api.TriangularRelation(start.long()), lambda: api.TriangularRelation(start, mask=torch.zeros(4)),
                lambda: api.SharedPrefixes(start, start), lambda: api.SharedPrefixes(start.long(), start[:1]), lambda: api.SharedPrefixes(start, start[:1].float())):
        with pytest.raises(ValueError):
            bad()
    relation, prefixes = api.TriangularRelation(start), api.SharedPrefixes(start, start[1:])
    with pytest.raises(AttributeError):
        relation.q_start = start.clone()
    with pytest.raises(AttributeError):
        prefixes.shared = start[1:].clone()
    # the kinds of relations are told apart
    with pytest.raises(TypeError):
        api._dense_args(relation, x, x, x, 1.0)
    with pytest.raises(TypeError):
        api._dense_args(api.DenseRelation(start, start), x, x, x, 1.0, None, api.TriangularRelation)
    page = torch.zeros(2, 16, 2, 64, dtype=torch.float16)
    cache = api.PagedCache(page, page, torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
    for bad in (torch.zeros(1, 2, 32, dtype=torch.float64), torch.zeros(1, 3, 32), torch.zeros(2, 2, 32), torch.zeros(1, 2, 64)[:, :, ::2], torch.zeros(1, 64)):
        with pytest.raises(ValueError):
            api._weights_of(bad, cache, "weights")
    for call in (lambda: api.tiga_apply_triangular_attention(relation, x, x, x, 1.0), lambda: api.tiga_apply_shared_attention(cache, prefixes, x, start, 1.0),
                 lambda: api.tiga_paged_attention_weights(cache, x, start, torch.zeros(4, 2), 1.0), lambda: api.tiga_paged_evict(cache, cache, torch.zeros(1, 2, 32), 4)):
        with pytest.raises(ValueError):             # arrays on the host
            call()
