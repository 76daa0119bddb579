"""What attention over dense and paged relations, rotary positions and cache writes refuse on the host, without a device; the
frequencies of rotary positions, which are computed there."""
import ctypes
import math

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


def forward(api, g, h, q=256, k=256, v=256, out=256, lse=256, ws=256, size=BIG):
    return api.load_library().tiga_apply_dense_attention(REF(g), REF(h), q, k, v, out, lse, ws, size, None)


def backward(api, g, h, q=256, k=256, v=256, out=256, lse=256, go=256, gq=256, gk=256, gv=256, ws=256, size=BIG):
    return api.load_library().tiga_apply_dense_attention_backward(REF(g), REF(h), q, k, v, out, lse, go, gq, gk, gv, ws, size, None)


BAD_HEADS = [(dict(dtype=0), 2), (dict(dtype=3), 1), (dict(h=0), 1), (dict(hk=0), 1), (dict(h=5), 1), (dict(D=0), 1), (dict(D=60), 2), (dict(D=136), 2),
             (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1)]
BAD_STRIDES = [dict(q=(-256, 64)), dict(key=(128, 4)), dict(value=(100, 64))]


@pytest.mark.parametrize("bad,status", BAD_HEADS)
def test_descriptors(api, bad, status):
    h, g, L = heads(api, **bad), dense(api), api.load_library()
    assert forward(api, g, h) == status and backward(api, g, h) == status
    assert L.tiga_dense_attention_workspace_bytes(REF(g), REF(h), 0) == 0
    c = pages(api)
    assert L.tiga_apply_paged_attention(REF(c), REF(h), 256, 256, 10, 1, 256, 256, 256, BIG, None) == status
    assert L.tiga_paged_attention_workspace_bytes(REF(c), REF(h), 10) == 0
    assert L.tiga_paged_append(REF(c), REF(h), 256, 256, 256, 10, None, None) == status


@pytest.mark.parametrize("bad", BAD_STRIDES)
def test_strides(api, bad):
    assert forward(api, dense(api), heads(api, **bad)) == 1 and backward(api, dense(api), heads(api, **bad)) == 1


def test_dense_arguments(api):
    h = heads(api)
    assert forward(api, dense(api, n_q=-1), h) == 1 and forward(api, dense(api, n_seg=-1), h) == 1
    assert forward(api, dense(api, n_q=1 << 31), h) == 2 and forward(api, dense(api, n_seg=1 << 25), h) == 2
    assert forward(api, dense(api, n_q=1 << 30), heads(api, h=64)) == 2                  # packed rows of a group beyond 32 bits
    assert forward(api, dense(api, n_kv=(1 << 31) - 100), h) == 2                         # a tile's last row would not fit 32 bits
    assert forward(api, dense(api, q=0), h) == 1 and forward(api, dense(api, kv=258), h) == 1
    for name in ("q", "k", "v", "out"):
        assert forward(api, dense(api), h, **{name: None}) == 1 and forward(api, dense(api), h, **{name: 264}) == 1
    assert forward(api, dense(api), h, lse=260) == 1
    assert forward(api, dense(api), h, ws=None) == 3 and forward(api, dense(api), h, size=16) == 3 and forward(api, dense(api), h, ws=264) == 3
    assert forward(api, dense(api, n_q=0), h, q=None, out=None) == 0 and forward(api, dense(api, n_seg=0), h) == 0
    for name in ("q", "k", "v", "out", "lse", "go"):
        assert backward(api, dense(api), h, **{name: None}) == 1
    for name in ("gq", "gk", "gv"):
        assert backward(api, dense(api), h, **{name: 264}) == 1
    assert backward(api, dense(api), heads(api, go=(256, 60))) == 1
    assert backward(api, dense(api), h, size=16) == 3
    assert backward(api, dense(api), h, gq=None, gk=None, gv=None) == 0


def pages(api, key=256, value=256, table=256, lens=256, n_seg=2, n_pages=8, page_size=16, table_stride=4, max_pages=4, page_stride=2048, slot=128, head=64):
    return api._Pages(key, value, table, lens, n_seg, n_pages, page_size, table_stride, max_pages, page_stride, slot, head)


def test_paged_arguments(api):
    L, h = api.load_library(), heads(api)

    def call(c, q=256, start=256, n=10, out=256, lse=256, ws=256, size=BIG):
        return L.tiga_apply_paged_attention(REF(c), REF(h), q, start, n, 1, out, lse, ws, size, None)
    for bad in (dict(page_size=0), dict(n_pages=-1), dict(max_pages=-1), dict(table_stride=-1), dict(slot=100), dict(page_stride=-8), dict(head=4), dict(n_seg=-1),
                dict(key=None), dict(value=264), dict(table=None), dict(lens=None), dict(table=258)):
        assert call(pages(api, **bad)) == 1, bad
    assert call(pages(api, page_size=1 << 25)) == 2
    assert call(pages(api), q=None) == 1 and call(pages(api), start=None) == 1 and call(pages(api), out=264) == 1 and call(pages(api), n=-1) == 1
    assert call(pages(api), size=8) == 3 and call(pages(api), n=0) == 0 and call(pages(api, n_seg=0)) == 0

    def append(c, key=256, value=256, start=256, n=10, r=None, hh=h):
        return L.tiga_paged_append(REF(c), REF(hh), key, value, start, n, r, None)
    for bad in (dict(slot=0), dict(head=0), dict(page_stride=0), dict(key=None), dict(table=None), dict(lens=None)):
        assert append(pages(api, **bad)) == 1, bad
    assert append(pages(api), key=None) == 1 and append(pages(api), value=264) == 1 and append(pages(api), start=None) == 1 and append(pages(api), n=-1) == 1
    assert append(pages(api), hh=heads(api, key=(128, 4))) == 1 and append(pages(api), n=1 << 31) == 2 and append(pages(api), n=0) == 0
    for turned, layout, m, freq in ((0, 0, 1.0, 256), (3, 0, 1.0, 256), (66, 0, 1.0, 256), (32, 2, 1.0, 256), (32, 0, float("nan"), 256), (32, 0, 1.0, None), (32, 0, 1.0, 260)):
        assert append(pages(api), r=REF(api._Rotary(freq, turned, layout, m))) == 1


def test_rotary_arguments(api):
    L, s = api.load_library(), api._Stride

    def call(r=(256, 32, 0, 1.0), x=256, xs=(256, 64), y=512, ys=(256, 64), dtype=1, n=4, h=4, D=64, pos=256, kind=0):
        return L.tiga_apply_rotary(REF(api._Rotary(*r)), x, REF(s(*xs)), y, REF(s(*ys)), dtype, n, h, D, pos, kind, 0, None)
    for bad in (dict(r=(None, 32, 0, 1.0)), dict(r=(256, 31, 0, 1.0)), dict(r=(256, 66, 0, 1.0)), dict(r=(256, 32, 5, 1.0)), dict(r=(256, 32, 0, float("inf"))), dict(x=None),
                dict(y=513), dict(dtype=3), dict(n=-1), dict(h=0), dict(D=0), dict(pos=None), dict(pos=260, kind=1), dict(kind=2), dict(xs=(-1, 64)), dict(ys=(0, 64)),
                dict(ys=(256, 0)), dict(x=512, ys=(512, 64))):
        assert call(**bad) == 1, bad
    assert call(n=0, x=None, y=None, pos=None) == 0


def test_frequencies(api):
    f, m = api.tiga_rotary_frequencies(8, base=10000.0)
    assert m == 1.0 and torch.allclose(f, torch.tensor([1.0, 0.1, 0.01, 0.001], dtype=torch.float64), rtol=1e-14, atol=0)
    g, m = api.tiga_rotary_frequencies(8, scaling=api.ROT_LINEAR, factor=4.0)
    assert m == 1.0 and torch.allclose(g, f / 4, rtol=1e-14, atol=0)
    g, m = api.tiga_rotary_frequencies(8, scaling=api.ROT_BASE, factor=4.0)
    assert torch.allclose(g[[0, 3]], torch.stack([f[0], f[3] / 4]), rtol=1e-13, atol=0)      # the first pair stays, the last is interpolated in full
    g, m = api.tiga_rotary_frequencies(64, scaling=api.ROT_BANDS, factor=8.0, length=4096.0, slow=1.0, fast=32.0)
    f, _ = api.tiga_rotary_frequencies(64)
    r = 4096 * f / (2 * math.pi)
    assert abs(m - (0.1 * math.log(8) + 1)) < 1e-7
    assert torch.equal(g[r > 32], f[r > 32]) and torch.allclose(g[r < 1], f[r < 1] / 8, rtol=1e-14, atol=0)
    mid = (r > 1) & (r < 32)
    keep = (r - 1) / 31
    assert mid.any() and torch.allclose(g[mid], (keep * f + (1 - keep) * f / 8)[mid], rtol=1e-13, atol=0)
    for bad in (dict(turned=0), dict(turned=3), dict(turned=8, base=0.0), dict(turned=8, base=float("inf")), dict(turned=8, scaling=4), dict(turned=8, scaling=1, factor=0.5),
                dict(turned=2, scaling=2, factor=2.0), dict(turned=8, scaling=3, factor=2.0, length=0.0), dict(turned=8, scaling=3, factor=2.0, length=10.0, slow=3.0, fast=3.0)):
        with pytest.raises(api.TigaError) as e:
            api.tiga_rotary_frequencies(**bad)
        assert e.value.status == 1, bad


def test_arrays_on_the_host_are_refused(api):
    x = torch.zeros(4, 2, 64, dtype=torch.float16)
    start = torch.tensor([0, 4], dtype=torch.int32)
    with pytest.raises(ValueError):
        api.tiga_apply_dense_attention(api.DenseRelation(start, start), x, x, x, 1.0)
    with pytest.raises(ValueError):
        api.Rotary(torch.ones(4, dtype=torch.float64))
    with pytest.raises(ValueError):
        api.DenseRelation(start, torch.tensor([0, 4, 5], dtype=torch.int32))
    with pytest.raises(ValueError):
        api.DenseRelation(start.long(), start)
    with pytest.raises(ValueError):
        api.PagedCache(torch.zeros(2, 16, 2, 64), torch.zeros(2, 16, 2, 64), torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
