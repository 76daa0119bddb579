"""Eviction writes its target by many warps at once: rows of `to` that lie in one another are refused, whatever the strides; layouts whose
rows lie apart are written as any other."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

REF = ctypes.byref


@pytest.fixture(scope="module")
def api():
    from paper_2609_24802_b200 import build
    build.build_library()
    from paper_2609_24802_b200 import api
    return api


# strides of a page, a slot and a head; 8 pages of 16 slots, 2 heads of 64
OVERLAPPING = [(2048, 128, 56), (2048, 120, 64), (2040, 128, 64), (2048, 64, 128), (2048, 64, 64), (1920, 128, 64), (2048, 128, 1984), (64, 1024, 512 - 8), (64, 1024, 8192), (0, 128, 64),
               (2048, 0, 64), (2048, 128, 0), (1 << 62, 128, 56), (1 << 62, 1 << 62, 0)]


@pytest.mark.parametrize("page,slot,head", OVERLAPPING)
def test_rows_in_one_another_are_refused(api, page, slot, head):
    L, s = api.load_library(), api._Stride(0, 0)
    heads = api._Heads(1, 2, 2, 64, 1.0, s, s, s, s)
    cache = api._Pages(256, 256, 256, 256, 2, 8, 16, 4, 4, 2048, 128, 64)
    to = api._Pages(256, 256, 256, None, 2, 8, 16, 4, 4, page, slot, head)
    assert L.tiga_paged_evict(REF(cache), REF(to), REF(heads), REF(api._Weights(512, 200, 100, 64)), 32, 4, None, 1024, 256, None) == 1


def target(kind, n, page, heads, D, dtype):
    """Key and value pages [n, page, heads, D] in arrays of their own, or in one another's gaps."""
    def zeros(*shape):
        return torch.zeros(shape, dtype=dtype, device="cuda")
    if kind == "heads in front":
        return [zeros(n, heads, page, D).transpose(1, 2) for _ in range(2)]
    if kind == "key beside value":
        both = zeros(n, page, heads, 2, D)
        return [both[:, :, :, i] for i in range(2)]
    if kind == "value behind key in a page":
        both = zeros(n, 2, page, heads, D)
        return [both[:, i] for i in range(2)]
    if kind == "pages innermost":
        return [zeros(page, heads, n, D).permute(2, 0, 1, 3) for _ in range(2)]
    if kind == "gaps":
        return [zeros(n + 1, page + 3, heads + 2, D + 8)[:n, 2:2 + page, 1:1 + heads, :D] for _ in range(2)]
    return [zeros(1, page, 1, D) for _ in range(2)]             # a single page and head, whose strides mean nothing


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["heads in front", "key beside value", "value behind key in a page", "pages innermost", "gaps", "single"])
def test_rows_that_lie_apart(api, kind):
    from test_gpu_evict import make, plain
    single = kind == "single"
    c = make([100] if single else [300, 50, 120], 1 if single else 2, 64, torch.bfloat16, 16, 64 if single else 16, 64, seed=31)
    to = target(kind, c["to_key"].shape[0], c["to_key"].shape[1], c["to_key"].shape[2], 64, torch.bfloat16)
    if single:
        c["to_key"], c["to_value"], c["to_table"] = c["to_key"][:1], c["to_value"][:1], torch.zeros_like(c["to_table"])
    for t, name in zip(to, ("to_key", "to_value")):
        t.copy_(c[name])
    key, value, kept, left, new = plain(c, 64, 9)
    cache = api.PagedCache(c["key"], c["value"], c["table"], c["lens"])
    got, got_left = api.tiga_paged_evict(cache, api.PagedCache(*to, c["to_table"], c["to_lens"]), c["weights"], 64, 9)
    assert torch.equal(got, kept) and torch.equal(got_left, left) and torch.equal(c["to_lens"], new)
    assert torch.equal(to[0].contiguous().view(torch.int16), key) and torch.equal(to[1].contiguous().view(torch.int16), value)
