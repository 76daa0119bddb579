"""Descriptors of dense and paged relations: what they refuse when they are made, without a device."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def api():
    from paper_2609_24802_b200 import build
    build.build_library()
    from paper_2609_24802_b200 import api
    return api


def pages(n_pages=3, page=16, heads=2, D=64, dtype=torch.float16):
    return torch.zeros(n_pages, page, heads, D, dtype=dtype)


def places(n_seg=1, max_pages=2):
    return torch.zeros(n_seg, max_pages, dtype=torch.int32), torch.zeros(n_seg, dtype=torch.int32)


def test_pages_whose_features_share_storage_are_refused(api):
    """One element seen as D features: the kernels would read, and write, D elements per slot."""
    thin = pages(D=8)[..., :1].expand(3, 16, 2, 64)
    assert thin.stride() == (256, 16, 8, 0)
    for key, value in ((thin, thin), (thin, pages()), (pages(), thin)):
        with pytest.raises(ValueError):
            api.PagedCache(key, value, *places())
    apart = pages(D=128)[..., ::2]
    with pytest.raises(ValueError):
        api.PagedCache(apart, apart, *places())


def test_pages_in_any_order_of_slots_and_heads_are_taken(api):
    for t in (pages(), pages(page=2, heads=16).transpose(1, 2), pages(D=128)[..., 64:], pages(n_pages=1), pages(page=1), pages(heads=1), pages(n_pages=0)):
        cache = api.PagedCache(t, t, *places())
        assert (cache.c.n_pages, cache.c.page_size) == t.shape[:2]


def test_a_table_with_entries_needs_an_address(api):
    """(Without entries it may have none: nothing of it is read.)"""
    L, s, ref = api.load_library(), api._Stride, ctypes.byref
    h = api._Heads(1, 4, 2, 64, 1.0, s(256, 64), s(128, 64), s(128, 64), s(256, 64))

    def call(max_pages, table, size):
        c = api._Pages(256, 256, table, 256, 2, 8, 16, 4, max_pages, 2048, 128, 64)
        return L.tiga_apply_paged_attention(ref(c), ref(h), 256, 256, 10, 1, 256, 256, 256, size, None)
    assert call(4, None, 1 << 40) == 1 and call(4, 258, 1 << 40) == 1
    assert call(0, None, 16) == 3               # goes on to the next check: the workspace is too small


def test_arrays_of_a_descriptor_are_written_into_not_replaced(api):
    """The descriptor keeps addresses: with another array in its place it would go on reading the old one."""
    cache = api.PagedCache(pages(), pages(), *places())
    for name in ("key", "value", "table", "kv_len"):
        with pytest.raises(AttributeError):
            setattr(cache, name, getattr(cache, name).clone())
    kv_len = cache.kv_len
    cache.kv_len += 3
    cache.kv_len[0] += 1
    assert cache.kv_len is kv_len and kv_len.tolist() == [4] and cache.c.kv_len == kv_len.data_ptr()
    start = torch.tensor([0, 4], dtype=torch.int32)
    relation = api.DenseRelation(start, start.clone())
    for name, other in (("q_start", start.clone()), ("kv_start", start), ("mask", torch.ones(4, dtype=torch.bool))):
        with pytest.raises(AttributeError):
            setattr(relation, name, other)
    relation.note = cache.note = "anything else may be kept here"
    assert relation.q_start is start and relation.mask is None
