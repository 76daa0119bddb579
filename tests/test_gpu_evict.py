"""Eviction from a paged cache: which positions stay is a matter of whole numbers, and rows move as they are, so everything is compared
exactly with a plain restatement."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def tiga():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_24802_b200 import api
    return api


def make(lens, kv_heads, D, dtype, page, to_page, keep, seed=0, kind="spread", places=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, per, room = len(lens), max(1, -(-max(lens) // page)), -(-keep // to_page)
    bits = torch.int16
    draw = lambda shape: torch.randint(-30000, 30000, shape, generator=g, device="cuda", dtype=bits)  # noqa: E731
    c = dict(key=draw((B * per + 2, page, kv_heads, D)).view(dtype), value=draw((B * per + 2, page, kv_heads, D)).view(dtype),
             table=torch.randperm(B * per + 2, generator=g, device="cuda")[:B * per].to(torch.int32).reshape(B, per).contiguous(),
             lens=torch.tensor(lens, dtype=torch.int32, device="cuda"),
             to_key=draw((B * room + 1, to_page, kv_heads, D)).view(dtype), to_value=draw((B * room + 1, to_page, kv_heads, D)).view(dtype),
             to_table=torch.randperm(B * room + 1, generator=g, device="cuda")[:B * room].to(torch.int32).reshape(B, room).contiguous(),
             to_lens=torch.full((B,), -5, dtype=torch.int32, device="cuda"))
    w = torch.randn((B, kv_heads, per * page if places is None else places), generator=g, device="cuda")
    if kind == "spread":
        w = torch.exp(3 * w) * (torch.rand(w.shape, generator=g, device="cuda") < 0.9)
    elif kind == "ties":
        w = torch.randint(0, 4, w.shape, generator=g, device="cuda").float()
    elif kind == "near":            # neighbours in the last digits
        w = (torch.full_like(w, 1.0).view(torch.int32) + torch.randint(0, 3000, w.shape, generator=g, device="cuda", dtype=torch.int32)).view(torch.float32)
    c["weights"] = w.contiguous()
    return c


def order(w):
    """A key that grows with the weight; NaN in front of everything."""
    return -math.inf if math.isnan(w) else w


def plain(c, keep, recent):
    B, hk, W = c["weights"].shape
    page, to_page = c["key"].shape[1], c["to_key"].shape[1]
    table, to_table, lens = c["table"].tolist(), c["to_table"].tolist(), c["lens"].tolist()
    weights = c["weights"].tolist()
    key, value = c["to_key"].view(torch.int16).clone(), c["to_value"].view(torch.int16).clone()
    kept = torch.full((B, hk, keep), -1, dtype=torch.int32)
    left = torch.zeros((B, hk, c["to_table"].shape[1] * to_page))
    new = []
    move = []
    for b in range(B):
        for h in range(hk):
            there = [j for j in range(min(max(lens[b], 0), len(table[b]) * page)) if 0 <= table[b][j // page] < c["key"].shape[0]]
            w = lambda j: weights[b][h][j] if j < W else 0.0  # noqa: E731
            last = [j for j in there if j >= lens[b] - recent]
            rest = sorted((j for j in there if j < lens[b] - recent), key=lambda j: (0 if not math.isnan(w(j)) else 1, -order(w(j)), j))
            stay = sorted(last + rest[:keep - len(last)]) if len(there) > keep else there
            for r, j in enumerate(stay):
                kept[b, h, r] = j
                left[b, h, r] = w(j)
                if 0 <= to_table[b][r // to_page] < key.shape[0]:
                    move.append((to_table[b][r // to_page], r % to_page, h, table[b][j // page], j % page))
        new.append(len(stay))
    if move:
        m = torch.tensor(move, device="cuda").T
        key[m[0], m[1], m[2]] = c["key"].view(torch.int16)[m[3], m[4], m[2]]
        value[m[0], m[1], m[2]] = c["value"].view(torch.int16)[m[3], m[4], m[2]]
    return key, value, kept.cuda(), left.cuda(), torch.tensor(new, dtype=torch.int32, device="cuda")


def check(tiga, c, keep, recent):
    key, value, kept, left, new = plain(c, keep, recent)
    source = [c[x].clone() for x in ("key", "value", "table", "lens", "weights")]
    cache, to = tiga.PagedCache(c["key"], c["value"], c["table"], c["lens"]), tiga.PagedCache(c["to_key"], c["to_value"], c["to_table"], c["to_lens"])
    got_kept, got_left = tiga.tiga_paged_evict(cache, to, c["weights"], keep, recent)
    assert torch.equal(c["to_lens"], new)
    assert torch.equal(got_kept, kept)
    same = lambda a, b: torch.equal(a.contiguous().view(torch.int32 if a.dtype is torch.float32 else torch.int16), b.contiguous().view(torch.int32 if b.dtype is torch.float32 else torch.int16))  # noqa: E731
    assert torch.equal(torch.nan_to_num(got_left, nan=-9.0), torch.nan_to_num(left, nan=-9.0))
    assert torch.equal(c["to_key"].view(torch.int16), key) and torch.equal(c["to_value"].view(torch.int16), value)
    for x, old in zip(("key", "value", "lens", "weights"), (source[0], source[1], source[3], source[4])):
        assert torch.equal(c[x], old) if x == "lens" else same(c[x], old), "what is read stays as it is"
    return got_kept


@pytest.mark.parametrize("kind", ["spread", "ties", "near"])
@pytest.mark.parametrize("lens,page,to_page,keep,recent", [([1], 16, 16, 1, 0), ([1], 16, 16, 1, 1), ([0, 5], 8, 8, 3, 1), ([100], 16, 16, 100, 10), ([100], 16, 16, 99, 0), ([100, 30, 31, 33], 16, 8, 32, 32),
                                                           ([777], 16, 32, 256, 64), ([1000, 3, 500], 7, 48, 100, 7), ([2500], 64, 128, 2049, 1), ([5000, 4097], 128, 16, 1000, 300)])
def test_lengths_pages_and_budgets(tiga, lens, page, to_page, keep, recent, kind):
    check(tiga, make(lens, 2, 64, BF16, page, to_page, keep, seed=len(lens) + page, kind=kind), keep, recent)


@pytest.mark.parametrize("kv_heads,D,dtype", [(1, 8, F16), (3, 16, BF16), (2, 40, F16), (8, 128, BF16), (5, 72, BF16), (4, 96, F16), (1, 120, F16)])
def test_heads_and_widths(tiga, kv_heads, D, dtype):
    check(tiga, make([300, 65], kv_heads, D, dtype, 16, 16, 70, seed=D), 70, 9)


@pytest.mark.parametrize("kind", ["spread", "ties", "near"])
def test_long_lists_are_shared_by_a_cluster(tiga, kind):
    """More than 8192 places and few lists: eight blocks a list; and lists that shared memory does not hold."""
    check(tiga, make([20011, 300], 2, 8, F16, 16, 64, 5000, seed=3, kind=kind), 5000, 100)
    check(tiga, make([20011], 1, 8, F16, 16, 64, 20011, seed=4, kind=kind), 20011, 100)


def test_lists_that_shared_memory_does_not_hold(tiga):
    check(tiga, make([50021] + [100] * 40, 1, 8, F16, 64, 64, 300, seed=5), 300, 20)
    check(tiga, make([350021], 1, 8, F16, 64, 64, 1000, seed=6), 1000, 20)


def test_special_weights(tiga):
    c = make([64], 2, 16, F16, 16, 16, 40, seed=7)
    w = c["weights"]
    w[0, 0, :] = 0.0
    w[0, 0, ::2] = -0.0                     # equal to zero: the lower position stays
    w[0, 0, 60] = float("inf")
    w[0, 1, :] = float("nan")
    w[0, 1, 5:30] = -float("inf")
    w[0, 1, 31] = -3.0
    kept = check(tiga, c, 40, 2)
    assert kept[0, 0].tolist() == list(range(37)) + [60, 62, 63]


def test_fewer_weights_than_positions(tiga):
    check(tiga, make([300], 2, 64, BF16, 16, 16, 100, seed=8, places=50), 100, 10)


def test_missing_pages(tiga):
    """Positions without a page are not kept; places without one are not written."""
    c = make([200, 90], 2, 64, BF16, 16, 16, 64, seed=9)
    c["table"][0, 2], c["table"][0, 12], c["table"][1, 0] = -1, 1 << 20, -7
    c["to_table"][0, 1], c["to_table"][1, 3] = -1, 99999
    check(tiga, c, 64, 20)
    c = make([200, 90], 2, 64, BF16, 16, 16, 64, seed=10)
    c["table"][1] = -1
    check(tiga, c, 64, 20)
    c = make([200], 1, 64, BF16, 16, 16, 64, seed=11)
    c["lens"][0] = 5000                     # longer than its table
    check(tiga, c, 64, 64)
    c["lens"][0] = -3
    check(tiga, c, 64, 64)


def test_heads_in_front_and_both_caches_in_the_same_arrays(tiga):
    c = make([150, 40], 3, 64, F16, 16, 16, 48, seed=12)
    n = c["key"].shape[0]
    want = plain(c, 48, 8)
    pool = [torch.cat([c[a], c["to_" + a]]).transpose(1, 2).contiguous().transpose(1, 2) for a in ("key", "value")]
    cache = tiga.PagedCache(*pool, c["table"], c["lens"])
    to = tiga.PagedCache(*pool, c["to_table"] + n, c["to_lens"])
    kept, left = tiga.tiga_paged_evict(cache, to, c["weights"], 48, 8)
    assert torch.equal(pool[0][n:].contiguous().view(torch.int16), want[0]) and torch.equal(pool[1][n:].contiguous().view(torch.int16), want[1])
    assert torch.equal(kept, want[2]) and torch.equal(left, want[3])


def test_captured_and_replayed_with_other_lengths(tiga):
    c = make([150, 40], 2, 64, F16, 16, 16, 48, seed=13)
    cache, to = tiga.PagedCache(c["key"], c["value"], c["table"], c["lens"]), tiga.PagedCache(c["to_key"], c["to_value"], c["to_table"], c["to_lens"])
    kept, left = tiga.tiga_paged_evict(cache, to, c["weights"], 48, 8)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tiga.tiga_paged_evict(cache, to, c["weights"], 48, 8, kept=kept, to_weights=left)
    c["lens"].copy_(torch.tensor([60, 100], dtype=torch.int32))
    want = plain(c, 48, 8)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(kept, want[2]) and torch.equal(left, want[3]) and torch.equal(c["to_lens"], want[4])
    assert torch.equal(c["to_key"].view(torch.int16), want[0])


def test_on_another_stream(tiga):
    c = make([150, 40], 2, 64, F16, 16, 16, 48, seed=14)
    want = plain(c, 48, 8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    cache, to = tiga.PagedCache(c["key"], c["value"], c["table"], c["lens"]), tiga.PagedCache(c["to_key"], c["to_value"], c["to_table"], c["to_lens"])
    kept, left = tiga.tiga_paged_evict(cache, to, c["weights"], 48, 8, stream=side)
    side.synchronize()
    assert torch.equal(kept, want[2]) and torch.equal(left, want[3]) and torch.equal(c["to_value"].view(torch.int16), want[1])


@pytest.mark.parametrize("kind", ["spread", "ties", "near"])
def test_many_lists(tiga, kind):
    """More lists than the device has SMs: small blocks."""
    check(tiga, make([1 + (i * 53) % 900 for i in range(90)], 2, 8, F16, 16, 16, 200, seed=15, kind=kind), 200, 30)


@pytest.mark.parametrize("page", [1, 3, 5, 24, 31, 33, 63, 65, 100])
def test_page_sizes(tiga, page):
    """Pages of odd sizes, some of them missing: every position is looked up in its own page, whatever the sizes of the steps along a list."""
    for seed, lens in ((17, [1200, 40, 0, 333]), (18, [9000])):             # a block a list, a cluster
        c = make(lens, 2, 8, F16, page, 16, 250, seed=seed)
        g = torch.Generator(device="cuda").manual_seed(seed)
        c["table"][torch.rand(c["table"].shape, generator=g, device="cuda") < 0.3] = -1
        check(tiga, c, 250, 40)


def test_pages_beyond_32_bits(tiga):
    """Pages whose elements lie behind the 2^31st."""
    stride = (1 << 31) // 3 + 8 - ((1 << 31) // 3) % 8
    raw = [torch.empty(4 * stride + 4096, dtype=BF16, device="cuda") for _ in range(2)]
    pool = [torch.as_strided(t, (5, 16, 2, 64), (stride, 128, 64, 1)) for t in raw]
    c = make([60], 2, 64, BF16, 16, 16, 20, seed=16)
    for t, name in zip(pool, ("key", "value")):
        t[1:].copy_(c[name][c["table"][0].long()].flip(0))
    want = plain(c, 20, 5)
    cache = tiga.PagedCache(*pool, torch.tensor([[4, 3, 2, 1]], dtype=torch.int32, device="cuda"), c["lens"])
    to = tiga.PagedCache(c["to_key"], c["to_value"], c["to_table"], c["to_lens"])
    kept, left = tiga.tiga_paged_evict(cache, to, c["weights"], 20, 5)
    assert torch.equal(kept, want[2]) and torch.equal(c["to_key"].view(torch.int16), want[0]) and torch.equal(c["to_value"].view(torch.int16), want[1])
