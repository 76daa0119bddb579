"""The operators of a decoder together, as a program uses them: packed prompts through the triangle and into a cache, users that share a
prompt, the weights that their positions receive, eviction, and on with what is left.  Every stage against 64 bits on what the stage in front
left behind (tolerances: attention_reference.py)."""
import pytest

from attention_reference import attend, close, turn
from test_gpu_evict import plain

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

HEADS, KV, D, PAGE = 4, 2, 64, 16
SCALE = D ** -0.5


@pytest.fixture(scope="module")
def tiga():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_24802_b200 import api
    return api


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def triangle(n, m):
    return torch.arange(m, device="cuda")[None] <= m - n + torch.arange(n, device="cuda")[:, None]


def of_sequence(cache, s):
    """Keys and values of a sequence, [tokens, kv_heads, D]."""
    n, pages = int(cache.kv_len[s]), cache.table[s].long()
    return [t[pages].flatten(0, 1)[:n] for t in (cache.key, cache.value)]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_prompt_users_weights_and_eviction(tiga, dtype):
    g = torch.Generator(device="cuda").manual_seed(7)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(dtype)  # noqa: E731
    freq, _ = tiga.tiga_rotary_frequencies(D)
    rotary = tiga.Rotary(freq.cuda())
    # two prompts in one batch
    lens = [70, 133]
    start = ints(0, 70, 203)
    q, k, v = normal(203, HEADS, D), normal(203, KV, D), normal(203, KV, D)
    positions = torch.cat([torch.arange(n) for n in lens]).to(torch.int32).cuda()
    rq, rk = tiga.tiga_apply_rotary(rotary, q, positions), tiga.tiga_apply_rotary(rotary, k, positions)
    out, lse, _ = tiga.tiga_apply_triangular_attention(tiga.TriangularRelation(start), rq, rk, v, SCALE)
    pool = [torch.full((40, PAGE, KV, D), float("nan"), dtype=dtype, device="cuda") for _ in range(2)]
    order = torch.randperm(40, generator=torch.Generator().manual_seed(1)).to(torch.int32)
    prompts = tiga.PagedCache(*pool, torch.stack([order[:9], order[9:18]]).cuda(), ints(*lens))
    tiga.tiga_paged_append(prompts, k, v, start, rotary=rotary)
    paged, paged_lse, _ = tiga.tiga_apply_paged_attention(prompts, rq, start, SCALE)
    for s, (a, b) in enumerate(((0, 70), (70, 203))):
        keys, values = of_sequence(prompts, s)
        assert torch.equal(keys, rk[a:b]) and torch.equal(values, v[a:b])
        want = attend(rq[a:b], keys, values, SCALE, triangle(b - a, b - a))
        for got, name in ((out, "out"), (paged, "out"), (lse, "lse"), (paged_lse, "lse")):
            close(got[a:b], want[name], want[name + "_tol"], name)

    # three users go on from the second prompt: its eight whole pages are theirs together, the page behind them is copied for each
    own = order[18:30].reshape(3, 4)
    for u in range(3):
        for t in pool:
            t[int(own[u, 0]), :5] = t[int(order[17]), :5]
    users = tiga.PagedCache(*pool, torch.cat([order[9:17].expand(3, 8), own], 1).contiguous().cuda(), ints(133, 133, 133))
    prefixes = tiga.SharedPrefixes(ints(0, 3), ints(128))
    weights = torch.zeros(3, KV, 12 * PAGE, device="cuda")
    total, tol = weights.double(), weights.double()
    each = ints(0, 1, 2, 3)
    for step in range(12):
        users.kv_len += 1
        q, k, v = normal(3, HEADS, D), normal(3, KV, D), normal(3, KV, D)
        rq = tiga.tiga_apply_rotary(rotary, q, users.kv_len - 1)
        tiga.tiga_paged_append(users, k, v, each, rotary=rotary)
        out, lse, _ = tiga.tiga_apply_shared_attention(users, prefixes, rq, each, SCALE)
        tiga.tiga_paged_attention_weights(users, rq, each, lse, SCALE, before=weights, weights=weights)
        for u in range(3):
            keys, values = of_sequence(users, u)
            n = len(keys)
            assert n == 134 + step
            want = attend(rq[u:u + 1], keys, values, SCALE, torch.ones(1, n, dtype=torch.bool, device="cuda"))
            close(out[u:u + 1], want["out"], want["out_tol"], "out")
            close(lse[u:u + 1], want["lse"], want["lse_tol"], "lse")
            p = torch.exp(torch.einsum("hd,mhd->hm", rq[u].double(), keys.double().repeat_interleave(2, 1)) * SCALE - want["lse"][0][:, None])
            total[u, :, :n] += p.reshape(KV, 2, n).sum(1)
            # a weight is off by 2^-22 for each of its score, lse and exponential (scores here are below 8), and by what lse is
            tol[u, :, :n] += (p * (16 * 2.0 ** -20 + 2 * want["lse_tol"][0][:, None])).reshape(KV, 2, n).sum(1) + total[u, :, :n] * 2.0 ** -23
    close(weights, total, tol + 2.0 ** -120, "weights")

    # cut to 60 positions each, in pages of another size
    room = [torch.full((3 * 8, 8, KV, D), float("nan"), dtype=dtype, device="cuda") for _ in range(2)]
    left = tiga.PagedCache(*room, torch.randperm(24, generator=torch.Generator().manual_seed(2)).to(torch.int32).reshape(3, 8).cuda(), ints(0, 0, 0))
    want = plain(dict(key=pool[0], value=pool[1], table=users.table, lens=users.kv_len, to_key=room[0], to_value=room[1], to_table=left.table, weights=weights), 60, 16)
    kept, left_weights = tiga.tiga_paged_evict(users, left, weights, 60, 16)
    assert torch.equal(kept, want[2]) and torch.equal(left_weights[:, :, :60], want[3][:, :, :60]) and left.kv_len.tolist() == [60, 60, 60]
    assert torch.equal(room[0].view(torch.int16), want[0]) and torch.equal(room[1].view(torch.int16), want[1])

    # and on: the next token has its own position, its key is rotated in front of the write
    q, k, v = normal(3, HEADS, D), normal(3, KV, D), normal(3, KV, D)
    now = users.kv_len.clone()
    left.kv_len += 1
    rq, rk = tiga.tiga_apply_rotary(rotary, q, now), tiga.tiga_apply_rotary(rotary, k, now)
    exact, size = turn(k, now, freq, 1.0, False)
    assert bool(((rk.double() - exact).abs() <= size * 2.0 ** -7 + 1e-6).all())
    tiga.tiga_paged_append(left, rk, v, each)
    out, lse, _ = tiga.tiga_apply_paged_attention(left, rq, each, SCALE)
    tiga.tiga_paged_attention_weights(left, rq, each, lse, SCALE, before=left_weights, weights=left_weights)
    for u in range(3):
        old = of_sequence(users, u)
        at = kept[u].long()                 # per head
        keys, values = (torch.cat([torch.stack([t[at[h], h] for h in range(KV)], 1), new[u:u + 1]]) for t, new in zip(old, (rk, v)))
        want = attend(rq[u:u + 1], keys, values, SCALE, torch.ones(1, 61, dtype=torch.bool, device="cuda"))
        close(out[u:u + 1], want["out"], want["out_tol"], "out")
        close(lse[u:u + 1], want["lse"], want["lse_tol"], "lse")
    assert torch.all(left_weights[:, :, 60] > 0) and torch.all(left_weights[:, :, 61:] == 0)


def test_what_python_refuses_on_the_device(tiga):
    q, start = torch.zeros(2, HEADS, D, dtype=torch.float16, device="cuda"), ints(0, 1, 2)
    page = torch.zeros(4, PAGE, KV, D, dtype=torch.float16, device="cuda")
    cache = tiga.PagedCache(page, page, torch.zeros(2, 2, dtype=torch.int32, device="cuda"), ints(3, 3))
    to = tiga.PagedCache(page.clone(), page.clone(), torch.zeros(2, 1, dtype=torch.int32, device="cuda"), ints(0, 0))
    lse, w = torch.zeros(2, HEADS, device="cuda"), torch.zeros(2, KV, 32, device="cuda")
    prefixes = tiga.SharedPrefixes(ints(0, 2), ints(0))
    for bad in (lambda: tiga.tiga_apply_shared_attention(cache, prefixes, q.bfloat16(), start, 1.0), lambda: tiga.tiga_apply_shared_attention(cache, prefixes, q, start[:2], 1.0),
                lambda: tiga.tiga_paged_attention_weights(cache, q, start, lse.double(), 1.0), lambda: tiga.tiga_paged_attention_weights(cache, q, start, lse[:1], 1.0),
                lambda: tiga.tiga_paged_attention_weights(cache, q, start, lse, 1.0, weights=w[:1]), lambda: tiga.tiga_paged_attention_weights(cache, q, start, lse.cpu(), 1.0),
                lambda: tiga.tiga_paged_evict(cache, tiga.PagedCache(page.bfloat16(), page.bfloat16(), to.table, to.kv_len), w, 4),
                lambda: tiga.tiga_paged_evict(cache, to, w, 4, kept=torch.zeros(2, KV, 5, dtype=torch.int32, device="cuda")),
                lambda: tiga.tiga_paged_evict(cache, to, w.cpu(), 4)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: tiga.tiga_paged_evict(cache, to, w, 0), lambda: tiga.tiga_paged_evict(cache, to, w, 17), lambda: tiga.tiga_paged_evict(cache, to, w, 4, 5),
                lambda: tiga.tiga_paged_evict(cache, cache, w, 4), lambda: tiga.tiga_paged_evict(cache, to, w, 4, to_weights=w)):
        with pytest.raises(tiga.TigaError):
            bad()
    with pytest.raises(TypeError):
        tiga.tiga_apply_triangular_attention(tiga.DenseRelation(start, start), q, q, q, 1.0)
    with pytest.raises(TypeError):
        tiga.tiga_apply_dense_attention(tiga.TriangularRelation(start), q, q, q, 1.0)


def test_no_rows_and_no_sequences(tiga):
    none = torch.zeros(0, HEADS, D, dtype=torch.float16, device="cuda")
    page = torch.zeros(4, PAGE, KV, D, dtype=torch.float16, device="cuda")
    out, lse, _ = tiga.tiga_apply_triangular_attention(tiga.TriangularRelation(ints(0, 0)), none, none, none, 1.0)
    assert out.shape == none.shape and lse.shape == (0, HEADS)
    cache = tiga.PagedCache(page, page, torch.zeros(2, 2, dtype=torch.int32, device="cuda"), ints(20, 0))
    out, lse, _ = tiga.tiga_apply_shared_attention(cache, tiga.SharedPrefixes(ints(0, 2), ints(16)), none, ints(0, 0, 0), 1.0)
    assert out.shape == none.shape
    before = torch.rand(2, KV, 32, device="cuda")
    w, _ = tiga.tiga_paged_attention_weights(cache, none, ints(0, 0, 0), lse, 1.0, before=before)
    assert torch.equal(w[0, :, :20], before[0, :, :20]) and torch.all(w[0, :, 20:] == 0) and torch.all(w[1] == 0)
    empty = tiga.PagedCache(page, page, torch.zeros(0, 2, dtype=torch.int32, device="cuda"), ints())
    kept, left = tiga.tiga_paged_evict(empty, empty, torch.zeros(0, KV, 32, device="cuda"), 4)
    assert kept.shape == (0, KV, 4)
    torch.cuda.synchronize()
