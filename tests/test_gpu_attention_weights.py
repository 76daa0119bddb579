"""GPU parity of the attention weights that cached positions receive, against 64 bits.

A weight exp(scale <q, k> - lse) is formed in fp32: the products are exact, their sum is off by (D + 8) 2^-23 of sum |q k|, the scaled
score, lse in base 2 and their difference by 2^-23 of |score| and |lse| each, the exponential by 2^-22; all of this is relative to the
weight.  A sum of n positive terms in fp32 adds n 2^-24 of itself.  Weights below 2^-126 are formed as zero."""
import pytest

from attention_reference import close
from parity import Guard

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def tiga():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_24802_b200 import api
    return api


def starts(lengths):
    s = [0]
    for n in lengths:
        s.append(s[-1] + n)
    return torch.tensor(s, dtype=torch.int32, device="cuda")


def normal(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def make(q_len, kv_len, heads, kv_heads, D, dtype, page, seed=0, spread=1.0):
    """A cache whose pages lie in any order; every slot that no sequence holds is NaN."""
    need = sum(-(-n // page) for n in kv_len)
    pages = torch.full((need + 2, page, kv_heads, D), float("nan"), dtype=dtype, device="cuda")
    order = torch.randperm(need + 2, generator=torch.Generator().manual_seed(seed)).tolist()
    table = torch.full((len(kv_len), max(1, max(-(-n // page) for n in kv_len)) + 1), -1, dtype=torch.int32)
    keys = []
    for b, n in enumerate(kv_len):
        keys.append(normal((n, kv_heads, D), dtype, 31 * seed + b + 1, spread))
        for i in range(-(-n // page)):
            table[b, i] = order.pop()
            m = min(page, n - i * page)
            pages[int(table[b, i]), :m] = keys[-1][i * page:i * page + m]
    return dict(q_len=q_len, kv_len=kv_len, q=normal((sum(q_len), heads, D), dtype, seed + 77, spread), pages=pages, table=table.cuda(), page=page,
                lens=torch.tensor(kv_len, dtype=torch.int32, device="cuda"), keys=keys, scale=D ** -0.5)


def seen_of(n, m, causal):
    at = torch.arange(m, device="cuda")
    return (at[None] <= m - n + torch.arange(n, device="cuda")[:, None]) if causal else torch.ones(n, m, dtype=torch.bool, device="cuda")


def masses(c, causal):
    """lse of the attention, rounded to fp32."""
    parts, q0 = [], 0
    for n, k in zip(c["q_len"], c["keys"]):
        q = c["q"][q0:q0 + n].double()
        s = torch.einsum("nhd,mhd->nhm", q, k.double().repeat_interleave(q.shape[1] // k.shape[1], 1)) * c["scale"]
        parts.append(torch.logsumexp(s.masked_fill(~seen_of(n, len(k), causal)[:, None], -float("inf")), -1) if len(k) else torch.full(q.shape[:2], -float("inf"), device="cuda"))
        q0 += n
    return torch.cat(parts).float().contiguous()


def reference(c, lse, causal, before, out):
    """What `out` holds afterwards, and how far the library may be from it."""
    want = out.double().clone()
    tol = torch.zeros_like(want)
    q0 = 0
    for b, (n, k) in enumerate(zip(c["q_len"], c["keys"])):
        m, hk, D = k.shape
        q, l = c["q"][q0:q0 + n].double(), lse[q0:q0 + n].double()
        kk = k.double().repeat_interleave(q.shape[1] // hk, 1)
        s = torch.einsum("nhd,mhd->nhm", q, kk) * c["scale"]
        size = torch.einsum("nhd,mhd->nhm", q.abs(), kk.abs()) * abs(c["scale"])
        reads = seen_of(n, m, causal)[:, None] & (l != -float("inf"))[..., None]
        p = torch.where(reads, torch.exp(s - l[..., None]), 0.0)
        off = (D + 8) * 2.0 ** -23 * size + 2.0 ** -22 * (s.abs() + torch.where(torch.isinf(l), 0.0, l.abs())[..., None]) + 2.0 ** -22
        fold = lambda t: t.reshape(n, hk, t.shape[1] // hk, m).sum((0, 2))  # noqa: E731
        w = min(m, out.shape[2])
        old = 0.0 if before is None else before[b, :, :w].double()
        want[b, :, :w] = (old + fold(p)[:, :w])
        rows = n * q.shape[1] // hk
        tol[b, :, :w] = (fold(torch.where(reads, p * off, 0.0)) + (rows + 4) * 2.0 ** -24 * fold(p))[:, :w] + 2.0 ** -24 * want[b, :, :w].abs() + rows * 2.0 ** -125
        q0 += n
    return want, tol


def check(tiga, c, causal=True, added=True, length=None, lse=None):
    cache = tiga.PagedCache(c["pages"], c["pages"], c["table"], c["lens"])
    lse = masses(c, causal) if lse is None else lse
    B, hk = len(c["kv_len"]), c["pages"].shape[2]
    W = c["table"].shape[1] * c["page"] if length is None else length
    before = torch.rand((B, hk, W), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda") if added else None
    results = []
    for _ in range(2):
        guard = Guard(torch)
        out = guard.empty((B, hk, W))
        out.fill_(-7.0)
        want, tol = reference(c, lse, causal, before, out)
        tiga.tiga_paged_attention_weights(cache, c["q"], starts(c["q_len"]), lse, c["scale"], causal=causal, before=before, weights=out,
                                          ws=guard.workspace(tiga.tiga_paged_weights_workspace_bytes(cache, c["q"])))
        guard.check()
        close(out, want, tol, "weights")
        results.append(out)
    assert torch.equal(*results), "reruns must be bit identical"
    if added:               # in place
        tiga.tiga_paged_attention_weights(cache, c["q"], starts(c["q_len"]), lse, c["scale"], causal=causal, before=before, weights=before)
        for b, n in enumerate(c["kv_len"]):
            assert torch.equal(before[b, :, :n], results[0][b, :, :n])
    return results[0]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("q_len,kv_len,page", [([1], [1], 16), ([1], [777], 16), ([1, 1, 1], [5, 300, 64], 1), ([1, 1], [129, 0], 8), ([5], [5], 16), ([130], [130], 48),
                                               ([128, 1, 33], [300, 1000, 33], 64), ([0, 7, 0], [10, 200, 0], 32), ([200], [515], 128), ([40, 3], [700, 131], 7),
                                               ([9], [300], 1000), ([600, 8, 9], [600, 300, 400], 16)])
def test_lengths_and_pages(tiga, q_len, kv_len, page, dtype):
    check(tiga, make(q_len, kv_len, 4, 2, 64, dtype, page, seed=page), added=dtype is F16)


@pytest.mark.parametrize("heads,kv_heads,D,dtype", [(1, 1, 8, F16), (8, 1, 64, BF16), (6, 2, 40, F16), (32, 8, 128, BF16), (5, 5, 96, F16), (40, 5, 72, BF16), (64, 1, 128, F16),
                                                    (144, 1, 64, BF16)])
def test_heads_and_widths(tiga, heads, kv_heads, D, dtype):
    check(tiga, make([1, 17, 2], [90, 150, 260], heads, kv_heads, D, dtype, 16, seed=D))


def test_without_the_triangle(tiga):
    check(tiga, make([70, 1, 5], [200, 30, 5], 4, 2, 64, F16, 16, seed=4), causal=False)


def test_more_new_tokens_than_cache(tiga):
    check(tiga, make([12], [5], 2, 2, 64, BF16, 16, seed=5))


def test_long_chunks_and_many_sequences(tiga):
    check(tiga, make([1], [30011], 8, 2, 128, BF16, 64, seed=6))
    check(tiga, make([1] * 70, [(i * 97) % 900 + 1 for i in range(70)], 8, 2, 64, F16, 16, seed=7))
    check(tiga, make([1500, 1, 1, 250], [2500, 2000, 3, 250], 8, 4, 128, F16, 32, seed=8))
    check(tiga, make([1 + i % 3 for i in range(300)], [4 + (i * 37) % 400 for i in range(300)], 4, 2, 64, BF16, 16, seed=17))


def test_fewer_places_than_positions(tiga):
    check(tiga, make([3, 2], [300, 50], 4, 2, 64, BF16, 16, seed=9), length=130)


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
def test_scales(tiga, scale):
    c = make([33], [300], 2, 1, 64, F16, 16, seed=10)
    c["scale"] = scale
    check(tiga, c)


def test_rows_that_read_nothing_and_pages_that_are_missing(tiga):
    c = make([40], [200], 2, 1, 64, BF16, 16, seed=11)
    lse = masses(c, True)
    lse[7] = -float("inf")
    c["q"][7] = float("nan")                # (a row that reads nothing: whatever it holds)
    lse[9, 1] = float("inf")                # weights of zero
    a = check(tiga, c, lse=lse)
    c["table"][0, 3] = -1
    c["table"][0, 5] = 1 << 20
    cache = tiga.PagedCache(c["pages"], c["pages"], c["table"], c["lens"])
    out, _ = tiga.tiga_paged_attention_weights(cache, c["q"], starts([40]), lse, c["scale"])
    gone = torch.zeros(200, dtype=torch.bool, device="cuda")
    gone[48:64] = gone[80:96] = True
    b, _ = tiga.tiga_paged_attention_weights(tiga.PagedCache(c["pages"], c["pages"], c["table"].clone().masked_fill_(c["table"] < 0, 0).clamp_(max=c["pages"].shape[0] - 1),
                                                             c["lens"]), c["q"], starts([40]), lse, c["scale"])
    assert torch.all(out[0, 0, :200][gone] == 0) and torch.equal(out[0, 0, :200][~gone], b[0, 0, :200][~gone]) and torch.all(out[0, 0, 200:] == 0)
    assert a.shape == out.shape


def test_strided_queries_heads_in_front_and_strided_weights(tiga):
    c = make([20, 1], [100, 50], 4, 2, 64, BF16, 16, seed=12)
    lse = masses(c, True)
    cache = tiga.PagedCache(c["pages"], c["pages"], c["table"], c["lens"])
    want, _ = tiga.tiga_paged_attention_weights(cache, c["q"], starts([20, 1]), lse, c["scale"])
    wide = torch.zeros((21, 8, 64), dtype=BF16, device="cuda")
    wide[:, 1::2] = c["q"]
    front = c["pages"].transpose(1, 2).contiguous().transpose(1, 2)
    out = torch.zeros((2, 2, 2 * want.shape[2]), device="cuda").transpose(0, 1)[:, :, 4:4 + want.shape[2]]
    tiga.tiga_paged_attention_weights(tiga.PagedCache(front, front, c["table"], c["lens"]), wide[:, 1::2], starts([20, 1]), lse, c["scale"], weights=out)
    assert torch.equal(out, want)


def test_sums_agree_with_the_attention(tiga):
    """Every row's weights sum to one: with the library's own lse the sums over the positions are the rows and heads of a group."""
    c = make([60, 1, 7], [300, 70, 7], 6, 2, 64, F16, 16, seed=13)
    values = torch.zeros_like(c["pages"])
    cache = tiga.PagedCache(c["pages"], values, c["table"], c["lens"])
    _, lse, _ = tiga.tiga_apply_paged_attention(cache, c["q"], starts(c["q_len"]), c["scale"])
    w, _ = tiga.tiga_paged_attention_weights(cache, c["q"], starts(c["q_len"]), lse, c["scale"])
    rows = torch.tensor(c["q_len"], device="cuda", dtype=torch.float64) * 3
    assert torch.allclose(w.double().sum(-1), rows[:, None].expand(3, 2), rtol=2e-5, atol=0)


def test_captured_and_replayed(tiga):
    """Each replay adds a token's weights to what is there."""
    c = make([1, 1], [200, 90], 4, 2, 64, BF16, 16, seed=14)
    lse = masses(c, True)
    cache = tiga.PagedCache(c["pages"], c["pages"], c["table"], c["lens"])
    start = starts([1, 1])
    once, ws = tiga.tiga_paged_attention_weights(cache, c["q"], start, lse, c["scale"])
    total = torch.zeros_like(once)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tiga.tiga_paged_attention_weights(cache, c["q"], start, lse, c["scale"], before=total, weights=total, ws=ws)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.allclose(total, 3 * once, rtol=2.0 ** -22, atol=0)


def test_pages_beyond_32_bits(tiga):
    """Pages whose elements lie behind the 2^31st, brought in boxes and row by row."""
    for page in (16, 7):
        c = make([1, 40], [50, 60], 4, 2, 64, BF16, page, seed=15)
        n = c["pages"].shape[0]
        stride = (1 << 31) // (n - 2) // 8 * 8 + 8
        pool = torch.as_strided(torch.empty((n - 1) * stride + 4096, dtype=BF16, device="cuda"), (n, page, 2, 64), (stride, 128, 64, 1))
        pool.copy_(c["pages"])
        c["pages"] = pool
        check(tiga, c)
        del c, pool
        torch.cuda.empty_cache()
