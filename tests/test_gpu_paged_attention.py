"""GPU parity of attention over paged caches and of the writes into them, against 64 bits (tolerances: attention_reference.py):
single tokens, chunks, pages that end inside of tiles, missing pages, poisoned slots, offsets beyond 32 bits, graphs."""
import pytest

from attention_reference import attend, close, half_step, turn
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


def make(q_len, kv_len, heads, kv_heads, D, dtype, page, seed=0, spare=3, heads_first=False):
    """A cache whose pages lie in any order; every slot that no sequence holds is NaN."""
    B, per = len(q_len), max(1, max(-(-n // page) for n in kv_len)) + 1
    need = sum(-(-n // page) for n in kv_len)
    shape = (need + spare, kv_heads, page, D) if heads_first else (need + spare, page, kv_heads, D)
    view = (lambda t: t.transpose(1, 2)) if heads_first else (lambda t: t)
    kp, vp = (view(torch.full(shape, float("nan"), dtype=dtype, device="cuda")) for _ in range(2))
    order = torch.randperm(need + spare, generator=torch.Generator().manual_seed(seed)).tolist()
    table = torch.full((B, per), -1, dtype=torch.int32)
    keys, values = [], []
    for b, n in enumerate(kv_len):
        k, v = normal((n, kv_heads, D), dtype, 31 * seed + 2 * b + 1), normal((n, kv_heads, D), dtype, 31 * seed + 2 * b + 2)
        keys.append(k)
        values.append(v)
        for i in range(-(-n // page)):
            table[b, i] = order.pop()
            m = min(page, n - i * page)
            kp[int(table[b, i]), :m], vp[int(table[b, i]), :m] = k[i * page:i * page + m], v[i * page:i * page + m]
    return dict(q_len=q_len, kv_len=kv_len, q=normal((sum(q_len), heads, D), dtype, seed + 77), key_pages=kp, value_pages=vp, table=table.cuda(),
                lens=torch.tensor(kv_len, dtype=torch.int32, device="cuda"), keys=keys, values=values, scale=D ** -0.5, page=page)


def reference(c, causal, gone=()):
    parts, q0 = [], 0
    for b, (n, m) in enumerate(zip(c["q_len"], c["kv_len"])):
        at = torch.arange(m, device="cuda")
        seen = (at[None] <= m - n + torch.arange(n, device="cuda")[:, None]) if causal else torch.ones(n, m, dtype=torch.bool, device="cuda")
        for s, page in gone:
            if s == b:
                seen = seen & (at // c["page"] != page)[None]
        parts.append(attend(c["q"][q0:q0 + n], c["keys"][b], c["values"][b], c["scale"], seen))
        q0 += n
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}


def run(tiga, c, causal=True, cache=None):
    guard = Guard(torch)
    cache = cache or tiga.PagedCache(c["key_pages"], c["value_pages"], c["table"], c["lens"])
    out, lse = guard.empty(c["q"].shape, c["q"].dtype), guard.empty(c["q"].shape[:2])
    tiga.tiga_apply_paged_attention(cache, c["q"], starts(c["q_len"]), c["scale"], causal=causal, out=out, lse=lse,
                                    ws=guard.workspace(tiga.tiga_paged_attention_workspace_bytes(cache, c["q"])))
    guard.check()
    return out, lse


def check(tiga, c, causal=True, gone=()):
    out, lse = run(tiga, c, causal)
    want = reference(c, causal, gone)
    close(out, want["out"], want["out_tol"], "out")
    close(lse, want["lse"], want["lse_tol"], "lse")
    again = run(tiga, c, causal)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1]), "reruns must be bit identical"
    return out, lse


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("q_len,kv_len,page", [([1], [1], 16), ([1], [777], 16), ([1, 1, 1], [5, 300, 64], 1), ([1, 1], [129, 0], 8), ([5], [5], 16), ([130], [130], 48),
                                               ([128, 1, 33], [300, 1000, 33], 64), ([0, 7, 0], [10, 200, 0], 32), ([200], [515], 128), ([40, 3], [700, 131], 7), ([9], [300], 1000)])
def test_lengths_and_pages(tiga, q_len, kv_len, page, dtype):
    check(tiga, make(q_len, kv_len, 4, 2, 64, dtype, page, seed=page))


@pytest.mark.parametrize("heads,kv_heads,D,dtype", [(1, 1, 8, F16), (8, 1, 64, BF16), (6, 2, 40, F16), (32, 8, 128, BF16), (5, 5, 96, F16), (40, 5, 72, BF16), (64, 1, 128, F16),
                                                    (144, 1, 64, BF16)])
def test_heads_and_widths(tiga, heads, kv_heads, D, dtype):
    check(tiga, make([1, 17, 2], [90, 150, 260], heads, kv_heads, D, dtype, 16, seed=D))


def test_pages_with_heads_in_front(tiga):
    check(tiga, make([3, 20], [100, 77], 4, 4, 64, BF16, 16, seed=3, heads_first=True))


def test_chunk_reads_the_whole_cache_without_the_triangle(tiga):
    check(tiga, make([70, 1, 5], [200, 30, 5], 4, 2, 64, F16, 16, seed=4), causal=False)


def test_more_new_tokens_than_cache(tiga):
    """Rows in front of position zero read nothing."""
    c = make([12], [5], 2, 2, 64, BF16, 16, seed=5)
    out, lse = check(tiga, c)
    assert torch.all(out[:7] == 0) and torch.all(lse[:7] == -float("inf"))


def test_many_splits_and_batches(tiga):
    check(tiga, make([1], [30011], 8, 2, 128, BF16, 64, seed=6))
    check(tiga, make([1] * 70, [(i * 97) % 900 + 1 for i in range(70)], 8, 2, 64, F16, 16, seed=7))
    check(tiga, make([600, 1, 1, 250], [1500, 2000, 3, 250], 8, 4, 128, F16, 32, seed=8))


def test_long_chunks_whose_tiles_are_counted_by_a_kernel_of_their_own(tiga):
    """More than 64 tiles of 256 packed rows under the triangle: the workspace also holds the counts."""
    check(tiga, make([4200, 90], [4300, 90], 4, 1, 64, BF16, 64, seed=15))
    check(tiga, make([5000], [5000], 4, 1, 32, F16, 16, seed=16))


def test_more_sequences_than_the_blocks_count_themselves(tiga):
    check(tiga, make([1 + i % 3 for i in range(300)], [4 + (i * 37) % 400 for i in range(300)], 4, 2, 64, BF16, 16, seed=17))


def test_on_another_stream(tiga):
    """Rotate, append and attend on a stream that is not the current one; outputs and workspaces are allocated for it."""
    c = make([3, 40], [100, 77], 4, 2, 64, F16, 16, seed=18)
    want = run(tiga, c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    cache = tiga.PagedCache(c["key_pages"], c["value_pages"], c["table"], c["lens"])
    freq, _ = tiga.tiga_rotary_frequencies(64)
    rot = tiga.Rotary(freq.cuda())
    side.wait_stream(torch.cuda.current_stream())
    start = starts(c["q_len"])
    side.wait_stream(torch.cuda.current_stream())
    same = tiga.tiga_apply_rotary(rot, c["q"], torch.zeros(43, dtype=torch.int64, device="cuda"), stream=side)
    out, lse, ws = tiga.tiga_apply_paged_attention(cache, same, start, c["scale"], stream=side)
    side.synchronize()
    assert torch.equal(same, c["q"]) and torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_missing_pages_are_read_as_masked_keys(tiga):
    c = make([1, 30], [200, 150], 4, 2, 64, BF16, 16, seed=9)
    c["table"][0, 3], c["table"][1, 0], c["table"][1, 1] = -1, 2 ** 31 - 1, c["key_pages"].shape[0]
    check(tiga, c, gone=[(0, 3), (1, 0), (1, 1)])
    c["table"].fill_(-7)
    out, lse = run(tiga, c)
    assert torch.all(out == 0) and torch.all(lse == -float("inf"))


def test_lengths_beyond_the_table_are_cut(tiga):
    c = make([1], [100], 2, 2, 64, F16, 16, seed=10)
    want = run(tiga, c, causal=False)
    c["table"] = c["table"][:, :7].contiguous()         # 112 places, the last 12 of them empty
    c["key_pages"].nan_to_num_(nan=0.0)
    c["value_pages"].nan_to_num_(nan=0.0)
    c["lens"].fill_(2 ** 31 - 1)
    got = run(tiga, c, causal=False)
    c["lens"].fill_(112)
    assert torch.equal(got[0], run(tiga, c, causal=False)[0])
    c["lens"].fill_(-3)
    out, lse = run(tiga, c)
    assert torch.all(out == 0) and torch.all(lse == -float("inf")) and not torch.equal(got[1], want[1])


def test_shared_pages(tiga):
    """Two sequences with a common beginning."""
    c = make([1, 1], [64, 64], 4, 2, 64, BF16, 16, seed=11)
    c["table"][1, :4] = c["table"][0, :4]
    c["keys"][1], c["values"][1] = c["keys"][0], c["values"][0]
    check(tiga, c)


def test_offsets_beyond_32_bits(tiga):
    """A cache of more than 2^32 bytes and 2^31 elements per array: the sequence's pages lie at its end."""
    page, hk, D = 64, 8, 128
    n_pages = (1 << 31) // (page * hk * D) + 40
    pages = torch.zeros(n_pages, page, hk, D, dtype=BF16, device="cuda")
    values = torch.zeros_like(pages)
    c = make([1, 5], [300, 200], 8, hk, D, BF16, page, seed=12, spare=0)
    k = c["key_pages"].shape[0]
    pages[-k:], values[-k:] = c["key_pages"], c["value_pages"]
    c["table"] = torch.where(c["table"] >= 0, c["table"] + (n_pages - k), c["table"]).to(torch.int32)
    c["key_pages"], c["value_pages"] = pages, values
    check(tiga, c)


def test_rows_outside_of_the_segments_stay(tiga):
    c = make([1, 5], [30, 20], 2, 2, 64, BF16, 16, seed=13)
    want = run(tiga, c)
    q = torch.cat([c["q"], c["q"]])
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    cache = tiga.PagedCache(c["key_pages"], c["value_pages"], c["table"], c["lens"])
    tiga.tiga_apply_paged_attention(cache, q, starts(c["q_len"]), c["scale"], out=out, lse=lse)
    assert torch.equal(out[:6], want[0]) and torch.equal(lse[:6], want[1]) and torch.all(out[6:] == 7) and torch.all(lse[6:] == 7)


@pytest.mark.parametrize("pairs,turned,D,dtype", [(False, 64, 64, BF16), (True, 32, 80, F16), (False, 36, 72, F16), (True, 6, 8, BF16), (None, 0, 40, F16)])
@pytest.mark.parametrize("q_len,kv_len,page", [([1], [1], 16), ([3, 1, 40], [50, 17, 40], 16), ([9], [5], 4), ([0, 100, 2], [3, 300, 7], 48)])
def test_append(tiga, q_len, kv_len, page, pairs, turned, D, dtype):
    c = make(q_len, kv_len, 2, 2, D, dtype, page, seed=D + page)
    new = normal((sum(q_len), 2, 2, D), dtype, 5)
    key, value = new[:, 0], new[:, 1]
    rot = None
    if turned:
        freq, m = tiga.tiga_rotary_frequencies(turned, scaling=tiga.ROT_BANDS, factor=4.0, length=100.0)
        rot = tiga.Rotary(freq.cuda(), pairs=pairs, magnitude=m)
    kp, vp = c["key_pages"].clone(), c["value_pages"].clone()
    cache = tiga.PagedCache(kp, vp, c["table"], c["lens"])
    tiga.tiga_paged_append(cache, key, value, starts(q_len), rotary=rot)
    wk, wv, q0 = c["key_pages"].double(), c["value_pages"].double(), 0
    tol = torch.zeros_like(wk)
    for b, (n, m_) in enumerate(zip(q_len, kv_len)):
        for t in range(n):
            pos = m_ - n + t
            if pos < 0:
                continue
            p, s = int(c["table"][b, pos // page]), pos % page
            row = key[q0 + t:q0 + t + 1]
            if rot:
                y, size = turn(row, torch.tensor([pos], device="cuda"), freq, m, pairs)
                tol[p, s] = (half_step(dtype) + 2.0 ** -21) * size[0] + 2.0 ** -25
                tol[p, s, :, turned:] = 0
            else:
                y = row.double()
            wk[p, s], wv[p, s] = y[0], value[q0 + t].double()
        q0 += n
    assert torch.equal(torch.isnan(kp), torch.isnan(wk)) and torch.equal(vp.double().nan_to_num(nan=99.0), wv.nan_to_num(nan=99.0))
    close(kp.nan_to_num(nan=0.0), wk.nan_to_num(nan=0.0), tol, "key pages")


def test_append_without_a_page_writes_nowhere(tiga):
    c = make([4, 4], [20, 20], 2, 2, 64, F16, 16, seed=14)
    c["table"][0, 1], c["table"][1, 1] = -1, 2 ** 31 - 1
    kp, vp = c["key_pages"].clone(), c["value_pages"].clone()
    cache = tiga.PagedCache(kp, vp, c["table"], c["lens"])
    new = normal((8, 2, 64), F16, 3)
    tiga.tiga_paged_append(cache, new, new, starts([4, 4]))
    c["lens"].fill_(1000)                   # positions behind the table
    tiga.tiga_paged_append(cache, new, new, starts([4, 4]))
    for a, b in ((kp, c["key_pages"]), (vp, c["value_pages"])):
        assert torch.equal(a.nan_to_num(nan=99.0), b.nan_to_num(nan=99.0))


def test_serving_run_matches_the_dense_relation(tiga):
    """Rotate, append and attend: a prompt in chunks, then token by token, captured in one graph, against one dense reference."""
    heads, hk, D, page, n = 8, 2, 64, 16, 75
    freq, m = tiga.tiga_rotary_frequencies(D)
    rot = tiga.Rotary(freq.cuda(), magnitude=m)
    x = normal((n, heads + 2 * hk, D), BF16, 41)
    q, k, v = x[:, :heads], x[:, heads:heads + hk], x[:, heads + hk:]
    pos = torch.arange(n, device="cuda")
    rq, rk = tiga.tiga_apply_rotary(rot, q, pos), tiga.tiga_apply_rotary(rot, k, pos)
    seen = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
    want = attend(rq, rk, v, D ** -0.5, seen)
    pages = torch.full((8, page, hk, D), float("nan"), dtype=BF16, device="cuda")
    lens = torch.zeros(1, dtype=torch.int32, device="cuda")
    table = torch.tensor([[5, 0, 3, 7, 1]], dtype=torch.int32, device="cuda")
    cache = tiga.PagedCache(pages, pages.clone(), table, lens)
    got, done = [], 0
    for size in (50, 13):
        rows = slice(done, done + size)
        lens.fill_(done + size)
        tiga.tiga_paged_append(cache, k[rows], v[rows], starts([size]), rotary=rot)
        got.append(tiga.tiga_apply_paged_attention(cache, rq[rows], starts([size]), D ** -0.5)[0])
        done += size
    # single tokens: one graph, replayed with the next token in its buffers
    bq, bk, bv, bp, one = torch.empty_like(q[:1]), torch.empty_like(k[:1]), torch.empty_like(v[:1]), torch.zeros(1, dtype=torch.int32, device="cuda"), starts([1])
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        lens.add_(1)
        turned = tiga.tiga_apply_rotary(rot, bq, bp)
        tiga.tiga_paged_append(cache, bk, bv, one, rotary=rot)
        out, _, ws = tiga.tiga_apply_paged_attention(cache, turned, one, D ** -0.5)
    for t in range(done, n):
        bq.copy_(q[t:t + 1])
        bk.copy_(k[t:t + 1])
        bv.copy_(v[t:t + 1])
        bp.fill_(t)
        graph.replay()
        got.append(out.clone())
    close(torch.cat(got), want["out"], want["out_tol"], "out")
