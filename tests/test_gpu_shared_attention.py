"""GPU parity of attention over paged caches that share prefixes, against 64 bits (tolerances: attention_reference.py; the states of a row
are joined in fp32, as partial states are)."""
import pytest

from attention_reference import attend, close
from parity import Guard

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def tiga():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_24802_b200 import api
    return api


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def starts(lengths):
    s = [0]
    for n in lengths:
        s.append(s[-1] + n)
    return ints(s)


def normal(shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def make(groups, heads, kv_heads, D, dtype, page, seed=0):
    """groups: (shared positions, [(new tokens, positions behind the shared ones), ...]).  The whole pages of the shared positions are the
    same for a group's sequences; slots that no sequence holds are NaN."""
    tables, keys, values, q_len, kv_len, group_start, shared = [], [], [], [], [], [0], []
    blocks = []                     # pages in the order of their numbers, before they are shuffled
    for i, (common, members) in enumerate(groups):
        k0, v0 = normal((common, kv_heads, D), dtype, 1000 * seed + 2 * i), normal((common, kv_heads, D), dtype, 1000 * seed + 2 * i + 1)
        whole, ids = common // page, []
        for b in range(whole):
            ids.append(len(blocks))
            blocks.append((k0[b * page:(b + 1) * page], v0[b * page:(b + 1) * page]))
        for n, m in members:
            at = 7919 * seed + len(keys) + 31
            k, v = torch.cat([k0, normal((m, kv_heads, D), dtype, 2 * at)]), torch.cat([v0, normal((m, kv_heads, D), dtype, 2 * at + 1)])
            mine = list(ids)
            for b in range(whole, -(-(common + m) // page)):
                mine.append(len(blocks))
                blocks.append((k[b * page:(b + 1) * page], v[b * page:(b + 1) * page]))
            tables.append(mine)
            keys.append(k)
            values.append(v)
            q_len.append(n)
            kv_len.append(common + m)
        group_start.append(len(keys))
        shared.append(whole * page)
    order = torch.randperm(len(blocks) + 2, generator=torch.Generator().manual_seed(seed)).tolist()
    kp, vp = (torch.full((len(blocks) + 2, page, kv_heads, D), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
    for i, (k, v) in enumerate(blocks):
        kp[order[i], :len(k)], vp[order[i], :len(v)] = k, v
    table = torch.full((len(keys), max(1, max(len(t) for t in tables)) + 1), -1, dtype=torch.int32)
    for i, t in enumerate(tables):
        table[i, :len(t)] = torch.tensor([order[b] for b in t], dtype=torch.int32)
    return dict(q_len=q_len, kv_len=kv_len, keys=keys, values=values, key_pages=kp, value_pages=vp, table=table.cuda(), lens=ints(kv_len),
                group_start=ints(group_start), shared=ints(shared), q=normal((sum(q_len), heads, D), dtype, seed + 77), scale=D ** -0.5)


def reference(c, causal):
    parts, q0 = [], 0
    for n, k, v in zip(c["q_len"], c["keys"], c["values"]):
        m = len(k)
        at = torch.arange(m, device="cuda")
        seen = (at[None] <= m - n + torch.arange(n, device="cuda")[:, None]) if causal else torch.ones(n, m, dtype=torch.bool, device="cuda")
        parts.append(attend(c["q"][q0:q0 + n], k, v, c["scale"], seen))
        q0 += n
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}


def run(tiga, c, causal=True, untouched=False):
    guard = Guard(torch)
    cache = tiga.PagedCache(c["key_pages"], c["value_pages"], c["table"], c["lens"])
    prefixes = tiga.SharedPrefixes(c["group_start"], c["shared"])
    out, lse = guard.empty(c["q"].shape, c["q"].dtype), guard.empty(c["q"].shape[:2])
    tiga.tiga_apply_shared_attention(cache, prefixes, c["q"], starts(c["q_len"]), c["scale"], causal=causal, out=out, lse=lse,
                                     ws=guard.workspace(tiga.tiga_shared_attention_workspace_bytes(cache, prefixes, c["q"])))
    guard.check(allow_untouched=[out, lse] if untouched else ())
    return out, lse


def check(tiga, c, causal=True):
    out, lse = run(tiga, c, causal)
    want = reference(c, causal)
    close(out, want["out"], want["out_tol"], "out")
    close(lse, want["lse"], want["lse_tol"], "lse")
    again = run(tiga, c, causal)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1]), "reruns must be bit identical"
    return out, lse


GROUPS = [
    [(320, [(1, 77), (1, 5), (1, 200), (1, 1)])],
    [(1024, [(1, 1 + 13 * i) for i in range(40)])],
    [(512, [(1, 1)])],                                                   # one sequence shares with nobody
    [(0, [(1, 10), (1, 20)])],                                            # nothing is shared
    [(640, [(3, 70), (1, 9), (5, 5), (2, 300), (1, 40), (4, 11)]), (256, [(1, 3), (1, 4), (1, 5), (1, 6)]), (1000, [(7, 80), (9, 90), (1, 1)])],
    [(777, [(1, 30), (0, 12), (2, 2), (1, 100), (1, 3)])],                # shared positions end inside of a page, a sequence without new tokens
    [(384, [(60, 60), (40, 200), (33, 33), (1, 7)])],                     # chunks that fill their tiles alone
    [(2000, [(20, 25), (15, 15), (31, 100), (8, 9), (40, 41), (1, 1), (2, 5)])],
]


@pytest.mark.parametrize("dtype,page", [(F16, 16), (BF16, 64)])
@pytest.mark.parametrize("groups", GROUPS)
def test_groups(tiga, groups, dtype, page):
    check(tiga, make(groups, 8, 2, 64, dtype, page, seed=len(groups)))


@pytest.mark.parametrize("page", [1, 7, 8, 24, 48, 100, 128])
def test_pages(tiga, page):
    """Shared positions that end inside of a group of 32, pages that hold no group of 8."""
    check(tiga, make([(700, [(1, 50), (2, 7), (1, 200), (1, 1), (3, 90)]), (300, [(1, 1), (1, 2), (1, 3), (1, 40)])], 4, 1, 64, BF16, page, seed=page))


@pytest.mark.parametrize("heads,kv_heads,D,dtype", [(1, 1, 8, F16), (8, 1, 64, BF16), (6, 2, 40, F16), (32, 8, 128, BF16), (5, 5, 96, F16), (40, 5, 72, BF16), (64, 1, 128, F16),
                                                    (144, 1, 64, BF16)])
def test_heads_and_widths(tiga, heads, kv_heads, D, dtype):
    check(tiga, make([(512, [(1, 30), (2, 60), (1, 5), (1, 9), (1, 150)])], heads, kv_heads, D, dtype, 16, seed=D))


def test_without_the_triangle(tiga):
    check(tiga, make([(512, [(3, 30), (2, 60), (1, 5), (1, 9)])], 4, 2, 64, F16, 16, seed=4), causal=False)


def test_long_prefixes_and_many_sequences(tiga):
    check(tiga, make([(20000, [(1, 100 + i) for i in range(20)])], 8, 2, 128, BF16, 64, seed=5))
    check(tiga, make([(300 + 16 * (i % 5), [(1 + (i + k) % 2, 2 + (i * 7 + k * 13) % 90) for k in range(1 + i % 6)]) for i in range(100)], 4, 2, 64, F16, 16, seed=6))


def test_what_is_called_shared_is_cut_to_what_all_rows_read(tiga):
    """Three new tokens each, and a prefix said to reach to their ends: the first of them reads less."""
    c = make([(640, [(3, 3), (3, 3), (3, 3), (3, 3), (3, 3)])], 4, 2, 64, BF16, 16, seed=7)
    want = check(tiga, c)
    c["table"][1:, 40] = c["table"][0, 40]          # (the tail's page differs; only whole pages may be called shared)
    c["keys"] = [torch.cat([k[:640], c["keys"][0][640:]]) for k in c["keys"]]
    c["values"] = [torch.cat([v[:640], c["values"][0][640:]]) for v in c["values"]]
    for said in (640, 641, 643, 656, 1 << 30):
        c["shared"] = ints([said])
        check(tiga, c)
    assert want is not None


def test_sequences_outside_of_every_group(tiga):
    c = make([(0, [(1, 300), (2, 40)]), (512, [(1, 30), (2, 60), (1, 5), (1, 9)]), (0, [(1, 77), (3, 3)])], 4, 2, 64, F16, 16, seed=8)
    c["group_start"], c["shared"] = ints([2, 6]), ints([512])
    check(tiga, c)
    c["group_start"], c["shared"] = ints([0]), ints([])
    check(tiga, c)


def test_groups_that_do_not_ascend_lead_nowhere(tiga):
    """Bounds that overlap or run backwards: nothing is written outside of the arrays (the guard bands), and sequences that a group does not
    hold keep their results."""
    c = make([(512, [(1, 30), (2, 60), (1, 5), (1, 9)]), (512, [(1, 10), (1, 20), (1, 30), (1, 40)])], 4, 2, 64, F16, 16, seed=9)
    for bounds in ([0, 9, 2, 8], [8, 4, 0, 0], [-5, 100, -7, 3], [0, 8, 8, 8]):
        c["group_start"], c["shared"] = ints(bounds), ints([512, 512, 512])
        run(tiga, c, untouched=True)


def test_new_tokens_that_do_not_ascend_lead_nowhere(tiga):
    c = make([(512, [(1, 30), (2, 60), (1, 5), (1, 9)])], 4, 2, 64, F16, 16, seed=10)
    guard = Guard(torch)
    cache, prefixes = tiga.PagedCache(c["key_pages"], c["value_pages"], c["table"], c["lens"]), tiga.SharedPrefixes(c["group_start"], c["shared"])
    for bounds in ([0, 3, 1, 5, 2], [5, 4, 3, 2, 1], [-9, 2, 900, 3, 4]):
        out = guard.empty(c["q"].shape, F16)
        tiga.tiga_apply_shared_attention(cache, prefixes, c["q"], ints(bounds), c["scale"], out=out, want_lse=False,
                                         ws=guard.workspace(tiga.tiga_shared_attention_workspace_bytes(cache, prefixes, c["q"])))
        guard.check(allow_untouched=[out])


def test_missing_pages(tiga):
    """A missing page among the shared ones is missing for the group; one behind them for its sequence."""
    c = make([(512, [(1, 30), (2, 60), (1, 5), (1, 9)])], 4, 2, 64, BF16, 16, seed=11)
    c["table"][:, 3], c["table"][1, 33] = -1, 1 << 20
    out, lse = run(tiga, c)
    cache = tiga.PagedCache(c["key_pages"], c["value_pages"], c["table"], c["lens"])
    want, want_lse, _ = tiga.tiga_apply_paged_attention(cache, c["q"], starts(c["q_len"]), c["scale"])
    # both are within 2 u + u^2 of sum |p v| (attention_reference.py); values here are below 6
    assert float((out.double() - want.double()).abs().max()) <= 2 * 2.1 * 2.0 ** -8 * 6 and torch.allclose(lse, want_lse, rtol=0, atol=2e-5)


def test_captured_and_replayed_with_other_lengths(tiga):
    c = make([(512, [(1, 30), (1, 60), (1, 5), (1, 9)])], 4, 2, 64, BF16, 16, seed=12)
    cache, prefixes = tiga.PagedCache(c["key_pages"], c["value_pages"], c["table"], c["lens"]), tiga.SharedPrefixes(c["group_start"], c["shared"])
    start = starts(c["q_len"])
    out, lse, ws = tiga.tiga_apply_shared_attention(cache, prefixes, c["q"], start, c["scale"])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tiga.tiga_apply_shared_attention(cache, prefixes, c["q"], start, c["scale"], out=out, lse=lse, ws=ws)
    for shared, lens in ((512, [520, 570, 512, 513]), (256, [542, 300, 517, 257]), (0, [1, 2, 3, 4])):
        c["lens"].copy_(ints(lens))
        c["shared"].copy_(ints([shared]))
        graph.replay()
        torch.cuda.synchronize()
        want = reference(dict(c, keys=[k[:n] for k, n in zip(c["keys"], lens)], values=[v[:n] for v, n in zip(c["values"], lens)]), True)
        close(out, want["out"], want["out_tol"], "out")
        close(lse, want["lse"], want["lse_tol"], "lse")


def test_on_another_stream_with_strided_queries(tiga):
    c = make([(512, [(1, 30), (2, 60), (1, 5), (1, 9)])], 4, 2, 64, F16, 16, seed=13)
    want = run(tiga, c)
    wide = torch.zeros((5, 8, 64), dtype=F16, device="cuda")
    wide[:, 1::2] = c["q"]
    cache, prefixes = tiga.PagedCache(c["key_pages"], c["value_pages"], c["table"], c["lens"]), tiga.SharedPrefixes(c["group_start"], c["shared"])
    side = torch.cuda.Stream()
    start = starts(c["q_len"])
    side.wait_stream(torch.cuda.current_stream())
    out, lse, _ = tiga.tiga_apply_shared_attention(cache, prefixes, wide[:, 1::2], start, c["scale"], stream=side)
    side.synchronize()
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_more_groups_and_sequences_than_the_plan_holds(tiga):
    """Over a thousand groups of two, and a thousand sequences in one group."""
    check(tiga, make([(128 + 16 * (i % 3), [(1, 1 + i % 5), (1, 2)]) for i in range(1100)], 8, 1, 32, F16, 16, seed=14))
    check(tiga, make([(256, [(1, 1 + i % 7) for i in range(1100)])], 4, 2, 32, BF16, 16, seed=15))


def test_lengths_beyond_the_table(tiga):
    """Rows count their positions from the sequence's length, of which the table holds less."""
    c = make([(512, [(1, 30), (2, 60), (1, 5), (1, 9)])], 4, 2, 64, F16, 16, seed=16)
    c["table"] = c["table"][:, :33].contiguous()
    c["lens"] = ints([600, 529, 700, 10 ** 9])
    for name in ("key_pages", "value_pages"):           # (slots behind the sequences' tokens are NaN, and now some are read)
        c[name] = torch.nan_to_num(c[name], nan=0.5)
    out, lse = run(tiga, c)
    cache = tiga.PagedCache(c["key_pages"], c["value_pages"], c["table"], c["lens"])
    want, want_lse, _ = tiga.tiga_apply_paged_attention(cache, c["q"], starts(c["q_len"]), c["scale"])
    # both are within 2 u + u^2 of sum |p v| (attention_reference.py); values here are below 6
    assert float((out.double() - want.double()).abs().max()) <= 2 * 2.1 * 2.0 ** -11 * 6 and torch.allclose(lse, want_lse, rtol=0, atol=2e-5)


def test_pages_beyond_32_bits(tiga):
    c = make([(128, [(1, 30), (2, 17), (1, 5), (1, 9)])], 8, 2, 64, BF16, 16, seed=17)
    n = c["key_pages"].shape[0]
    stride = (1 << 31) // (n - 2) // 8 * 8 + 8
    for name in ("key_pages", "value_pages"):
        pool = torch.as_strided(torch.empty((n - 1) * stride + 4096, dtype=BF16, device="cuda"), (n, 16, 2, 64), (stride, 128, 64, 1))
        pool.copy_(c[name])
        c[name] = pool
    check(tiga, c)
