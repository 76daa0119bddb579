"""GPU parity of the online-softmax reducer over block-diagonal dense relations, forward and backward, against 64 bits: tolerances
are derived in attention_reference.py.  Lengths of zero and one, lengths around the tiles of 64 and 128, empty rows, masks,
strides, poisoned keys, graphs, streams."""
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


def starts(lengths, first=0):
    s = [first]
    for n in lengths:
        s.append(s[-1] + n)
    return torch.tensor(s, dtype=torch.int32, device="cuda")


def normal(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def case(q_len, kv_len, heads, kv_heads, D, dtype, mask=None, seed=0, packed=False, scale=None, spread=1.0):
    nq, nk = sum(q_len), sum(kv_len)
    c = dict(q_len=q_len, kv_len=kv_len, scale=D ** -0.5 if scale is None else scale, dtype=dtype,
             q=normal((nq, heads, D), dtype, 7 * seed + 1, spread), go=normal((nq, heads, D), dtype, 7 * seed + 2, 0.1))
    if packed:      # keys and values from one projection, heads in front of the pair: strided rows and heads
        kv = normal((nk, kv_heads, 2, D), dtype, 7 * seed + 3, spread)
        c["k"], c["v"] = kv[:, :, 0], kv[:, :, 1]
    else:
        c["k"], c["v"] = normal((nk, kv_heads, D), dtype, 7 * seed + 3, spread), normal((nk, kv_heads, D), dtype, 7 * seed + 4)
    c["mask"] = None
    if mask is not None:
        c["mask"] = torch.rand(nk, generator=torch.Generator(device="cuda").manual_seed(seed + 5), device="cuda") < mask
    return c


def reference(c, backward=True):
    parts, q0, k0 = [], 0, 0
    for n, m in zip(c["q_len"], c["kv_len"]):
        keep = torch.ones(m, dtype=torch.bool, device="cuda") if c["mask"] is None else c["mask"][k0:k0 + m].bool()
        parts.append(attend(c["q"][q0:q0 + n], c["k"][k0:k0 + m], c["v"][k0:k0 + m], c["scale"], keep[None].expand(n, m),
                            c["go"][q0:q0 + n] if backward else None))
        q0, k0 = q0 + n, k0 + m
    return {name: torch.cat([p[name] for p in parts]) for name in parts[0]}


def run(tiga, c, backward=True, guard=None):
    guard = guard or Guard(torch)
    g = tiga.DenseRelation(starts(c["q_len"]), starts(c["kv_len"]), c["mask"])
    q, k, v = c["q"], c["k"], c["v"]
    r = {"out": guard.empty(q.shape, q.dtype), "lse": guard.empty(q.shape[:2])}
    tiga.tiga_apply_dense_attention(g, q, k, v, c["scale"], out=r["out"], lse=r["lse"],
                                    ws=guard.workspace(tiga.tiga_dense_attention_workspace_bytes(g, q, k, v)))
    if backward:
        for name, like in (("grad_q", q), ("grad_key", k), ("grad_value", k)):
            r[name] = guard.empty(like.shape, like.dtype)
        tiga.tiga_apply_dense_attention_backward(g, q, k, v, r["out"], r["lse"], c["go"], c["scale"], grad_q=r["grad_q"], grad_key=r["grad_key"],
                                                 grad_value=r["grad_value"],
                                                 ws=guard.workspace(tiga.tiga_dense_attention_workspace_bytes(g, q, k, v, True)))
    guard.check()
    return r


def check(tiga, c, backward=True):
    want = reference(c, backward)
    got = run(tiga, c, backward)
    for name in got:
        close(got[name], want[name], want[name + "_tol"], name)
    again = run(tiga, c, backward)
    for name in got:
        assert torch.equal(got[name], again[name]), f"{name}: reruns must be bit identical"
    return got


LENGTHS = [([65], [65]), ([1], [1]), ([1], [300]), ([300], [1]), ([0, 5, 0, 130], [7, 0, 3, 129]), ([128], [128]), ([257, 3], [255, 513]),
           ([64, 64, 64], [0, 0, 64]), ([31, 1, 2, 90, 17], [63, 64, 65, 127, 1])]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("q_len,kv_len", LENGTHS)
def test_lengths(tiga, q_len, kv_len, dtype):
    check(tiga, case(q_len, kv_len, 2, 2, 64, dtype, seed=len(q_len)))


@pytest.mark.parametrize("heads,kv_heads,D,dtype", [(1, 1, 8, F16), (4, 2, 16, BF16), (6, 2, 32, F16), (5, 1, 40, BF16), (3, 3, 72, F16), (8, 2, 80, BF16),
                                                    (4, 1, 96, F16), (12, 4, 128, BF16), (8, 1, 128, F16), (40, 8, 64, BF16)])
def test_heads_and_widths(tiga, heads, kv_heads, D, dtype):
    check(tiga, case([70, 9, 33], [50, 131, 200], heads, kv_heads, D, dtype, seed=D, packed=True))


@pytest.mark.parametrize("dtype,D,keep", [(F16, 64, 0.5), (BF16, 128, 0.02), (BF16, 64, 0.0)])
def test_masks(tiga, dtype, D, keep):
    c = case([40, 130, 7], [300, 1, 140], 4, 2, D, dtype, mask=keep, seed=11)
    if keep:
        c["mask"][300] = False              # the second segment's rows read nothing
    got = check(tiga, c)
    assert torch.all(got["out"][40:170] == 0) and torch.all(got["lse"][40:170] == float("-inf"))
    off = ~c["mask"]
    assert torch.all(got["grad_key"][off] == 0) and torch.all(got["grad_value"][off] == 0) and torch.all(got["grad_q"][40:170] == 0)


@pytest.mark.parametrize("poison", [float("nan"), float("inf"), -float("inf"), "lowest"])
def test_masked_keys_have_no_influence(tiga, poison):
    c = case([40, 70], [200, 90], 2, 1, 64, BF16, mask=0.6, seed=12)
    clean = run(tiga, c)
    fill = torch.finfo(BF16).min if poison == "lowest" else poison
    for name in ("k", "v"):
        c[name] = c[name].clone()
        c[name][~c["mask"]] = fill
    got = run(tiga, c)
    for name in got:
        assert torch.equal(got[name], clean[name]), name


def test_many_rows_and_keys(tiga):
    """More tiles than the device has SMs, long sums, work that is split over the keys and over the rows."""
    check(tiga, case([1000, 333], [700, 1999], 8, 2, 128, BF16, seed=13))
    check(tiga, case([3], [20000], 2, 2, 64, F16, seed=14))
    check(tiga, case([5000], [5], 4, 4, 64, BF16, seed=15))


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_large_and_growing_scores(tiga, dtype):
    """Scores of a few hundred, rising along the keys, so that the running maximum moves in every tile."""
    c = case([130], [700], 2, 2, 64, dtype, seed=16, spread=4.0)
    c["k"] = (c["k"].float() * torch.linspace(0.1, 1.5, 700, device="cuda")[:, None, None]).to(dtype)
    check(tiga, c)
    c = case([40], [300], 2, 2, 64, dtype, seed=17, scale=0.0)
    check(tiga, c)
    c = case([40], [300], 2, 2, 64, dtype, seed=18, scale=-0.3)
    check(tiga, c)


def test_small_weights_and_gradients_keep_their_digits_in_f16(tiga):
    c = case([60], [9000], 1, 1, 64, F16, seed=19, spread=0.2)
    c["go"] = (c["go"].float() * 2.0 ** -9).to(F16)
    check(tiga, c)


def test_single_key_has_weight_one(tiga):
    c = case([50], [1], 2, 2, 64, BF16, seed=20)
    got = run(tiga, c)
    assert torch.equal(got["out"], c["v"].expand(50, 2, 64))
    # dP and delta are the same sum in two orders, each off by at most (D + 8) 2^-23 of sum |go v|; p is off by a few 2^-23 of nothing
    q, k, v, go = (c[n].double() for n in ("q", "k", "v", "go"))
    ds = c["scale"] * 2 * 72 * 2.0 ** -23 * (go * v).abs().sum(-1, keepdim=True)
    assert torch.all(got["grad_q"].abs() <= 1.01 * ds * k.abs()) and torch.all(got["grad_key"].abs() <= 1.01 * (ds * q.abs()).sum(0, keepdim=True))


def test_scores_of_a_single_key_have_no_gradient(tiga):
    """One key, or one that the mask leaves: exact zeros, in whole tiles and in tiles that several blocks share."""
    for q_len, kv_len, left in (([50], [1], None), ([20000, 7], [1, 1], None), ([300, 40], [9, 30], (4, 20))):
        c = case(q_len, kv_len, 4, 2, 64, BF16, seed=35)
        if left:
            c["mask"] = torch.zeros(sum(kv_len), dtype=torch.bool, device="cuda")
            c["mask"][left[0]] = c["mask"][kv_len[0] + left[1]] = True
        got = check(tiga, c)
        assert torch.all(got["grad_q"] == 0) and torch.all(got["grad_key"] == 0) and torch.any(got["grad_value"] != 0)


@pytest.mark.parametrize("dtype,D", [(F16, 64), (BF16, 128), (BF16, 40)])
@pytest.mark.parametrize("n", [2, 3, 7, 16, 17])
def test_few_keys(tiga, n, dtype, D):
    """delta is summed over the keys themselves: dS is rounded once and the result once, as over many keys (2 u + u^2, no share of out's
    rounding; seventeen keys and more have that share)."""
    c = case([70, 3, 200], [n, 1, n], 4, 2, D, dtype, seed=36 + n)
    want, got = reference(c), run(tiga, c)
    for name in got:
        close(got[name], want[name], want[name + "_tol"] * (0.7 if name in ("grad_q", "grad_key") and n <= 16 else 1.0) + torch.finfo(dtype).smallest_normal, name)


def test_rows_outside_of_the_segments_stay(tiga):
    c = case([10, 20], [30, 40], 2, 2, 64, BF16, seed=21)
    want = run(tiga, c)
    wide = {n: torch.cat([torch.zeros(3, *c[n].shape[1:], dtype=BF16, device="cuda"), c[n], torch.zeros(5, *c[n].shape[1:], dtype=BF16, device="cuda")]) for n in ("q", "k", "v", "go")}
    g = tiga.DenseRelation(starts([10, 20], 3), starts([30, 40], 3))
    out, lse = torch.full_like(wide["q"], 7.0), torch.full(wide["q"].shape[:2], 7.0, device="cuda")
    tiga.tiga_apply_dense_attention(g, wide["q"], wide["k"], wide["v"], c["scale"], out=out, lse=lse)
    grads = [torch.full_like(wide[n], 7.0) for n in ("q", "k", "k")]
    tiga.tiga_apply_dense_attention_backward(g, wide["q"], wide["k"], wide["v"], out, lse, wide["go"], c["scale"], *grads)
    for t, name in zip([out, lse] + grads, ("out", "lse", "grad_q", "grad_key", "grad_value")):
        n = want[name].shape[0]
        assert torch.all(t[:3] == 7) and torch.all(t[3 + n:] == 7), name
        assert torch.equal(t[3:3 + n], want[name]), name


def test_bounds_beyond_the_arrays_are_clamped(tiga):
    """Descending, negative and far bounds lead nowhere outside of the arrays; what is written there lies inside (guard bands)."""
    c = case([50], [60], 2, 2, 64, F16, seed=22)
    guard = Guard(torch)
    out, lse = guard.empty(c["q"].shape, F16), guard.empty(c["q"].shape[:2])
    g = tiga.DenseRelation(torch.tensor([-5, 20, 10, 2 ** 31 - 1], dtype=torch.int32, device="cuda"),
                           torch.tensor([2 ** 31 - 1, -2 ** 31, 30, 100], dtype=torch.int32, device="cuda"))
    tiga.tiga_apply_dense_attention(g, c["q"], c["k"], c["v"], c["scale"], out=out, lse=lse,
                                    ws=guard.workspace(tiga.tiga_dense_attention_workspace_bytes(g, c["q"], c["k"], c["v"])))
    tiga.tiga_apply_dense_attention_backward(g, c["q"], c["k"], c["v"], torch.zeros_like(c["q"]), torch.zeros(c["q"].shape[:2], device="cuda"), c["go"], c["scale"],
                                             grad_q=guard.empty(c["q"].shape, F16), grad_key=guard.empty(c["k"].shape, F16), grad_value=guard.empty(c["k"].shape, F16),
                                             ws=guard.workspace(tiga.tiga_dense_attention_workspace_bytes(g, c["q"], c["k"], c["v"], True)))
    guard.check(allow_untouched=[v for _, _, v, kind in guard.items if kind == "out"])


def test_shared_storage_and_odd_strides(tiga):
    """Broadcast keys (row or head stride 0), rows further apart than their heads."""
    c = case([20], [40], 4, 2, 64, BF16, seed=23)
    c["k"] = normal((40, 1, 64), BF16, 3).expand(40, 2, 64)
    c["v"] = normal((1, 2, 64), BF16, 4).expand(40, 2, 64)
    c["q"] = normal((20, 3, 4, 72), BF16, 5)[:, 1, :, :64]
    c["go"] = normal((20, 4, 64), BF16, 6, 0.1).transpose(0, 1).contiguous().transpose(0, 1)
    check(tiga, c)


def test_gradients_against_differences(tiga):
    """The formula itself: differences of sum(out * go) in 64 bits along random directions."""
    c = case([9], [13], 2, 1, 16, F16, seed=24)
    got = run(tiga, c)
    f = lambda q, k, v: (attend(q, k, v, c["scale"], torch.ones(9, 13, dtype=torch.bool, device="cuda"))["out"] * c["go"].double()).sum()  # noqa: E731
    x = {"grad_q": c["q"].double(), "grad_key": c["k"].double(), "grad_value": c["v"].double()}
    want = reference(c)
    for name in x:
        d = normal(x[name].shape, torch.float64, 99)
        at = lambda e: f(*(x[n] + (e * d if n == name else 0) for n in x))  # noqa: E731
        slope = (at(1e-4) - at(-1e-4)) / 2e-4
        assert abs(float((got[name].double() * d).sum() - slope)) <= float((want[name + "_tol"] * d.abs()).sum()) + 1e-6 * float(abs(slope) + 1)


def test_only_the_wanted_gradients(tiga):
    c = case([70], [90], 4, 2, 64, BF16, seed=25)
    want = run(tiga, c)
    g = tiga.DenseRelation(starts([70]), starts([90]))
    args = (g, c["q"], c["k"], c["v"], want["out"], want["lse"], c["go"], c["scale"])
    gq, gk, gv, _ = tiga.tiga_apply_dense_attention_backward(*args, want_kv=False)
    assert gk is None and gv is None and torch.equal(gq, want["grad_q"])
    gq, gk, gv, _ = tiga.tiga_apply_dense_attention_backward(*args, want_q=False)
    assert gq is None and torch.equal(gk, want["grad_key"]) and torch.equal(gv, want["grad_value"])
    gv = torch.empty_like(c["v"])
    tiga.tiga_apply_dense_attention_backward(*args, want_q=False, want_kv=False, grad_value=gv)
    assert torch.equal(gv, want["grad_value"])


def test_nothing_on_one_side(tiga):
    """No rows at all, no keys at all, no segments: zeros where something is left to write."""
    c = case([0, 0], [5, 3], 2, 2, 64, F16, seed=32)
    got = run(tiga, c)
    assert torch.all(got["grad_key"] == 0) and torch.all(got["grad_value"] == 0) and got["out"].shape == (0, 2, 64)
    c = case([5], [0], 2, 2, 64, BF16, seed=33)
    got = run(tiga, c)
    assert torch.all(got["out"] == 0) and torch.all(got["lse"] == -float("inf")) and torch.all(got["grad_q"] == 0)
    g = tiga.DenseRelation(starts([]), starts([]))
    out = torch.full_like(c["q"], 7.0)
    tiga.tiga_apply_dense_attention(g, c["q"], c["k"], c["v"], 1.0, out=out)
    assert torch.all(out == 7)


def test_without_lse(tiga):
    c = case([70, 300], [90, 513], 4, 2, 64, BF16, seed=34)
    g = tiga.DenseRelation(starts(c["q_len"]), starts(c["kv_len"]))
    out, lse, _ = tiga.tiga_apply_dense_attention(g, c["q"], c["k"], c["v"], c["scale"], want_lse=False)
    assert lse is None and torch.equal(out, run(tiga, c, backward=False)["out"])


def test_graph_replays_with_other_lengths(tiga):
    """Bounds are read on the device: one captured step serves other lengths and other data."""
    a, b = case([60, 70], [200, 150], 4, 2, 64, BF16, seed=26), case([100, 30], [9, 341], 4, 2, 64, BF16, seed=27)
    qs, ks = starts(a["q_len"]), starts(a["kv_len"])
    x = {n: a[n].clone() for n in ("q", "k", "v", "go")}
    g = tiga.DenseRelation(qs, ks)
    side = torch.cuda.Stream()
    step = lambda: tiga.tiga_apply_dense_attention(g, x["q"], x["k"], x["v"], a["scale"])  # noqa: E731
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out, lse, ws = step()
        gq, gk, gv, ws2 = tiga.tiga_apply_dense_attention_backward(g, x["q"], x["k"], x["v"], out, lse, x["go"], a["scale"])
    for c in (b, a):
        qs.copy_(starts(c["q_len"]))
        ks[: len(c["kv_len"]) + 1].copy_(starts(c["kv_len"]))
        for n in x:
            x[n][: c[n].shape[0]].copy_(c[n])
        graph.replay()
        want = run(tiga, c)
        for t, name in zip((out, lse, gq, gk, gv), ("out", "lse", "grad_q", "grad_key", "grad_value")):
            assert torch.equal(t[: want[name].shape[0]], want[name]), name


def test_two_streams_at_once(tiga):
    cs = [case([300], [400], 4, 4, 64, BF16, seed=28 + i) for i in range(2)]
    want = [run(tiga, c) for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    got = []
    for _ in range(3):
        for c, s in zip(cs, streams):
            g = tiga.DenseRelation(starts(c["q_len"]), starts(c["kv_len"]))
            s.wait_stream(torch.cuda.current_stream())
            got.append((g, tiga.tiga_apply_dense_attention(g, c["q"], c["k"], c["v"], c["scale"], stream=s)))
    torch.cuda.synchronize()
    for i, (_, (out, lse, _)) in enumerate(got):
        assert torch.equal(out, want[i % 2]["out"]) and torch.equal(lse, want[i % 2]["lse"])


def test_many_segments(tiga):
    """Thousands of segments of a few rows, some empty."""
    n = 3000
    q_len = [(i * 7) % 4 for i in range(n)]
    kv_len = [(i * 5) % 11 for i in range(n)]
    c = case(q_len, kv_len, 2, 1, 32, BF16, seed=31)
    got = run(tiga, c)
    q0 = k0 = 0
    qs, ks = [0], [0]
    for a, b in zip(q_len, kv_len):
        qs.append(qs[-1] + a)
        ks.append(ks[-1] + b)
    for s in list(range(0, 40)) + list(range(n - 40, n)):
        q0, q1, k0, k1 = qs[s], qs[s + 1], ks[s], ks[s + 1]
        want = attend(c["q"][q0:q1], c["k"][k0:k1], c["v"][k0:k1], c["scale"], torch.ones(q1 - q0, k1 - k0, dtype=torch.bool, device="cuda"), c["go"][q0:q1])
        for name, (a, b) in (("out", (q0, q1)), ("lse", (q0, q1)), ("grad_q", (q0, q1)), ("grad_key", (k0, k1)), ("grad_value", (k0, k1))):
            close(got[name][a:b], want[name], want[name + "_tol"], f"{name} of segment {s}")
