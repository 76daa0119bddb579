"""GPU parity of the online-softmax reducer over triangular relations (causal attention of packed sequences), forward and backward,
against 64 bits: tolerances are derived in attention_reference.py."""
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
    c = dict(q_len=q_len, kv_len=kv_len, scale=D ** -0.5 if scale is None else scale, mask=None,
             q=normal((nq, heads, D), dtype, 7 * seed + 1, spread), go=normal((nq, heads, D), dtype, 7 * seed + 2, 0.1))
    if packed:
        kv = normal((nk, kv_heads, 2, D), dtype, 7 * seed + 3, spread)
        c["k"], c["v"] = kv[:, :, 0], kv[:, :, 1]
    else:
        c["k"], c["v"] = normal((nk, kv_heads, D), dtype, 7 * seed + 3, spread), normal((nk, kv_heads, D), dtype, 7 * seed + 4)
    if mask is not None:
        c["mask"] = torch.rand(nk, generator=torch.Generator(device="cuda").manual_seed(seed + 5), device="cuda") < mask
    return c


def triangle(n, m, keep=None):
    seen = torch.arange(m, device="cuda")[None] <= m - n + torch.arange(n, device="cuda")[:, None]
    return seen if keep is None else seen & keep[None]


def reference(c):
    parts, q0, k0 = [], 0, 0
    for n, m in zip(c["q_len"], c["kv_len"]):
        keep = None if c["mask"] is None else c["mask"][k0:k0 + m].bool()
        parts.append(attend(c["q"][q0:q0 + n], c["k"][k0:k0 + m], c["v"][k0:k0 + m], c["scale"], triangle(n, m, keep), c["go"][q0:q0 + n]))
        # A weight below 2^-126 (the smallest normal fp32 number) is formed as zero: off by up to that, which times the other factors of a
        # gradient stays below tolerances relative to the weight.  |dP - delta| <= 2 |grad_out| |value|; a key or query at most its largest.
        size = [t.double() for t in (c["q"][q0:q0 + n], c["k"][k0:k0 + m], c["v"][k0:k0 + m], c["go"][q0:q0 + n])]
        if c["mask"] is not None:
            size[1:3] = [torch.where(keep[:, None, None], t, 0.0) for t in size[1:3]]
        qs, ks, go = (float(size[i].abs().max()) if size[i].numel() else 0.0 for i in (0, 1, 3))
        ds = 2 * abs(c["scale"]) * (float(size[3].norm(dim=-1).max()) if n else 0.0) * (float(size[2].norm(dim=-1).max()) if m else 0.0)
        rows = n * c["q"].shape[1] // c["k"].shape[1]
        for name, term in (("grad_q", m * ds * ks), ("grad_key", rows * ds * qs), ("grad_value", rows * go)):
            parts[-1][name + "_tol"] += 2.0 ** -126 * term
        q0, k0 = q0 + n, k0 + m
    return {name: torch.cat([p[name] for p in parts]) for name in parts[0]}


def run(tiga, c, q_start=None, kv_start=None, untouched=False):
    guard = Guard(torch)
    g = tiga.TriangularRelation(starts(c["q_len"]) if q_start is None else q_start, starts(c["kv_len"]) if kv_start is None else kv_start, c["mask"])
    q, k, v = c["q"], c["k"], c["v"]
    r = {"out": guard.empty(q.shape, q.dtype), "lse": guard.empty(q.shape[:2])}
    tiga.tiga_apply_triangular_attention(g, q, k, v, c["scale"], out=r["out"], lse=r["lse"],
                                         ws=guard.workspace(tiga.tiga_triangular_attention_workspace_bytes(g, q, k, v)))
    for name, like in (("grad_q", q), ("grad_key", k), ("grad_value", k)):
        r[name] = guard.empty(like.shape, like.dtype)
    tiga.tiga_apply_triangular_attention_backward(g, q, k, v, r["out"], r["lse"], c["go"], c["scale"], grad_q=r["grad_q"], grad_key=r["grad_key"],
                                                  grad_value=r["grad_value"],
                                                  ws=guard.workspace(tiga.tiga_triangular_attention_workspace_bytes(g, q, k, v, True)))
    guard.check(allow_untouched=list(r.values()) if untouched else ())
    return r


def check(tiga, c):
    want, got = reference(c), run(tiga, c)
    for name in got:
        close(got[name], want[name], want[name + "_tol"], name)
    again = run(tiga, c)
    for name in got:
        assert torch.equal(got[name], again[name]), f"{name}: reruns must be bit identical"
    return got


LENGTHS = [([1], [1]), ([2], [2]), ([17], [17]), ([65], [65]), ([128, 1, 129], [128, 1, 129]), ([0, 257, 0, 3], [0, 257, 7, 3]), ([300], [1000]), ([40, 3], [400, 130]),
           ([130, 20], [50, 0]), ([31, 1, 2, 90, 17], [63, 64, 65, 127, 17]), ([600], [600])]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("q_len,kv_len", LENGTHS)
def test_lengths(tiga, q_len, kv_len, dtype):
    check(tiga, case(q_len, kv_len, 4, 2, 64, dtype, seed=len(q_len)))


@pytest.mark.parametrize("heads,kv_heads,D,dtype", [(1, 1, 8, F16), (4, 2, 16, BF16), (6, 2, 32, F16), (5, 1, 40, BF16), (3, 3, 72, F16), (8, 2, 80, BF16),
                                                    (7, 1, 96, F16), (12, 4, 128, BF16), (8, 1, 128, F16), (40, 8, 64, BF16), (64, 1, 64, F16)])
def test_heads_and_widths(tiga, heads, kv_heads, D, dtype):
    check(tiga, case([70, 9, 133], [70, 131, 200], heads, kv_heads, D, dtype, seed=D, packed=True))


@pytest.mark.parametrize("dtype,D,keep", [(F16, 64, 0.5), (BF16, 128, 0.1), (BF16, 64, 0.0)])
def test_masks(tiga, dtype, D, keep):
    """Masked keys under the triangle: rows in front of the first key that is left read nothing."""
    c = case([140, 130, 7], [140, 300, 7], 4, 2, D, dtype, mask=keep, seed=11)
    c["mask"][:20] = False
    got = check(tiga, c)
    assert torch.all(got["out"][:20] == 0) and torch.all(got["lse"][:20] == float("-inf")) and torch.all(got["grad_q"][:20] == 0)
    assert torch.all(got["grad_key"][~c["mask"]] == 0) and torch.all(got["grad_value"][~c["mask"]] == 0)


@pytest.mark.parametrize("poison", [float("nan"), float("inf"), "lowest"])
def test_what_no_row_reads_has_no_influence(tiga, poison):
    c = case([140, 70, 0], [140, 90, 30], 2, 1, 64, BF16, mask=0.6, seed=12)
    clean = run(tiga, c)
    fill = torch.finfo(BF16).min if poison == "lowest" else poison
    off = ~c["mask"]
    off[230:] = True                # keys of a segment without rows
    for name in ("k", "v"):
        c[name] = c[name].clone()
        c[name][off] = fill
    got = run(tiga, c)
    for name in got:
        assert torch.equal(got[name], clean[name]), name


def test_rows_that_read_one_key(tiga):
    """A row's only weight is 1 whatever the score: no gradient for the row's query, and the value's is the row's."""
    c = case([1, 1, 5], [1, 1, 5], 2, 2, 64, F16, seed=13)
    got = check(tiga, c)
    assert torch.all(got["grad_q"][:3] == 0) and torch.all(got["grad_key"][:2] == 0)
    assert torch.equal(got["out"][:2], c["v"][:2]) and torch.equal(got["grad_value"][:2], c["go"][:2])


def test_long_sequences(tiga):
    """More tiles than the device has SMs, tiles shared by many blocks, few rows at the end of many keys."""
    check(tiga, case([1500, 333], [1500, 1999], 8, 2, 128, BF16, seed=14))
    check(tiga, case([3], [20000], 2, 2, 64, F16, seed=15))
    check(tiga, case([5000], [5000], 2, 1, 64, BF16, seed=16))


def test_more_segments_than_the_blocks_count_themselves(tiga):
    lens = [1 + (i * 37) % 70 for i in range(300)]
    check(tiga, case(lens, [n + (i % 3) * 20 for i, n in enumerate(lens)], 4, 2, 64, F16, seed=17))


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_large_and_growing_scores(tiga, dtype):
    c = case([700], [700], 2, 2, 64, dtype, seed=18, spread=4.0)
    c["k"] = (c["k"].float() * torch.linspace(0.1, 1.5, 700, device="cuda")[:, None, None]).to(dtype)
    check(tiga, c)
    check(tiga, case([300], [300], 2, 2, 64, dtype, seed=19, scale=0.0))
    check(tiga, case([300], [300], 2, 2, 64, dtype, seed=20, scale=-0.3))


def test_shared_heads_and_rows(tiga):
    """Keys whose heads share storage (a stride of zero), queries whose rows do."""
    c = case([200], [200], 4, 2, 64, BF16, seed=21)
    c["k"], c["q"] = c["k"][:, :1].expand(-1, 2, -1), c["q"][:1].expand(200, -1, -1)
    check(tiga, c)


def test_rows_outside_of_every_segment_are_left_alone(tiga):
    c = case([40, 60], [40, 60], 2, 1, 64, BF16, seed=22)
    want = run(tiga, c)
    pad = lambda t: torch.cat([torch.full_like(t[:5], float("nan")), t, torch.full_like(t[:9], float("nan"))])  # noqa: E731
    c = {name: pad(x) if name in ("q", "k", "v", "go") else x for name, x in c.items()}
    got = run(tiga, c, starts([40, 60], 5), starts([40, 60], 5), untouched=True)
    for name in want:
        assert torch.equal(got[name][5:105], want[name]), name
        assert torch.all(torch.isnan(got[name][:5])) and torch.all(torch.isnan(got[name][105:])), name


def test_gradients_against_differences(tiga):
    """d/de of <out(x + e d), grad_out> against <grad_x, d>, by central differences of the 64-bit formula."""
    c = case([50, 33], [50, 70], 4, 2, 64, F16, seed=23)
    got = run(tiga, c)
    for name, grad in (("q", "grad_q"), ("k", "grad_key"), ("v", "grad_value")):
        d = normal(c[name].shape, torch.float64, 99)
        e = 1e-5
        side = []
        for sign in (1, -1):
            q0 = k0 = 0
            total = 0.0
            for n, m in zip(c["q_len"], c["kv_len"]):
                a = {x: c[x].double() + (sign * e * d if x == name else 0) for x in "qkv"}
                q, k, v = a["q"][q0:q0 + n], a["k"][k0:k0 + m].repeat_interleave(2, 1), a["v"][k0:k0 + m].repeat_interleave(2, 1)
                s = (torch.einsum("nhd,mhd->hnm", q, k) * c["scale"]).masked_fill(~triangle(n, m)[None], -float("inf"))
                total = total + (torch.einsum("hnm,mhd->nhd", torch.softmax(s, -1), v) * c["go"][q0:q0 + n].double()).sum()
                q0, k0 = q0 + n, k0 + m
            side.append(total)
        want, have = float((side[0] - side[1]) / (2 * e)), float((got[grad].double() * d).sum())
        # each entry is off by at most a few half steps of its size (attention_reference.py); 16 of them in the mean square over all entries
        assert abs(want - have) <= 16 * 2.0 ** -11 * float((got[grad].double() * d).norm()) + 1e-6 * abs(want), name


def test_captured_and_replayed_with_other_lengths(tiga):
    c = case([100, 28], [100, 28], 4, 2, 64, BF16, seed=24)
    start = starts([100, 28])
    g = tiga.TriangularRelation(start)
    out, lse, ws = tiga.tiga_apply_triangular_attention(g, c["q"], c["k"], c["v"], c["scale"])
    grads = tiga.tiga_apply_triangular_attention_backward(g, c["q"], c["k"], c["v"], out, lse, c["go"], c["scale"])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tiga.tiga_apply_triangular_attention(g, c["q"], c["k"], c["v"], c["scale"], out=out, lse=lse, ws=ws)
        tiga.tiga_apply_triangular_attention_backward(g, c["q"], c["k"], c["v"], out, lse, c["go"], c["scale"], *grads[:3], ws=grads[3])
    start.copy_(starts([5, 123]))
    graph.replay()
    torch.cuda.synchronize()
    want = reference(dict(c, q_len=[5, 123], kv_len=[5, 123]))
    for name, x in zip(("out", "lse", "grad_q", "grad_key", "grad_value"), (out, lse, *grads[:3])):
        close(x, want[name], want[name + "_tol"], name)


def test_on_another_stream(tiga):
    c = case([100, 28], [100, 28], 4, 2, 64, F16, seed=25)
    want = run(tiga, c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = tiga.TriangularRelation(starts(c["q_len"]))
    side.wait_stream(torch.cuda.current_stream())
    out, lse, _ = tiga.tiga_apply_triangular_attention(g, c["q"], c["k"], c["v"], c["scale"], stream=side)
    grads = tiga.tiga_apply_triangular_attention_backward(g, c["q"], c["k"], c["v"], out, lse, c["go"], c["scale"], stream=side)
    side.synchronize()
    for name, x in zip(("out", "lse", "grad_q", "grad_key", "grad_value"), (out, lse, *grads[:3])):
        assert torch.equal(x, want[name]), name


def test_agrees_with_the_dense_relation_where_every_row_reads_all_keys(tiga):
    """A single row at the end reads all keys: the same work, cut the same way."""
    c = case([1, 1], [300, 77], 4, 2, 64, BF16, seed=26)
    got = run(tiga, c)
    g = tiga.DenseRelation(starts(c["q_len"]), starts(c["kv_len"]))
    out, lse, _ = tiga.tiga_apply_dense_attention(g, c["q"], c["k"], c["v"], c["scale"])
    grads = tiga.tiga_apply_dense_attention_backward(g, c["q"], c["k"], c["v"], out, lse, c["go"], c["scale"])
    for name, x in zip(("out", "lse", "grad_q", "grad_key", "grad_value"), (out, lse, *grads[:3])):
        assert torch.equal(x, got[name]), name


@pytest.mark.parametrize("D", [64, 72, 128])
def test_outputs_and_workspaces_on_any_boundary_of_16_bytes(tiga, D):
    """Results do not depend on whether rows begin on a sector."""
    c = case([300, 40], [300, 70], 4, 2, D, BF16, seed=27)
    want = run(tiga, c)
    g = tiga.TriangularRelation(starts(c["q_len"]), starts(c["kv_len"]))

    def shifted(shape, dtype):
        n = 1
        for s in shape:
            n *= s
        raw = torch.zeros(n + 64, dtype=dtype, device="cuda")
        raw = raw[(-raw.data_ptr() % 32) // raw.element_size() + 16 // raw.element_size():]
        assert raw.data_ptr() % 32 == 16
        return raw[:n].view(shape)
    out, lse = shifted(c["q"].shape, BF16), shifted(c["q"].shape[:2], torch.float32)
    ws = shifted((tiga.tiga_triangular_attention_workspace_bytes(g, c["q"], c["k"], c["v"]),), torch.uint8)
    tiga.tiga_apply_triangular_attention(g, c["q"], c["k"], c["v"], c["scale"], out=out, lse=lse, ws=ws)
    grads = [shifted(x.shape, BF16) for x in (c["q"], c["k"], c["k"])]
    ws = shifted((tiga.tiga_triangular_attention_workspace_bytes(g, c["q"], c["k"], c["v"], True),), torch.uint8)
    tiga.tiga_apply_triangular_attention_backward(g, c["q"], c["k"], c["v"], out, lse, c["go"], c["scale"], *grads, ws=ws)
    for name, x in zip(("out", "lse", "grad_q", "grad_key", "grad_value"), (out, lse, *grads)):
        assert torch.equal(x, want[name]), name


@pytest.mark.parametrize("lens", [[65], [300, 40]])
def test_gradients_that_are_wanted(tiga, lens):
    """Each gradient by itself is what it is beside the others."""
    c = case(lens, lens, 4, 2, 64, F16, seed=28)
    want = run(tiga, c)
    g = tiga.TriangularRelation(starts(lens))
    gq, none, no, _ = tiga.tiga_apply_triangular_attention_backward(g, c["q"], c["k"], c["v"], want["out"], want["lse"], c["go"], c["scale"], want_kv=False)
    assert none is None and no is None and torch.equal(gq, want["grad_q"])
    none, gk, gv, _ = tiga.tiga_apply_triangular_attention_backward(g, c["q"], c["k"], c["v"], want["out"], want["lse"], c["go"], c["scale"], want_q=False)
    assert none is None and torch.equal(gk, want["grad_key"]) and torch.equal(gv, want["grad_value"])
    only = torch.empty_like(c["k"])
    tiga.tiga_apply_triangular_attention_backward(g, c["q"], c["k"], c["v"], want["out"], want["lse"], c["go"], c["scale"], grad_value=only, want_q=False, want_kv=False)
    assert torch.equal(only, want["grad_value"])


def test_mask_that_leaves_one_key_under_the_triangle(tiga):
    c = case([20], [20], 2, 1, 64, BF16, seed=29)
    c["mask"] = torch.zeros(20, dtype=torch.bool, device="cuda")
    c["mask"][7] = True
    got = check(tiga, c)
    assert torch.all(got["out"][:7] == 0) and torch.all(got["grad_q"] == 0) and torch.all(got["grad_key"] == 0)
