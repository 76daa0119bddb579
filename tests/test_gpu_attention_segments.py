"""A segment's results are its own.  Against 64 bits (tolerances: attention_reference.py; what fp16 cannot hold of dS is counted there by
segment)."""
import pytest

from attention_reference import attend, close
from test_gpu_dense_attention import case, reference, run, starts

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def tiga():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_24802_b200 import api
    return api


# ------------------------------------------------------------------------------------------------ keys of segments without rows

POISON = [float("nan"), float("inf"), -float("inf"), "lowest"]
UNREAD = [([40, 0, 70, 0], [100, 60, 200, 300], None), ([0, 5, 0, 0], [1, 9, 1, 17], None), ([40, 0, 70, 0], [100, 60, 200, 300], 0.6), ([300, 0], [5, 2000], None), ([0], [130], None)]


def poison_unread_keys(tiga, q_len, kv_len, masked, poison, dtype):
    c = case(q_len, kv_len, 4, 2, 64, dtype, mask=masked, seed=41)
    c["go"] = (c["go"].float() * 2.0 ** -9).to(dtype)
    clean = run(tiga, c)
    want = reference(c)
    for name in clean:
        close(clean[name], want[name], want[name + "_tol"], name)
    unread, k0 = torch.zeros(sum(kv_len), dtype=torch.bool, device="cuda"), 0
    for n, m in zip(q_len, kv_len):
        unread[k0:k0 + m] = n == 0
        k0 += m
    for name in ("k", "v"):
        c[name] = c[name].clone()
        c[name][unread] = torch.finfo(dtype).min if poison == "lowest" else poison
    got = run(tiga, c)
    for name in got:
        assert torch.equal(got[name], clean[name]), name
    assert torch.all(got["grad_key"][unread] == 0) and torch.all(got["grad_value"][unread] == 0)


@pytest.mark.parametrize("poison", POISON)
@pytest.mark.parametrize("q_len,kv_len,masked", UNREAD)
def test_keys_of_segments_without_rows_have_no_influence(tiga, q_len, kv_len, masked, poison):
    poison_unread_keys(tiga, q_len, kv_len, masked, poison, BF16)


@pytest.mark.parametrize("poison", POISON)
@pytest.mark.parametrize("q_len,kv_len,masked", UNREAD)
def test_keys_of_segments_without_rows_set_no_scale_in_f16(tiga, q_len, kv_len, masked, poison):
    poison_unread_keys(tiga, q_len, kv_len, masked, poison, F16)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("poison", POISON)
def test_rows_that_read_nothing_have_no_influence(tiga, poison, dtype):
    """Rows of segments without keys, or whose mask leaves none: queries and gradients of anything."""
    c = case([40, 70, 9, 130], [100, 0, 60, 30], 4, 2, 64, dtype, mask=0.6, seed=47)
    c["mask"][100:160] = False
    c["go"] = (c["go"].float() * 2.0 ** -9).to(dtype)
    clean = run(tiga, c)
    for name in ("q", "go"):
        c[name][40:119] = torch.finfo(dtype).min if poison == "lowest" else poison
    got = run(tiga, c)
    for name in got:
        assert torch.equal(got[name], clean[name]), name
    assert torch.all(got["grad_q"][40:119] == 0) and torch.all(got["out"][40:119] == 0)


# ------------------------------------------------------------------------------------------------ gradients of another size next door

def _beside(kinds, D=64, heads=2):
    """Segments "small" (long sums of small gradients) beside others, in fp16."""
    q_len, kv_len = zip(*[{"small": (60, 9000), "large": (90, 40), "broken": (7, 300), "few": (130, 12)}[k] for k in kinds])
    c = case(list(q_len), list(kv_len), heads, 1, D, F16, seed=42, spread=0.2)
    q0 = k0 = 0
    for kind, n, m in zip(kinds, q_len, kv_len):
        go, v = c["go"][q0:q0 + n], c["v"][k0:k0 + m]
        if kind == "large":
            go.copy_(go.float() * 2.0 ** 8)
            v.copy_(v.float() * 4)
        else:
            go.copy_(go.float() * 2.0 ** -9)
        if kind == "broken":
            go[0], v[1] = float("inf"), float("nan")
        q0, k0 = q0 + n, k0 + m
    return c


@pytest.mark.parametrize("kinds", [["small"], ["small", "large"], ["large", "small", "few"], ["small", "broken"], ["broken", "few", "large", "small"], ["large"] * 3 + ["small"] + ["broken"] * 3])
def test_small_gradients_keep_their_digits_beside_large_ones(tiga, kinds):
    c = _beside(kinds)

    def step():         # (without run()'s guards, which take a NaN for an element that was not written: broken segments have some)
        g = tiga.DenseRelation(starts(c["q_len"]), starts(c["kv_len"]))
        out, lse, _ = tiga.tiga_apply_dense_attention(g, c["q"], c["k"], c["v"], c["scale"])
        grads = tiga.tiga_apply_dense_attention_backward(g, c["q"], c["k"], c["v"], out, lse, c["go"], c["scale"])
        return dict(zip(("out", "lse", "grad_q", "grad_key", "grad_value"), (out, lse) + grads[:3]))
    got, q0, k0 = step(), 0, 0
    for kind, n, m in zip(kinds, c["q_len"], c["kv_len"]):
        if kind != "broken":
            want = attend(c["q"][q0:q0 + n], c["k"][k0:k0 + m], c["v"][k0:k0 + m], c["scale"], torch.ones(n, m, dtype=torch.bool, device="cuda"), c["go"][q0:q0 + n])
            for name, (a, b) in (("out", (q0, q0 + n)), ("lse", (q0, q0 + n)), ("grad_q", (q0, q0 + n)), ("grad_key", (k0, k0 + m)), ("grad_value", (k0, k0 + m))):
                close(got[name][a:b], want[name], want[name + "_tol"], f"{name} of a {kind} segment")
        q0, k0 = q0 + n, k0 + m
    again = step()
    for name in got:
        assert torch.equal(got[name].view(torch.int32 if name == "lse" else torch.int16), again[name].view(torch.int32 if name == "lse" else torch.int16)), name


@pytest.mark.parametrize("n", [40, 700])
def test_many_segments_of_many_sizes_in_f16(tiga, n):
    """Gradients of every segment 2^-10 to 2^10 times those of a plain one; few rows, some segments empty, more segments than blocks count themselves."""
    q_len = [(i * 7) % 4 + (90 if i % 50 == 3 else 0) for i in range(n)]
    kv_len = [(i * 5) % 23 + (400 if i % 60 == 3 else 0) for i in range(n)]
    c = case(q_len, kv_len, 2, 1, 32, F16, seed=43, spread=0.5)
    q0, at = 0, []
    for i, a in enumerate(q_len):
        at.append(q0)
        c["go"][q0:q0 + a] = (c["go"][q0:q0 + a].float() * 2.0 ** ((i * 11) % 21 - 10)).to(F16)
        q0 += a
    got, k0 = run(tiga, c), 0
    for s, (a, b) in enumerate(zip(q_len, kv_len)):
        if s % 7 in (0, 3):
            q0 = at[s]
            want = attend(c["q"][q0:q0 + a], c["k"][k0:k0 + b], c["v"][k0:k0 + b], c["scale"], torch.ones(a, b, dtype=torch.bool, device="cuda"), c["go"][q0:q0 + a])
            for name, (i, j) in (("grad_q", (q0, q0 + a)), ("grad_key", (k0, k0 + b)), ("grad_value", (k0, k0 + b))):
                close(got[name][i:j], want[name], want[name + "_tol"], f"{name} of segment {s}")
        k0 += b


@pytest.mark.parametrize("rows,keys,heads", [(60, 90, 2), (700, 900, 4)])
def test_graph_replays_start_from_no_norms_in_f16(tiga, rows, keys, heads):
    """One captured step, replayed with large gradients and then with small ones, bit for bit as eager calls: in one block, and where a
    kernel in front clears the norms."""
    a = case([rows, rows], [keys, keys], heads, heads, 64, F16, seed=51)
    b = case([rows + 30, rows - 30], [keys - 11, keys + 11], heads, heads, 64, F16, seed=52)
    b["go"] = (b["go"].float() * 2.0 ** -12).to(F16)
    qs, ks = starts(a["q_len"]), starts(a["kv_len"])
    x = {n: a[n].clone() for n in ("q", "k", "v", "go")}
    g = tiga.DenseRelation(qs, ks)

    def step():
        out, lse, ws = tiga.tiga_apply_dense_attention(g, x["q"], x["k"], x["v"], a["scale"])
        return out, lse, *tiga.tiga_apply_dense_attention_backward(g, x["q"], x["k"], x["v"], out, lse, x["go"], a["scale"]), ws
    step()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        got = step()
    for c in (a, b, a, b):
        qs.copy_(starts(c["q_len"]))
        ks.copy_(starts(c["kv_len"]))
        for n in x:
            x[n].copy_(c[n])
        graph.replay()
        want = run(tiga, c)
        for t, name in zip(got, ("out", "lse", "grad_q", "grad_key", "grad_value")):
            assert torch.equal(t, want[name]), name
