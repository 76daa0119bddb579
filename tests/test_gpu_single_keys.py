"""Gradients of rows whose mask leaves a single key: its weight is 1 whatever the score, so scores have no gradient.  Exactly zero where the row
reaches at most 32 keys; behind that what rounding leaves of dP - delta.

With one key out is the value exactly and both dP and delta are sums of the same D products in fp32, each off by at most (D + 8) 2^-23 of
sum_d |grad_out value|; times p (1 up to 2^-10), the scale and the key.  fp16 adds the smallest step of dS, as in attention_reference.py."""
import pytest

from attention_reference import tiny

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def tiga():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_24802_b200 import api
    return api


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def run(tiga, kind, n, m, kept, heads, kv_heads, D, dtype):
    """One segment; returns what grad_q holds and what it may hold at most if a row reads the key `kept` alone."""
    g = torch.Generator(device="cuda").manual_seed(n + m + kept)
    q, k, v, go = (torch.randn(s, generator=g, device="cuda").to(dtype) for s in ((n, heads, D), (m, kv_heads, D), (m, kv_heads, D), (n, heads, D)))
    mask = torch.zeros(m, dtype=torch.bool, device="cuda")
    mask[kept] = True
    scale = D ** -0.5
    forward, backward = getattr(tiga, f"tiga_apply_{kind}_attention"), getattr(tiga, f"tiga_apply_{kind}_attention_backward")
    relation = (tiga.DenseRelation if kind == "dense" else tiga.TriangularRelation)(ints(0, n), ints(0, m), mask)
    out, lse, _ = forward(relation, q, k, v, scale)
    grad_q, grad_key, grad_value, _ = backward(relation, q, k, v, out, lse, go, scale)
    reads = torch.ones(n, dtype=torch.bool, device="cuda") if kind == "dense" else m - n + torch.arange(n, device="cuda") >= kept
    one = v[kept].repeat_interleave(heads // kv_heads, 0)
    assert torch.equal(out[reads], one[None].expand(int(reads.sum()), -1, -1)) and torch.all(out[~reads] == 0) and torch.all(grad_q[~reads] == 0)
    key = k[kept].double().abs().repeat_interleave(heads // kv_heads, 0)
    floor = 2.0 ** -25 * 2.0 ** -13 * 2 * float(go.double().norm(dim=-1).max()) * float(v.double().norm(dim=-1).max()) if dtype == F16 else 0.0
    most = scale * (2 * (D + 8) * 2.0 ** -23 * (go.double() * one.double()).abs().sum(-1)[..., None] * (1 + 2.0 ** -9) + floor) * key[None] * (1 + 2.0 ** -7) + tiny(dtype)
    others = torch.ones(m, dtype=torch.bool, device="cuda")
    others[kept] = False
    assert torch.all(grad_key[others] == 0) and torch.all(grad_value[others] == 0)
    return grad_q, most


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("heads,kv_heads,D", [(2, 2, 64), (8, 2, 128), (3, 1, 40)])
@pytest.mark.parametrize("n,m,kept", [(40, 40, 3), (300, 300, 7), (300, 300, 40), (200, 700, 100), (1, 1000, 999), (1500, 1500, 33)])
def test_rows_that_reach_far(tiga, n, m, kept, heads, kv_heads, D, dtype):
    grad_q, most = run(tiga, "triangular", n, m, kept, heads, kv_heads, D, dtype)
    reaches = m - n + 1 + torch.arange(n, device="cuda")
    assert torch.all(grad_q[reaches <= 32] == 0)
    assert torch.all(grad_q.double().abs() <= most)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("m,kept", [(1, 0), (32, 31), (33, 5), (400, 0), (1000, 999)])
def test_dense_segments(tiga, m, kept, dtype):
    grad_q, most = run(tiga, "dense", 150, m, kept, 4, 2, 64, dtype)
    assert torch.all(grad_q == 0) if m <= 32 else torch.all(grad_q.double().abs() <= most)
