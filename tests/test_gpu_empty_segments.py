"""GPU parity of the triangular relation where most segments are empty, as in a batch with places for a fixed number of sequences, against
64 bits (tolerances: attention_reference.py)."""
import pytest

from test_gpu_triangular_attention import BF16, F16, case, check, tiga  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("n_seg", [1, 2, 9, 16, 17, 64, 255, 256, 257, 3000])
@pytest.mark.parametrize("where", ["front", "end", "spread"])
def test_few_rows_in_many_segments(tiga, n_seg, where, dtype):  # noqa: F811
    real = [37, 5, 16, 1][:max(1, min(4, n_seg // 2))]
    q_len = [0] * n_seg
    for i, n in enumerate(real):
        q_len[{"front": i, "end": n_seg - len(real) + i, "spread": i * (n_seg // len(real))}[where]] = n
    kv_len = [n + (7 if n == 5 else 0) for n in q_len]
    check(tiga, case(q_len, kv_len, 4, 2, 64, dtype, mask=0.7 if where == "spread" else None, seed=n_seg))


def test_captured_and_replayed_with_other_segments(tiga):  # noqa: F811
    """One graph for whatever number of sequences a batch of 1000 places holds."""
    from attention_reference import close
    from test_gpu_triangular_attention import reference, starts
    c = case([20, 30, 10], [20, 30, 10], 4, 2, 64, F16, seed=5)
    bounds = torch.full((1001,), 60, dtype=torch.int32, device="cuda")
    g = tiga.TriangularRelation(bounds)
    q, k, v = c["q"], c["k"], c["v"]
    out, lse, ws = tiga.tiga_apply_triangular_attention(g, q, k, v, c["scale"])
    grads = list(tiga.tiga_apply_triangular_attention_backward(g, q, k, v, out, lse, c["go"], c["scale"]))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tiga.tiga_apply_triangular_attention(g, q, k, v, c["scale"], out=out, lse=lse, ws=ws)
        tiga.tiga_apply_triangular_attention_backward(g, q, k, v, out, lse, c["go"], c["scale"], *grads[:3], ws=grads[3])
    for lens in ([60], [20, 30, 10], [1] * 60, [0] * 500 + [17, 43]):
        bounds.copy_(starts(lens + [0] * (1000 - len(lens))))
        graph.replay()
        torch.cuda.synchronize()
        want = reference(dict(c, q_len=lens, kv_len=lens))
        for name, got in zip(("out", "lse", "grad_q", "grad_key", "grad_value"), [out, lse] + grads[:3]):
            close(got, want[name], want[name + "_tol"], name)
