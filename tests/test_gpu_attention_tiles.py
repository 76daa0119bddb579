"""Items that follow one another in a block of the attention kernels: tiles of one half behind tiles of two, odd and even counts of
steps, single steps.  Against 64 bits (tolerances: attention_reference.py), and bit for bit against other runs."""
import pytest

from attention_reference import attend, close
from test_gpu_dense_attention import starts, normal

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def tiga():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_24802_b200 import api
    return api


@pytest.mark.parametrize("dtype,D,heads,kv_heads", [(BF16, 64, 8, 8), (F16, 128, 12, 6), (BF16, 128, 16, 4)])
def test_short_tiles_behind_long_ones(tiga, dtype, D, heads, kv_heads):
    """A tile of at most 128 rows deals its steps out to both halves, so the halves end with counts of their own; a tile of more rows
    does not bring them together.  About twenty items a block."""
    group = heads // kv_heads
    q_len, kv_len = [], []
    for i in range(240):
        q_len.append([300, 1, 129, 40, 256, 260][i % 6] // group + 1)
        kv_len.append([128 * 3, 100, 128 * 5 - 7, 1, 128 * 2, 128 * 7, 128][i % 7])
    q, k, v = normal((sum(q_len), heads, D), dtype, 1), normal((sum(kv_len), kv_heads, D), dtype, 2), normal((sum(kv_len), kv_heads, D), dtype, 3)
    g = tiga.DenseRelation(starts(q_len), starts(kv_len))
    out, lse, ws = tiga.tiga_apply_dense_attention(g, q, k, v, D ** -0.5)
    q0 = k0 = 0
    for i, (n, m) in enumerate(zip(q_len, kv_len)):
        if i % 5 < 2:
            want = attend(q[q0:q0 + n], k[k0:k0 + m], v[k0:k0 + m], D ** -0.5, torch.ones(n, m, dtype=torch.bool, device="cuda"))
            close(out[q0:q0 + n], want["out"], want["out_tol"], f"out of segment {i}")
            close(lse[q0:q0 + n], want["lse"], want["lse_tol"], f"lse of segment {i}")
        q0, k0 = q0 + n, k0 + m
    for _ in range(20):
        again = tiga.tiga_apply_dense_attention(g, q, k, v, D ** -0.5, ws=ws)
        assert torch.equal(again[0], out) and torch.equal(again[1], lse)
