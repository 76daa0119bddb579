"""A segment's results are its own.  Against 64 bits (tolerances: attention_reference.py; what fp16 cannot hold of dS is counted there by
segment)."""
import pytest

from attention_reference import close
from test_gpu_dense_attention import case, reference, run

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
