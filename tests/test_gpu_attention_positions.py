"""Positions of new tokens in caches that are longer than their table: append and attention agree on them, and attention reads what is
there of the triangle.  Against 64 bits (tolerances: attention_reference.py)."""
import pytest

from attention_reference import attend, close
from test_gpu_paged_attention import make, normal, run, starts

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def tiga():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_24802_b200 import api
    return api


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("q_len,kv_len,page,columns", [([10], [70], 16, 4), ([1], [70], 16, 4), ([10, 3, 9], [70, 64, 9], 16, 4), ([500, 20], [1000, 630], 64, 10), ([100], [150], 16, 2)])
def test_the_triangle_of_caches_beyond_their_table(tiga, q_len, kv_len, page, columns, dtype):
    """Token t is at position kv_len - n + t, whatever the table holds: it reads the positions up to its own that exist."""
    c = make(q_len, kv_len, 8, 2, 64, dtype, page, seed=44)
    c["table"] = c["table"][:, :columns].contiguous()
    out, lse = run(tiga, c)
    q0 = 0
    for b, (n, m) in enumerate(zip(q_len, kv_len)):
        there = min(m, columns * page)
        seen = torch.arange(there, device="cuda")[None] <= m - n + torch.arange(n, device="cuda")[:, None]
        want = attend(c["q"][q0:q0 + n], c["keys"][b][:there], c["values"][b][:there], c["scale"], seen)
        close(out[q0:q0 + n], want["out"], want["out_tol"], f"out of sequence {b}")
        close(lse[q0:q0 + n], want["lse"], want["lse_tol"], f"lse of sequence {b}")
        q0 += n


def test_the_longest_length_reads_the_whole_table(tiga):
    c = make([40], [160], 4, 2, 64, BF16, 16, seed=45)
    c["table"] = c["table"][:, :10].contiguous()
    want = run(tiga, c, causal=False)
    c["lens"].fill_(2 ** 31 - 1)
    got = run(tiga, c)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_appended_tokens_read_themselves_beyond_the_table(tiga):
    """Append and attention agree on positions: the tokens that still had a place read it."""
    page, hk, D, n, length = 16, 2, 64, 10, 70
    pages = torch.zeros(4, page, hk, D, dtype=BF16, device="cuda")
    cache = tiga.PagedCache(pages, pages.clone(), torch.arange(4, dtype=torch.int32, device="cuda")[None], torch.tensor([length], dtype=torch.int32, device="cuda"))
    q, v = normal((n, hk, D), BF16, 1), normal((n, hk, D), BF16, 2)
    tiga.tiga_paged_append(cache, q * 64, v, starts([n]))           # a token's own score is far above all others
    out, _, _ = tiga.tiga_apply_paged_attention(cache, q, starts([n]), 1.0)
    assert torch.equal(out[:4], v[:4])


@pytest.mark.parametrize("causal", [True, False])
def test_a_table_without_entries_holds_nothing(tiga, causal):
    """No place at all: rows read nothing and are written, as where every entry names no page."""
    c = make([5, 1], [12, 3], 4, 2, 64, F16, 16, seed=46)
    c["table"] = c["table"][:, :0].contiguous()
    out, lse = run(tiga, c, causal)
    assert torch.all(out == 0) and torch.all(lse == -float("inf"))
    before = c["key_pages"].clone()
    new = normal((6, 2, 64), F16, 3)
    tiga.tiga_paged_append(tiga.PagedCache(c["key_pages"], c["value_pages"], c["table"], c["lens"]), new, new, starts([5, 1]))
    assert torch.equal(c["key_pages"].nan_to_num(nan=9.0), before.nan_to_num(nan=9.0))
