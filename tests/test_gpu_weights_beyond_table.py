"""GPU parity of accumulated attention weights where a sequence is longer than its row of the page table: the positions behind it receive
nothing and keep what they had (tolerances: test_gpu_attention_weights.py)."""
import pytest

from attention_reference import close
from parity import Guard
from test_gpu_attention_weights import BF16, F16, make, masses, reference, starts, tiga  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def check(tiga, c, entries, length, causal=True, added=True):  # noqa: F811
    """The table cut to `entries` pages a sequence, room for `length` weights."""
    room = entries * c["page"]
    table = c["table"][:, :entries].contiguous()
    cache = tiga.PagedCache(c["pages"], c["pages"], table, c["lens"])
    lse = masses(c, causal)
    B, hk = len(c["kv_len"]), c["pages"].shape[2]
    before = torch.rand((B, hk, length + 5), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda") if added else None
    guard = Guard(torch)
    out = guard.empty((B, hk, length))
    out.fill_(-7.0)
    want, tol = reference(c, lse, causal, before, out)
    for b, n in enumerate(c["kv_len"]):
        here = slice(room, max(min(n, length), room))
        want[b, :, here] = before[b, :, here].double() if added else 0.0
        tol[b, :, here] = 0.0
    tiga.tiga_paged_attention_weights(cache, c["q"], starts(c["q_len"]), lse, c["scale"], causal=causal, before=before, weights=out,
                                      ws=guard.workspace(tiga.tiga_paged_weights_workspace_bytes(cache, c["q"])))
    guard.check()
    close(out, want, tol, "weights")
    if added:               # in place
        tiga.tiga_paged_attention_weights(cache, c["q"], starts(c["q_len"]), lse, c["scale"], causal=causal, before=before, weights=before)
        for b, n in enumerate(c["kv_len"]):
            n = min(n, length)
            assert torch.equal(before[b, :, :n], out[b, :, :n])


@pytest.mark.parametrize("added", [True, False])
@pytest.mark.parametrize("q_len,kv_len,page,entries,length", [([1], [777], 16, 10, 777), ([1, 1, 1], [5, 300, 64], 8, 8, 301), ([200, 3], [515, 700], 32, 4, 650),
                                                              ([0, 2], [90, 40], 7, 3, 100), ([9], [1000], 64, 1, 70), ([1] * 300, [1 + i for i in range(300)], 16, 2, 290)])
def test_sequences_longer_than_the_table(tiga, q_len, kv_len, page, entries, length, added):  # noqa: F811
    for causal, dtype in ((True, F16), (False, BF16)):
        check(tiga, make(q_len, kv_len, 4, 2, 64, dtype, page, seed=page), entries, length, causal, added)


def test_a_table_without_entries(tiga):  # noqa: F811
    check(tiga, make([1, 2], [50, 7], 4, 2, 64, BF16, 16, seed=3), 0, 40)


def test_strided_weights_behind_the_table(tiga):  # noqa: F811
    c = make([3], [90], 4, 2, 64, BF16, 16, seed=4)
    cache = tiga.PagedCache(c["pages"], c["pages"], c["table"][:, :2].contiguous(), c["lens"])
    lse = masses(c, True)
    before = torch.rand((2, 1, 96), device="cuda").transpose(0, 1)
    want, _ = tiga.tiga_paged_attention_weights(cache, c["q"], starts([3]), lse, c["scale"], before=before.contiguous())
    wide = torch.full((2, 3, 200), -3.0, device="cuda")
    tiga.tiga_paged_attention_weights(cache, c["q"], starts([3]), lse, c["scale"], before=before, weights=wide[:, 1:2, 4:100].transpose(0, 1))
    assert torch.equal(wide[:, 1, 4:94], want[0, :, :90]) and torch.equal(want[0, :, 32:90], before[0, :, 32:90])
    wide[:, 1, 4:94] = -3.0
    assert torch.all(wide == -3.0)
