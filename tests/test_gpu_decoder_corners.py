"""Corners of a decoder's operators that a program in service reaches, against 64 bits: users of a shared prompt who have nothing to say."""
import pytest

from attention_reference import close
from test_gpu_shared_attention import BF16, F16, check as check_shared, ints, make as make_shared, reference as shared_reference, starts, tiga  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ shared prefixes

IDLE = [
    [(512, [(0, 0), (1, 30), (1, 60), (1, 5), (1, 9)])],
    [(512, [(0, 0), (0, 0), (0, 0), (2, 30), (1, 60), (1, 5), (3, 9)])],
    [(640, [(0, 0), (1, 70), (0, 0), (1, 9), (1, 5), (0, 0)]), (256, [(0, 0), (0, 0)]), (1000, [(1, 80), (0, 0), (1, 90), (1, 1)])],
]


@pytest.mark.parametrize("groups", IDLE)
@pytest.mark.parametrize("row", ["cleared", "reused"])
@pytest.mark.parametrize("length", [0, 100])
def test_users_without_new_tokens_may_have_lost_their_pages(tiga, groups, row, length):  # noqa: F811
    """A member without new tokens reads nothing: neither its length nor its row of the table matters, in the first place or behind it."""
    c = make_shared(groups, 8, 2, 64, BF16, 16, seed=21)
    for s, n in enumerate(c["q_len"]):
        if n == 0:
            c["table"][s] = -1 if row == "cleared" else c["table"][c["q_len"].index(1)].flip(0)
            c["lens"][s] = length
    check_shared(tiga, c)
    check_shared(tiga, c, causal=False)


def test_a_user_leaves_between_replays(tiga):  # noqa: F811
    """The same graph, with the first member's token and then without it, when its pages are another's."""
    c = make_shared([(512, [(1, 30), (1, 60), (1, 5), (1, 9), (1, 1), (1, 90)])], 4, 2, 64, F16, 16, seed=22)
    cache, prefixes = tiga.PagedCache(c["key_pages"], c["value_pages"], c["table"], c["lens"]), tiga.SharedPrefixes(c["group_start"], c["shared"])
    start = starts([1] * 6)
    out, lse, ws = tiga.tiga_apply_shared_attention(cache, prefixes, c["q"], start, c["scale"])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tiga.tiga_apply_shared_attention(cache, prefixes, c["q"], start, c["scale"], out=out, lse=lse, ws=ws)
    for q_len in ([1] * 6, [0, 1, 1, 1, 1, 1], [0, 0, 1, 1, 1, 1]):
        for s, n in enumerate(q_len):
            if n == 0:
                c["table"][s], c["lens"][s] = c["table"][3].flip(0), 0
        start.copy_(starts(q_len))
        graph.replay()
        torch.cuda.synchronize()
        want, n = shared_reference(dict(c, q_len=q_len, q=c["q"][:sum(q_len)]), True), sum(q_len)
        close(out[:n], want["out"], want["out_tol"], "out")
        close(lse[:n], want["lse"], want["lse_tol"], "lse")
