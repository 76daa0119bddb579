"""Eviction from lists that one block's shared memory does not hold: a cluster for each of a few, one block for each of many.  Compared
exactly with a plain restatement, as in test_gpu_evict.py."""
import pytest

from test_gpu_evict import BF16, F16, check, make, tiga  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["spread", "ties", "near"])
@pytest.mark.parametrize("lens,heads,keep,recent", [([40960], 1, 700, 30), ([40961], 1, 700, 30), ([41000, 300, 0], 2, 5000, 100), ([45011], 1, 45011, 100), ([45011], 2, 45010, 45010),
                                                    ([50000] + [77] * 20, 1, 64, 64), ([43000] + [9] * 40, 1, 2000, 0)])
def test_lists(tiga, lens, heads, keep, recent, kind):  # noqa: F811
    check(tiga, make(lens, heads, 8, F16, 64, 64, keep, seed=len(lens) + keep, kind=kind), keep, recent)


@pytest.mark.parametrize("page", [1, 7, 24, 33, 100])
def test_missing_pages(tiga, page):  # noqa: F811
    c = make([44000, 1000], 1, 8, BF16, page, 16, 900, seed=page)
    g = torch.Generator(device="cuda").manual_seed(page)
    c["table"][torch.rand(c["table"].shape, generator=g, device="cuda") < 0.3] = -1
    check(tiga, c, 900, 40)


def test_special_weights(tiga):  # noqa: F811
    c = make([42000], 3, 8, F16, 16, 16, 500, seed=7)
    w = c["weights"]
    w[0, 0] = 0.0
    w[0, 1] = float("nan")
    w[0, 1, 30000:30100] = -float("inf")
    w[0, 2, ::3] = float("inf")
    check(tiga, c, 500, 20)


def test_fewer_weights_than_positions(tiga):  # noqa: F811
    check(tiga, make([42000], 2, 8, F16, 16, 16, 500, seed=8, places=20000), 500, 10)
    check(tiga, make([42000], 2, 8, F16, 16, 16, 500, seed=9, places=100), 500, 10)
