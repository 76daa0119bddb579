"""How attention cuts its work into units: the closed forms of the triangle against the tiles one by one, on the host."""
import ctypes
import os
import random
import subprocess

import pytest


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    from paper_2609_24802_b200 import build
    lib = str(tmp_path_factory.mktemp("cut") / "attention_cut.so")
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "attention_cut.cu")
    subprocess.run([build._nvcc()] + build.NVCC_FLAGS + ["-shared", src, "-o", lib], check=True, capture_output=True)
    lib = ctypes.CDLL(lib)
    lib.run_lattice.restype, lib.run_lattice.argtypes = ctypes.c_longlong, [ctypes.c_longlong] * 4
    return lib


def test_lattice_points(cut):
    rng = random.Random(1)
    for _ in range(4000):
        n, a, b, m = rng.randint(0, 40), rng.randint(0, 300), rng.randint(0, 5000), rng.randint(1, 300)
        assert cut.run_lattice(n, a, b, m) == sum((a * k + b) // m for k in range(n)), (n, a, b, m)
    for n, a, b, m in [(1 << 20, 256, 255 + 7 * 1000, 128 * 7), (100000, 128, (1 << 31) * 5, 128 * 5)]:
        assert cut.run_lattice(n, a, b, m) == sum((a * k + b) // m for k in range(n))


@pytest.mark.parametrize("keys", [0, 1])
@pytest.mark.parametrize("causal", [0, 1])
def test_units_in_front_of_a_tile(cut, keys, causal):
    rng = random.Random(2 + keys)
    cases = [(1, 1, 1, 1), (1, 0, 5, 5), (3, 7, 0, 0), (64, 1, 1, 1), (5, 300, 2, 2), (4, 4096, 4096, 4096), (1, 5000, 5000, 9000), (7, 3, 100000, 100000)]
    for _ in range(3000):
        nq = rng.choice([0, 1, 2, rng.randint(1, 300), rng.randint(1, 5000)])
        length = rng.choice([0, 1, nq, nq + rng.randint(0, 400), max(nq - rng.randint(0, 400), 0), rng.randint(0, 20000)])
        cases.append((rng.choice([1, 2, 3, 4, 5, 7, 8, 16, 64, 100]), nq, length if rng.random() < 0.8 else rng.randint(0, length), length))
    for group, nq, nk, length in cases:
        assert cut.run_cut(keys, causal, group, nq, nk, length) == 0, (keys, causal, group, nq, nk, length)
