"""How attention deals out its work to blocks, on the host."""
import ctypes
import os
import random
import subprocess

import pytest


@pytest.fixture(scope="module")
def pieces(tmp_path_factory):
    from paper_2609_24802_b200 import build
    lib = str(tmp_path_factory.mktemp("pieces") / "attention_pieces.so")
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "attention_pieces.cu")
    subprocess.run([build._nvcc()] + build.NVCC_FLAGS + ["-shared", src, "-o", lib], check=True, capture_output=True)
    lib = ctypes.CDLL(lib)
    lib.run_prepare_blocks.restype = ctypes.c_longlong
    lib.run_prepare_blocks.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_longlong] + [ctypes.c_int] * 3
    return lib


@pytest.mark.parametrize("lanes", [8, 16])
@pytest.mark.parametrize("heads", [1, 2, 16, 40])
def test_many_segments_have_many_blocks_prepare_them(pieces, heads, lanes):
    """Whatever the number of rows: a warp looks into at most 32 places for rows of few keys (one block, 8 warps, for 16 blocks' work of 16
    looks each), or the device has no more room."""
    for rows in (0, 1, 125, 5000):
        for n_seg in (1, 2, 15, 17, 100, 255, 256, 1000, 10000, 1 << 24):
            blocks = pieces.run_prepare_blocks(1, n_seg, rows, heads, lanes, 148)
            looks = n_seg * 16 * -(-heads * lanes // 32)
            assert 1 <= blocks <= 4 * 148 and (looks <= 32 * 8 * blocks or blocks == 4 * 148), (rows, n_seg, blocks)
            assert pieces.run_prepare_blocks(0, n_seg, rows, heads, lanes, 148) == pieces.run_prepare_blocks(0, 1, rows, heads, lanes, 148)


def test_a_short_segment_is_prepared_by_one_block(pieces):
    """65 rows of two heads, and one launch less."""
    assert pieces.run_prepare_blocks(1, 1, 65 + 33, 2, 8, 148) == 1


def lines(kind, causal, rng):
    """nq, nk, length of some segments, as the entry points make them."""
    n = []
    for _ in range(rng.randint(1, 12)):
        nq = rng.choice([0, 1, 1, rng.randint(1, 40), rng.randint(1, 400), rng.randint(1, 3000)])
        length = rng.choice([0, 1, nq, nq, nq + rng.randint(0, 500), rng.randint(0, 6000)])
        if kind == 6:
            if rng.random() < 0.3:
                n.append((nq, length, length + nq))            # a group's rows, all of which read what is shared
                continue
            nk = length if rng.random() < 0.9 else rng.randint(0, length)
        else:
            nk = length
        n.append((nq, nk, length))
    return n


# kinds and what a tile costs beside its steps, as in the kernels' calls; under the triangle or not
CUTS = [(0, 0, 0), (0, 0, 1), (1, 0, 0), (2, 0, 0), (3, 4, 1), (4, 2, 1), (5, 2, 1), (6, 5, 0), (6, 5, 1), (7, 0, 0), (7, 0, 1), (3, 7, 1), (5, 1, 1), (6, 1, 1), (6, 11, 1)]


@pytest.mark.parametrize("kind,cost,causal", CUTS)
def test_every_step_is_done_once_and_parts_are_found(pieces, kind, cost, causal):
    """All blocks of a line, one after the other: every step of every tile has one block, a tile's blocks follow one another, the block that ends a
    tile and whoever looks a tile up know which blocks had it, and no block puts two partial states in one place."""
    rng = random.Random(100 * kind + 10 * cost + causal)
    for _ in range(1500):
        n = lines(kind, causal, rng)
        group, kv_heads = rng.choice([1, 2, 3, 4, 5, 8, 16, 100]), rng.choice([1, 2, 3, 8])
        for grid in (1, rng.randint(2, 160), 148):
            args = (ctypes.c_int * (3 * len(n)))(*[v for e in n for v in e])
            assert pieces.run_pieces(kind, causal, cost, group, kv_heads, len(n), args, grid) == 0, (kind, causal, cost, group, kv_heads, n, grid)
