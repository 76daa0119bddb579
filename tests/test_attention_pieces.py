"""How attention deals out its work to blocks, on the host."""
import ctypes
import os
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
