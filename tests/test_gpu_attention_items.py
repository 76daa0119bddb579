"""The ring of items inside of an attention block: where its wait runs out, the warps that meet at a barrier leave at the same item."""
import ctypes
import os
import subprocess

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

RING = 4


@pytest.fixture(scope="module")
def ring(tmp_path_factory):
    from paper_2609_24802_b200 import build
    lib = str(tmp_path_factory.mktemp("ring") / "item_ring.so")
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "item_ring.cu")
    subprocess.run([build._nvcc()] + build.NVCC_FLAGS + ["-shared", src, "-o", lib], check=True, capture_output=True)
    f = ctypes.CDLL(lib).run_ring
    f.restype, f.argtypes = ctypes.c_int, [ctypes.c_int] * 3 + [ctypes.c_longlong, ctypes.c_void_p]
    return f


@pytest.mark.parametrize("slow", [0, 1])
@pytest.mark.parametrize("total,stop", [(0, 100), (1, 100), (3, 100), (40, 100), (40, 0), (40, 1), (40, 6), (40, 37)])
def test_warps_leave_together(ring, total, stop, slow):
    taken = torch.full((6,), -1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    assert ring(total, stop, slow, 1 << 24, taken.data_ptr()) == 0
    torch.cuda.synchronize()
    # a warp that does not return items lets RING more be handed out
    n = min(total, stop + RING)
    assert taken.tolist() == [n, n * (n - 1) // 2] * 2 + [min(total, stop), min(total, stop) * (min(total, stop) - 1) // 2]
