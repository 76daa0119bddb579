"""GPU parity of rotary positions against 64 bits.  An element is a cos - b sin in fp32: sine and cosine are off by at most 2^-22
(the reduced angle is rounded to fp32 once, sincospif is good to 2 units), the sum adds two roundings, the result is rounded to its
type once: (u + 2^-21) magnitude (|a| + |b|)."""
import pytest

from attention_reference import close, half_step, tiny, turn

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def tiga():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_24802_b200 import api
    return api


def normal(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


def check(tiga, x, pos, turned, pairs, inverse=False, scaling=0, out=None):
    freq, m = tiga.tiga_rotary_frequencies(turned, scaling=scaling, factor=8.0, length=4096.0)
    rot = tiga.Rotary(freq.cuda(), pairs=pairs, magnitude=m)
    want, size = turn(x, pos, freq, m, pairs, inverse)
    tail = x[..., turned:].clone()
    got = tiga.tiga_apply_rotary(rot, x, pos, out=out, inverse=inverse)
    tol = (half_step(x.dtype) + 2.0 ** -21) * size + tiny(x.dtype)
    close(got[..., :turned], want[..., :turned], tol[..., :turned], "turned")
    assert torch.equal(got[..., turned:], tail)
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("n,heads,D,turned", [(1, 1, 2, 2), (33, 8, 80, 32), (5, 3, 7, 6), (100, 5, 128, 128), (3, 40, 64, 36), (257, 2, 96, 48), (1, 128, 256, 256), (9, 1, 24, 8)])
def test_layouts(tiga, n, heads, D, turned, pairs, dtype):
    pos = torch.randint(0, 5000, (n,), generator=torch.Generator().manual_seed(n)).cuda().to(torch.int32 if n % 2 else torch.int64)
    x = normal((n, heads, D), dtype, n + D)
    y = check(tiga, x, pos, turned, pairs)
    check(tiga, y, pos, turned, pairs, inverse=True)


@pytest.mark.parametrize("scaling", [0, 1, 2, 3])
def test_far_positions_and_scalings(tiga, scaling):
    pos = torch.tensor([0, 1, -1, 4095, 1 << 20, (1 << 31) - 1, -(1 << 31), 1 << 40], device="cuda")
    # 2^40 turns keep 52 - 40 bits of fraction times the frequency's own rounding, in the reference as well: left out of fp32 bounds
    check(tiga, normal((7, 4, 128), torch.float32, 1), pos[:5].repeat(2)[:7], 128, False, scaling=scaling)
    check(tiga, normal((7, 4, 128), torch.bfloat16, 1), pos[:7], 128, True, scaling=scaling)


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_and_in_place(tiga, dtype):
    x = normal((50, 12, 64), dtype, 2)
    pos = torch.arange(50, device="cuda")
    check(tiga, x[:, 3:7], pos, 64, False)
    wide = normal((50, 4, 67), dtype, 3)
    check(tiga, wide[..., 1:65], pos, 64, True)             # rows that start on odd elements
    for pairs in (False, True):
        y = x.clone()[:, 2:9]
        assert check(tiga, y, pos, 32, pairs, out=y) is y
    z = normal((4, 50, 64), dtype, 4).transpose(0, 1)       # heads in front
    check(tiga, z, pos, 64, False, out=torch.empty_like(z))


def test_inverse_is_the_gradient(tiga):
    """<turn(x), g> = <x, inverse(g)>, and differences of it."""
    freq, m = tiga.tiga_rotary_frequencies(48, scaling=tiga.ROT_BANDS, factor=4.0, length=512.0)
    for pairs in (False, True):
        rot = tiga.Rotary(freq.cuda(), pairs=pairs, magnitude=m)
        x, g, pos = normal((40, 3, 64), torch.float32, 5), normal((40, 3, 64), torch.float32, 6), torch.arange(1000, 1040, device="cuda")
        a = (tiga.tiga_apply_rotary(rot, x, pos).double() * g).sum()
        b = (tiga.tiga_apply_rotary(rot, g, pos, inverse=True).double() * x).sum()
        size = 2 * m * (x.abs().double() * g.abs()).sum() * 2
        assert abs(float(a - b)) <= 2.0 ** -21 * float(size)


def test_nothing_behind_the_rows_is_written(tiga):
    freq, m = tiga.tiga_rotary_frequencies(64)
    rot = tiga.Rotary(freq.cuda())
    out = torch.full((20, 3, 72), 7.0, device="cuda", dtype=torch.float16)
    tiga.tiga_apply_rotary(rot, normal((10, 2, 64), torch.float16, 7), torch.arange(10, device="cuda"), out=out[5:15, :2, :64])
    assert torch.all(out[:5] == 7) and torch.all(out[15:] == 7) and torch.all(out[:, 2] == 7) and torch.all(out[..., 64:] == 7) and not torch.any(out[5:15, :2, :64] == 7)
    assert tiga.tiga_apply_rotary(rot, normal((0, 2, 64), torch.float16, 7), torch.arange(0, device="cuda")).shape == (0, 2, 64)
