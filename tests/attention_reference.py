"""Attention, rotary positions and cache writes in 64 bits, and the tolerances that the storage type allows.

A rounding to the storage type is off by at most u = eps / 2 relative to the value.  The library forms scores, maxima, masses and
sums in fp32 and rounds
  - the weights p once before the product with the values, and the result once:   out, grad_value off by 2 u + u^2 of sum |p v|;
  - p (dP - delta) once, delta comes from the rounded out:                         grad_q, grad_key off by 3 u + 3 u^2 of
    scale sum p (sum_d |go v| + sum_d |go out|) |k|.
fp32 adds the error of a score, (D + 8) 2^-23 scale sum_d |q k| (products are exact, every addition is off by at most 2^-23 of the
largest partial sum), twice as a relative error of a weight (numerator and mass; three times for the gradients: p, lse and the
score), and n 2^-23 for a sum of n terms, taken over pieces of at most 128 keys and their pieces: n is at most 128 + n / 128."""
import math

import torch


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def tiny(dtype):
    """Half of the smallest subnormal step."""
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def attend(q, k, v, scale, seen, go=None):
    """One segment: q [n, h, D], k and v [m, hk, D], seen [n, m] bool.  fp64 results, normalisers and tolerances."""
    dt, (n, h, D), (m, hk, _) = q.dtype, q.shape, k.shape
    u = half_step(dt)
    q, k, v = q.double(), k.double(), v.double()
    read = seen.any(0)
    k, v = torch.where(read[:, None, None], k, 0.0), torch.where(read[:, None, None], v, 0.0)     # unread keys may hold anything
    kk, vv = (t.repeat_interleave(h // hk, 1) for t in (k, v))
    s = torch.einsum("nhd,mhd->hnm", q, kk) * scale
    size = torch.einsum("nhd,mhd->hnm", q.abs(), kk.abs()) * abs(scale)
    s = s.masked_fill(~seen[None], -math.inf)
    lse = torch.logsumexp(s, -1) if m else torch.full((h, n), -math.inf, dtype=torch.float64, device=q.device)
    p = torch.exp(s - torch.where(torch.isinf(lse), 0.0, lse)[..., None])
    off = (D + 8) * 2.0 ** -23 * (size.masked_fill(~seen[None], 0.0).amax(-1) if m else torch.zeros_like(lse)) + (128 + m / 128) * 2.0 ** -23   # [h, n]
    out = torch.einsum("hnm,mhd->nhd", p, vv)
    A = torch.einsum("hnm,mhd->nhd", p, vv.abs())
    r = {"out": out, "lse": lse.T, "out_tol": (2 * u + u * u + 2 * off.T[..., None]) * A + tiny(dt),
         "lse_tol": 2 * off.T + 2.0 ** -22 * lse.T.abs().nan_to_num(posinf=0.0) + 2.0 ** -22}
    if go is None:
        return r
    go = go.double()
    dp = torch.einsum("nhd,mhd->hnm", go, vv)
    dp_size = torch.einsum("nhd,mhd->hnm", go.abs(), vv.abs()) + (go * out).abs().sum(-1).T[..., None]
    ds = p * (dp - (go * out).sum(-1).T[..., None]) * scale
    ds_size = p * dp_size * abs(scale)
    # fp16: dS is scaled by a power of two that puts the largest possible value above 2^13, its smallest step is 2^-24
    floor = 2.0 ** -25 * 2.0 ** -13 * 2 * float(go.norm(dim=-1).max() if n else 0) * float(v.norm(dim=-1).max() if m else 0) * abs(scale) if dt == torch.float16 else 0.0
    grad = 3 * u + 3 * u * u + 3 * off
    fold = lambda t: t.reshape(m, hk, h // hk, D).sum(2)  # noqa: E731
    r["grad_q"] = torch.einsum("hnm,mhd->nhd", ds, kk)
    r["grad_q_tol"] = grad.T[..., None] * torch.einsum("hnm,mhd->nhd", ds_size, kk.abs()) + floor * torch.einsum("nm,mhd->nhd", seen.double(), kk.abs()) + tiny(dt)
    r["grad_key"] = fold(torch.einsum("hnm,nhd->mhd", ds, q))
    r["grad_key_tol"] = fold(torch.einsum("hnm,nhd->mhd", ds_size * grad[..., None], q.abs()) + floor * torch.einsum("nm,nhd->mhd", seen.double(), q.abs())) + tiny(dt)
    r["grad_value"] = fold(torch.einsum("hnm,nhd->mhd", p, go))
    r["grad_value_tol"] = fold(torch.einsum("hnm,nhd->mhd", p * (2 * u + u * u + 3 * off)[..., None], go.abs())) + n * h // hk * 2.0 ** -23 * fold(torch.einsum("hnm,nhd->mhd", p, go.abs())) + tiny(dt)
    if dt == torch.float16:
        r["grad_value_tol"] += fold(2.0 ** -40 * torch.einsum("nm,nhd->mhd", seen.double(), go.abs()))
    return r


def close(got, want, tol, what):
    got = got.double()
    assert got.shape == want.shape, what
    both = torch.isinf(want) & (got == want)
    bad = ~both & ~((got - want).abs() <= tol)
    if bad.any():
        worst = ((got - want).abs() / tol)[bad].max()
        at = bad.nonzero()[0].tolist()
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst {float(worst):.3g} tolerances; first {at}: "
                             f"{float(got[tuple(at)])} for {float(want[tuple(at)])}")


def turn(x, positions, freq, magnitude, pairs, inverse=False):
    """Rotary positions in 64 bits of x [n, heads, D]."""
    x = x.double()
    t = positions.double()[:, None, None] * freq.double().to(x.device)
    c, s = magnitude * torch.cos(t), magnitude * torch.sin(t) * (-1 if inverse else 1)
    r = 2 * freq.numel()
    y = x.clone()
    i = torch.arange(freq.numel(), device=x.device)
    a, b = (2 * i, 2 * i + 1) if pairs else (i, i + r // 2)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    size = x.abs()
    size[..., a] = size[..., b] = abs(magnitude) * (x[..., a].abs() + x[..., b].abs())
    return y, size
