"""Plain 64-bit definitions of the query/key preparation and of window attention, and error bounds for the kernels.

Everything is written from the definitions, position by position, with full histories: nothing here knows about rings.
"""
import math

import torch

U32 = 2.0 ** -24          # half a step of fp32, relative


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def rounding(want, dtype):
    """One rounding of `want`: half a step relative to the value, and half of the fixed step below the smallest normal number (in fp16
    2^-14: the numbers below it are multiples of 2^-24, so a result there is off by up to 2^-25 however small it is)."""
    f = torch.finfo(dtype)
    return f.eps / 2 * want.abs() + f.smallest_normal * f.eps / 2


def rope_ref(x, weight, positions, inv_freq, eps, sections, spread, adjacent):
    """x [t, h, d] -> (result in 64 bits, bound on |a| + |b| of the pair each element comes from, before rotation)."""
    y = x.double().cpu()
    if weight is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * weight.double().cpu()
    f = inv_freq.double().cpu()
    pos = positions.double().cpu()
    pos = pos if pos.dim() == 2 else pos[None]
    out, mag = y.clone(), y.abs()
    n = len(f)
    for i in range(n):
        if spread:
            ax = i % 3 if i < 3 * sections[i % 3] else 0
        else:
            ax = next(a for a in range(len(sections)) if i < sum(sections[: a + 1]))
        ang = pos[ax] * f[i]
        c, s = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
        a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + n)
        out[..., a] = y[..., a] * c - y[..., b] * s
        out[..., b] = y[..., a] * s + y[..., b] * c
        mag[..., a] = mag[..., b] = y[..., a].abs() + y[..., b].abs()
    return out, mag


def rope_tolerance(want, mag, dtype):
    """Half a step of the result, and 32 fp32 half-steps of |a| + |b|: at most 20 roundings in the sum of squares (16 in the
    lane's chain, 3 across lanes, the division by d), halved by the root, + root, division, two products (14); the angle's
    fraction of a turn is rounded once (2 pi / 2 half-steps of a radian, 4), sine and cosine are within 2 steps (4), and the
    two products and their sum round three times; the double reduction adds less than 1e-7 radians at positions below 2^20
    and 6e-7 = 10 half-steps at 2^30."""
    return rounding(want, dtype) + 32 * U32 * mag


def visible(qpos, kpos, window, sinks):
    return (kpos <= qpos) & ((kpos < sinks) | (kpos > qpos - window))


def attend_ref(q, qpos, keys, vals, window, sinks, scale=None):
    """q [t, hq, d] at positions qpos over the full history keys, vals [n, hk, d] (position = row) -> ([t, hq, d], tolerance parts).
    Rows that a query does not see are left out before anything is computed with them."""
    t, hq, d = q.shape
    g = hq // keys.shape[1]
    scale = d ** -0.5 if scale is None else scale
    out = torch.zeros(t, hq, d, dtype=torch.float64)
    vmax = torch.zeros(t, hq, 1, dtype=torch.float64)
    smax = torch.zeros(t, hq, 1, dtype=torch.float64)
    kpos = torch.arange(keys.shape[0])
    q, keys, vals = q.double().cpu(), keys.double().cpu(), vals.double().cpu()
    for i in range(t):
        see = visible(int(qpos[i]), kpos, window, sinks)
        k, v = keys[see].repeat_interleave(g, 1), vals[see].repeat_interleave(g, 1)      # [m, hq, d]
        s = torch.einsum("hd,mhd->hm", q[i], k) * scale
        out[i] = torch.einsum("hm,mhd->hd", torch.softmax(s, 1), v)
        vmax[i, :, 0] = v.abs().amax((0, 2))
        smax[i, :, 0] = (q[i].abs()[None] * k.abs()).sum(-1).amax(0) * scale
    return out, vmax, smax


def attend_tolerance(out, vmax, smax, dtype):
    """The result is rounded once (half a step of it).  A weight of a 16-bit kernel is rounded to the type before the product with
    V: half a step of the largest |v|.  Each logit is a sum of up to 128 products in fp32 and an exponent: an error of e in it
    moves a weight by e of itself, numerator and denominator alike, so 2 * e * max|v|, with e below (128 + 8) * 2^-24 * sum |q||k|
    + 2^-17 * sum |q||k| for a query held as two 16-bit parts, + 8 * 2^-24 for the exponential; the sums of weights and of products
    add their own fp32 roundings, at most 64 in a chain."""
    e = (136 * U32 + (2.0 ** -17 if dtype != torch.float32 else 0.0)) * smax + 8 * U32
    p = half_step(dtype) if dtype != torch.float32 else 0.0
    return rounding(out, dtype) + (p + 2 * e + 2 * 64 * U32) * vmax


def slots_ref(history, window, sinks):
    """{slot: position} of the live slots after `history` tokens."""
    live = {}
    for pos in range(history):
        live[pos if pos < sinks else sinks + (pos - sinks) % window] = pos
    return live


def check(got, want, tol, what=""):
    got = got.double().cpu()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    bad = (got - want).abs() > tol
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {((got - want).abs() / tol).max():.2f} of the tolerance"
