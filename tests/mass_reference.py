"""Plain 64-bit definitions of attention over shared contexts and of the cache with accumulated weights, with what the bounds need.

A row's result is ``out = sum_j p_j v_j`` with ``p = softmax(scale q.k)`` over the rows it sees and, where it continues from a prior
``(out0, lse0)``, over those and one more of logit ``lse0`` and value ``out0``.  Where a kernel is off:

* outputs: as window_bounds says (one rounding of the result; logits; weights rounded to ``parts`` 16-bit parts; sums in fp32);
* ``lse``: the logits' error, the sum's relative error, and four fp32 roundings of the log itself (2^-24 of it each, base 2 and back);
* a mass: each weight is off by twice the logits' error, the sum's and the log's (they follow from ``lse``), 2^-21 of the exponential; weights
  are added up one by one in fp32, 2^-24 of their sum for each (and 2^-24 of the mass for the last addition).
"""
import torch

import window_reference as ref


def attend(q, keys, vals, sees, scale=None, prior=None):
    """q [t, hq, d], keys and vals [m, hk, d], sees [t, m] bool (on the CPU, in 64 bits) -> dict; weights [t, hq, m] among it."""
    q, keys, vals = q.double().cpu(), keys.double().cpu(), vals.double().cpu()
    t, hq, d = q.shape
    m, g = keys.shape[0], hq // keys.shape[1]
    scale = d ** -0.5 if scale is None else scale
    keys, vals = keys.repeat_interleave(g, 1), vals.repeat_interleave(g, 1)
    s = torch.full((t, hq, m), float("-inf"), dtype=torch.float64)
    size = torch.zeros(t, hq, 1, dtype=torch.float64)
    for h in range(hq):
        for i in range(t):                                       # rows out of sight do not enter, whatever they hold
            see = sees[i]
            s[i, h, see] = keys[see, h] @ q[i, h] * scale
            if see.any():
                size[i, h] = (keys[see, h].abs() @ q[i, h].abs()).max() * scale
    all_s = s if prior is None else torch.cat([s, prior[1].double().cpu()[..., None]], -1)
    lse = torch.logsumexp(all_s, -1)
    p = torch.where(torch.isinf(lse)[..., None], torch.zeros_like(s), torch.exp(s - lse[..., None]))
    clean = torch.where(sees.any(0)[:, None, None], vals, torch.zeros_like(vals))
    out, mass = torch.einsum("thm,mhd->thd", p, clean), torch.einsum("thm,mhd->thd", p, clean.abs())
    if prior is not None:
        w = torch.exp(prior[1].double().cpu() - lse)[..., None]
        w = torch.where(torch.isnan(w), torch.zeros_like(w), w)
        part = torch.where(w > 0, w * prior[0].double().cpu(), torch.zeros_like(out))
        out, mass = out + part, mass + part.abs()
    return dict(out=out, lse=lse, p=p, mass=mass, total=torch.einsum("tm,mhd->thd", sees.double(), clean.abs()), logit=size,
                top=p.amax(-1, keepdim=True), keys=int(sees.sum(1).max()) if m else 0, d=d)


def logit_error(x, dtype):
    half = ref.half_step(dtype)
    return ((x["d"] + 8) * 2.0 ** -23 + (half ** 2 if dtype != torch.float32 else 0.0)) * x["logit"] + 2.0 ** -21


def chain(x):
    return (x["keys"] / 16 + 64) * 2.0 ** -23


def out_tolerance(x, dtype, parts, lift, out_dtype=None):
    half = ref.half_step(dtype)
    tol = ref.rounding(x["out"], out_dtype or dtype) + (logit_error(x, dtype) + chain(x)) * (x["mass"] + x["out"].abs())
    if dtype != torch.float32:
        tol = tol + half ** parts * x["mass"]
    if dtype == torch.float16:
        tol = tol + 2.0 ** -(25 + lift) * x["top"] * x["total"] + 2.0 ** -24
    return tol


def lse_tolerance(x, dtype):
    return logit_error(x, dtype)[..., 0] + chain(x) + 4 * 2.0 ** -24 * x["lse"].abs()


def weight_tolerance(x, dtype):
    """[t, hq, m]: of each weight."""
    rel = 2 * logit_error(x, dtype)[..., 0] + chain(x) + 8 * 2.0 ** -24 * x["lse"].abs() + 2.0 ** -21
    return x["p"] * rel[..., None] + 2.0 ** -126


def mass_of(x, g):
    """[m, hk]: what rows receive from all tokens and heads of the group."""
    t, hq, m = x["p"].shape
    return x["p"].view(t, hq // g, g, m).sum((0, 2)).T


def mass_tolerance(x, g, dtype, before):
    """[m, hk]; before: masses that grow."""
    w = weight_tolerance(x, dtype)
    t, hq, m = w.shape
    total = mass_of(x, g)
    return w.view(t, hq // g, g, m).sum((0, 2)).T + (t * g + 8) * 2.0 ** -24 * total + 2.0 ** -24 * (before.double().cpu() + total)


def evict(mass, positions, keep, recent):
    """One unit's live records -> (slots that stay, holes below keep, rows that move into them), lists of ints."""
    n = len(mass)
    if n <= keep:
        return list(range(n)), [], []
    newest = max(positions)
    nan = [m != m for m in mass]

    def place(j):
        if positions[j] > newest - recent:
            return (0, 0.0, j)
        return (1, 0.0, j) if nan[j] else (2, -mass[j], j)

    stay = sorted(sorted(range(n), key=place)[:keep])
    return stay, [j for j in range(keep) if j not in set(stay)], [j for j in stay if j >= keep]
