"""Window attention in 64 bits with what an error bound needs, and bounds that follow the weights instead of the largest value.

``out = sum_j p_j v_j`` with the softmax weights ``p``.  Where a kernel is off:

* the result is rounded once;
* a logit that is off by ``e`` moves its weight by ``e`` of itself, numerator and denominator alike: together at most
  ``e * sum p |v - out| <= e * (mass + |out|)`` with ``mass = sum p |v|``.  A logit is a sum of d products in fp32 (each step off by at most
  2^-23 of the sum of magnitudes so far, as the tensor cores may cut instead of round; d + 8 steps with the scale and the subtraction) and
  an exponential (2^-21 with its argument's rounding).  A query that is held as two 16-bit parts is off by a half-step squared;
* a weight that enters the product with V rounded to ``parts`` 16-bit parts is off by half_step^parts of itself, while the sum of weights
  takes it whole: half_step^parts * mass.  fp16 parts of small weights are multiples of 2^-24: off by 2^-25 in units of the lifted weights,
  2^-(25 + lift) of the largest weight for each key;
* products and weights are summed in fp32, a step for every 16 keys and 64 to merge: 2^-23 of the mass (and of the result) a step.
"""
import torch

import window_reference as ref

LIFT_STEP, LIFT_PROMPT = 15, 7      # log2 factors of fp16 weights


def attend(q, qpos, keys, vals, window, sinks, scale=None, at=None):
    """q [t, hq, d] at positions qpos, keys and vals [n, hk, d] at positions `at` (default: their rows) -> dict of 64-bit tensors [t, hq, .]."""
    t, hq, d = q.shape
    g = hq // keys.shape[1]
    scale = d ** -0.5 if scale is None else scale
    pos = torch.arange(keys.shape[0], device=q.device) if at is None else at
    see = ref.visible(torch.as_tensor(list(qpos), device=q.device)[:, None], pos[None], window, sinks)
    x = {name: torch.empty(t, hq, d, dtype=torch.float64, device=q.device) for name in ("out", "mass", "total")}
    x.update({name: torch.empty(t, hq, 1, dtype=torch.float64, device=q.device) for name in ("logit", "top")})
    for h in range(hq):
        qq, k, v = q[:, h].double(), keys[:, h // g].double(), vals[:, h // g].double()
        p = torch.softmax((qq @ k.T * scale).masked_fill(~see, float("-inf")), 1)
        x["out"][:, h], x["mass"][:, h], x["total"][:, h] = p @ v, p @ v.abs(), see.double() @ v.abs()
        x["logit"][:, h] = ((qq.abs() @ k.abs().T) * scale).masked_fill(~see, 0).amax(1, keepdim=True)
        x["top"][:, h] = p.amax(1, keepdim=True)
    x["keys"] = int(see.sum(1).max())
    return {name: y.cpu() if isinstance(y, torch.Tensor) else y for name, y in x.items()}


def tolerance(x, dtype, parts, lift):
    d, half = x["out"].shape[2], ref.half_step(dtype)
    sixteen = dtype != torch.float32
    e = ((d + 8) * 2.0 ** -23 + (half ** 2 if sixteen else 0.0)) * x["logit"] + 2.0 ** -21
    chain = (x["keys"] / 16 + 64) * 2.0 ** -23
    tol = ref.rounding(x["out"], dtype) + (e + chain) * (x["mass"] + x["out"].abs())
    if sixteen:
        tol = tol + half ** parts * x["mass"]
    if dtype == torch.float16:
        tol = tol + 2.0 ** -(25 + lift) * x["top"] * x["total"]
    return tol


def step_tolerance(x, dtype):
    """Single tokens: weights in two parts."""
    return tolerance(x, dtype, 2, LIFT_STEP)


def prompt_tolerance(x, dtype):
    """Prompts: weights rounded once."""
    return tolerance(x, dtype, 1, LIFT_PROMPT)


def marks(n, heads, d, dtype, device="cpu"):
    """Values [n, heads, d] that name their block of 16 keys: 1 in column (block mod d), 0 elsewhere.  What comes out is each block's share."""
    v = torch.zeros(n, heads, d, dtype=dtype, device=device)
    j = torch.arange(n, device=device)
    v[j, :, j // 16 % d] = 1
    return v


def repeated(rows, n):
    """n rows that take the given ones in turn: keys that weigh the same are rounded the same way, so that errors of weights add up instead of
    evening out over a long axis."""
    return rows[torch.arange(n, device=rows.device) % rows.shape[0]]
