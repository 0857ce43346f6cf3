"""The bounds of window_bounds hold what the kernels do and no less: kernels emulated in 64 bits on the host, as they are and with parts of
their precision or some of their keys left out."""
import pytest
import torch

import window_bounds as wb
import window_reference as ref

DT = {"f16": torch.float16, "bf16": torch.bfloat16}


def _parts(x, dtype, n, lift=0):
    """x (64 bits, or fp32 values in 64 bits) as a sum of n 16-bit parts, in units of 2^-lift."""
    left, total = x * 2.0 ** lift, torch.zeros_like(x)
    for _ in range(n):
        part = left.float().to(dtype).double()
        total, left = total + part, left - part
    return total * 2.0 ** -lift


def _emulate(q, keys, vals, scale, dtype, query_parts, weight_parts, lift, lose=None):
    """One token: weights against the row's largest, summed whole, multiplied with V in parts; `lose`: keys that are left out."""
    g = q.shape[1] // keys.shape[1]
    out = torch.empty(q.shape, dtype=torch.float64)
    for h in range(q.shape[1]):
        qq = q[0, h].double() if query_parts == 0 else _parts(q[0, h].double(), dtype, query_parts)
        s = keys[:, h // g].double() @ qq * scale
        w = torch.exp(s - s.max())
        if lose is not None:
            w[lose] = 0
        out[0, h] = _parts(w, dtype, weight_parts, lift) @ vals[:, h // g].double() / w.sum()
    return out.to(dtype)


def _worst(got, x, tol):
    return ((got.double() - x["out"]).abs() / tol).max().item()


def _random(dtype, n, hk, g, d, seed=1):
    gen = torch.Generator().manual_seed(seed)
    rnd = lambda *shape: torch.randn(*shape, generator=gen)
    return rnd(1, hk * g, d), rnd(n, hk, d).to(dtype), rnd(n, hk, d).to(dtype)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,d", [(28, 64), (290, 128), (600, 64), (5004, 128)])
def test_single_tokens_need_both_parts_of_weights_and_queries(dtype, n, d):
    dt = DT[dtype]
    lift = wb.LIFT_STEP if dt == torch.float16 else 0
    k, v = (wb.repeated(y, n) for y in _random(dt, 8, 2, 4, d)[1:])
    for hot, dropped in ((0.2, (2, 1)), (1.0, (1, 2))):     # (with small logits the weights' rounding is what is left)
        q = _random(dt, 8, 2, 4, d)[0] * hot                # an fp32 query, as the preparation leaves it
        x = wb.attend(q, [n - 1], k, v, n, 0)
        tol = wb.step_tolerance(x, dt)
        assert _worst(_emulate(q, k, v, d ** -0.5, dt, 2, 2, lift), x, tol) <= 1
        assert _worst(_emulate(q, k, v, d ** -0.5, dt, *dropped, lift), x, tol) > 1.2, dropped
        assert _worst(_emulate(q, k, v, d ** -0.5, dt, 0, 1, lift), x, wb.prompt_tolerance(x, dt)) <= 1      # (prompts: queries as they come)


@pytest.mark.parametrize("lead", [17.6, 20.0])
def test_fp16_weights_beside_a_sink_need_the_factor(lead):
    dt, n, d = torch.float16, 4096, 64
    gen = torch.Generator().manual_seed(2)
    q, k, v = torch.zeros(1, 1, d), torch.zeros(n, 1, d, dtype=dt), (torch.rand(n, 1, d, generator=gen) * 1000 + 500).to(dt)
    q[..., 5], k[0, 0, 5], v[0] = 4.0, lead / 4, 0
    x = wb.attend(q, [n - 1], k, v, n, 0, 1.0)
    tol = wb.step_tolerance(x, dt)
    assert _worst(_emulate(q, k, v, 1.0, dt, 0, 2, wb.LIFT_STEP), x, tol) <= 1
    assert _worst(_emulate(q, k, v, 1.0, dt, 0, 2, 0), x, tol) > 10


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,d", [(2000, 64), (5004, 128), (9003, 128), (20000, 64)])
def test_lost_keys_of_a_long_axis_show(dtype, n, d):
    """Values that name their block of 16 keys: four lost keys, a block or a tile of keys are far outside of the bounds of either kernel."""
    dt = DT[dtype]
    q, k, _ = _random(dt, n, 1, 2, d)
    q = q.to(dt)
    v = wb.marks(n, 1, d, dt)
    x = wb.attend(q, [n - 1], k, v, n, 0)
    step, prompt = wb.step_tolerance(x, dt), wb.prompt_tolerance(x, dt)
    lift = wb.LIFT_PROMPT if dt == torch.float16 else 0
    assert _worst(_emulate(q, k, v, d ** -0.5, dt, 0, 2, lift), x, step) <= 1
    assert _worst(_emulate(q, k, v, d ** -0.5, dt, 0, 1, lift), x, prompt) <= 1
    for lose in (slice(n - 4, n), slice(16 * 7, 16 * 8), slice(64 * 11, 64 * 12), slice(n // 2, n // 2 + 70)):
        got = _emulate(q, k, v, d ** -0.5, dt, 0, 2, lift, lose)
        assert _worst(got, x, step) > 1.5 and _worst(got, x, prompt) > 1.5, lose
