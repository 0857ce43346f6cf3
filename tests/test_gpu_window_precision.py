"""Precision of the window attention on the GPU, held to bounds that follow the weights (window_bounds)."""
import ctypes as C

import pytest
import torch

import window_bounds as wb
import window_reference as ref

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _sh():
    from paper_2305_17118_b200 import binding as sh
    return sh


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.fixture(autouse=True)
def _no_wait_gave_up():
    yield
    _sh().window_status()


def _step(sh, q, k, v, lengths, kc, vc, window, sinks, scale, work):
    """window_decode with or without a workspace."""
    if work:
        return sh.window_decode(q, k, v, lengths, kc, vc, window=window, sinks=sinks, scale=scale)
    out = torch.zeros_like(q)
    win = sh._Window(sh._CODE_OF[q.dtype], q.shape[2], q.shape[1], k.shape[1], window, sinks, scale)
    rows = lambda x: C.byref(sh._Rows(x.data_ptr(), x.stride(0), x.stride(1)))
    cache = sh._WindowCache(kc.data_ptr(), vc.data_ptr(), *kc.stride()[:3])
    assert sh.lib.sh_window_decode(C.byref(win), q.shape[0], rows(q), rows(k), rows(v), lengths.data_ptr(), C.byref(cache), None, None, 0,
                                   rows(out), None, 0, torch.cuda.current_stream().cuda_stream) == sh.SH_OK
    return out


def _sink(dtype, n, hk, g, d, axis, lead):
    """n caches of `axis` rows whose first key, a sink with a value of zero, is ahead of all others by `lead`: what comes out is the
    small weights' share."""
    gen = torch.Generator(device="cuda").manual_seed(61)
    kc = torch.zeros(n, hk, axis, d, dtype=dtype, device="cuda")
    vc = (torch.rand(n, hk, axis, d, generator=gen, device="cuda") * 1000 + 500).to(dtype)
    q = torch.zeros(n, hk * g, d, dtype=dtype, device="cuda")
    q[:, :, 5] = 4.0
    kc[:, :, 0, 5] = lead / 4.0
    vc[:, :, 0] = 0
    return q, torch.zeros(n, hk, d, dtype=dtype, device="cuda"), vc[:, :, 7].clone(), kc, vc


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lead", [10.0, 17.6, 20.0])
@pytest.mark.parametrize("n,hk,g,axis,work", [(60, 8, 1, 4096, True), (1, 1, 3, 65536, True), (1, 1, 3, 65536, False)])
def test_small_weights_beside_a_sink_in_single_tokens(dtype, lead, n, hk, g, axis, work):
    """Units whose rows one CTA walks over, a workspace's parts, a cluster."""
    sh, dt, d = _sh(), DT[dtype], 64
    q, k, v, kc, vc = _sink(dt, n, hk, g, d, axis, lead)
    t = axis - 1                                                     # the new token takes the last slot
    got = _step(sh, q, k, v, _i32([t] * n), kc, vc, axis - 1, 1, 1.0, work)
    for i in (0, n - 1):
        x = wb.attend(q[i:i + 1], [t], kc[i].transpose(0, 1), vc[i].transpose(0, 1), axis - 1, 1, 1.0)
        ref.check(got[i:i + 1], x["out"], wb.step_tolerance(x, dt), f"unit {i}")


def _cache(rows, held, window, sinks):
    """[1, hk, sinks + window, d] with the rows [n, hk, d] of the first `held` positions in their slots; NaN where nothing is."""
    slots = ref.slots_ref(held, window, sinks)
    c = torch.full((1, rows.shape[1], sinks + window, rows.shape[2]), float("nan"), dtype=rows.dtype, device="cuda")
    at = [torch.tensor(list(x), dtype=torch.int64, device="cuda") for x in (slots.keys(), slots.values())]
    c[0, :, at[0]] = rows[at[1]].transpose(0, 1)
    return c


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("hot", [0.2, 1.0])
@pytest.mark.parametrize("n,d,work", [(28, 64, True), (290, 128, True), (600, 64, True), (5004, 128, True), (5004, 128, False)])
def test_single_tokens_keep_both_parts_of_weights_and_queries(dtype, hot, n, d, work):
    """Prepared queries over few distinct keys, which all of a kind weigh the same: a part of the weights or of the query that is missing
    would show (tests/test_window_bounds.py says how far)."""
    sh, dt = _sh(), DT[dtype]
    gen = torch.Generator(device="cuda").manual_seed(62)
    rnd = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    hk, g = 2, 4
    keys, vals = (wb.repeated(rnd(8, hk, d).to(dt), n) for _ in range(2))
    kc, vc = _cache(keys, n - 1, n, 0), _cache(vals, n - 1, n, 0)
    q, k, v = rnd(1, hk * g, d).to(dt), rnd(1, hk, d).to(dt), rnd(1, hk, d).to(dt)
    inv = (10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).float().cuda()
    weight = ((1 + 0.3 * rnd(d)) * hot).to(dt)
    if work:
        r = sh.Rope(inv, q_weight=weight, k_weight=weight)
        out = sh.window_decode(q, k, v, _i32([n - 1]), kc, vc, window=n, rope=r)
        want_q, mag = ref.rope_ref(q, weight, _i32([n - 1]), inv, r.eps, r.sections, False, False)
    else:                                                            # (a query that comes as it is)
        out = _step(sh, q, k, v, _i32([n - 1]), kc, vc, n, 0, d ** -0.5, False)
        want_q, mag = q.double().cpu(), torch.zeros(q.shape, dtype=torch.float64)
    keys, vals = torch.cat([keys[:n - 1], kc[:, :, n - 1]]).cpu(), torch.cat([vals[:n - 1], v]).cpu()
    x = wb.attend(want_q, [n - 1], keys, vals, n, 0)
    # the preparation in fp32: 32 half-steps of |a| + |b| (rope_tolerance), through the product with the key
    prepared = 32 * ref.U32 * wb.attend(mag, [n - 1], keys, vals, n, 0)["logit"]
    ref.check(out, x["out"], wb.step_tolerance(x, dt) + prepared * (x["mass"] + x["out"].abs()))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("hk,g,d,window,sinks,held,work", [
    (2, 4, 128, 5000, 4, 20011, True), (2, 4, 128, 5000, 4, 20011, False), (1, 11, 128, 9000, 3, 9100, True), (3, 2, 64, 20000, 0, 19999, True),
    (3, 2, 64, 20000, 0, 19999, False), (1, 1, 64, 2000, 1, 7000, True)])
def test_every_key_block_of_a_long_axis_counts_once_in_single_tokens(dtype, hk, g, d, window, sinks, held, work):
    """Values that name their block of 16 keys, over an axis that is dealt out: a block that is lost or counted twice is far outside."""
    sh, dt = _sh(), DT[dtype]
    gen = torch.Generator(device="cuda").manual_seed(63)
    rnd = lambda *shape: torch.randn(*shape, generator=gen, device="cuda").to(dt)
    keys, vals = rnd(held + 1, hk, d), wb.marks(held + 1, hk, d, dt, "cuda")
    kc, vc, q = _cache(keys, held, window, sinks), _cache(vals, held, window, sinks), rnd(1, hk * g, d)
    out = _step(sh, q, keys[held:], vals[held:], _i32([held]), kc, vc, window, sinks, d ** -0.5, work)
    x = wb.attend(q, [held], keys, vals, window, sinks)
    ref.check(out, x["out"], wb.step_tolerance(x, dt))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("hk,g,d,window,sinks,n,held", [
    (1, 4, 128, 2000, 4, 40, 2500), (1, 4, 64, 5000, 0, 140, 4000), (2, 3, 128, 1200, 0, 70, 5000), (1, 71, 64, 1500, 130, 3, 1630),
    (8, 4, 128, 20000, 0, 64, 15000), (1, 2, 128, 9000, 1, 2, 9500), (1, 8, 64, 3000, 4, 1500, 0), (8, 4, 128, 1000, 2, 1200, 3100)])
def test_every_key_block_counts_once_in_prompts(dtype, hk, g, d, window, sinks, n, held):
    """The same for chunks over a long context (dealt out to several CTAs and merged, but for the last) and for one that looks at itself."""
    sh, dt = _sh(), DT[dtype]
    gen = torch.Generator(device="cuda").manual_seed(64)
    rnd = lambda *shape: torch.randn(*shape, generator=gen, device="cuda").to(dt)
    keys, vals, q = rnd(held + n, hk, d), wb.marks(held + n, hk, d, dt, "cuda"), rnd(n, hk * g, d)
    kc, vc = _cache(keys, held, window, sinks), _cache(vals, held, window, sinks)
    win = sh._Window(sh._CODE_OF[dt], d, hk * g, hk, window, sinks, 0.0)
    if dt != torch.float32:
        assert (sh.lib.sh_window_prefill_workspace_bytes(C.byref(win), n, 1, 1) > 0) == (n != 1200)
    out = sh.window_prefill(q, keys[held:], vals[held:], _i32([0, n]), window=window, sinks=sinks, lengths=_i32([held]), k_cache=kc, v_cache=vc)
    x = wb.attend(q, range(held, held + n), keys, vals, window, sinks)
    ref.check(out, x["out"], wb.prompt_tolerance(x, dt))
