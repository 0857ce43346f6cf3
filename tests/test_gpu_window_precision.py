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
