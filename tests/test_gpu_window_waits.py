"""The give-up path of the prompt kernel's bounded waits, in the bounds-checked build of the library: its waits last 0.2 seconds, and
sh_window_selftest makes the CTA of one work item give up (on the host's order, with nothing in flight; no other fault)."""
import ctypes as C

import pytest
import torch

import window_reference as ref

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture()
def shb(monkeypatch):
    """The binding with the bounds-checked library in place of the normal one."""
    import gc
    from paper_2305_17118_b200 import binding, build
    gc.collect()
    dbg = binding.declare(C.CDLL(build.build(debug_bounds=True)))
    dbg.sh_window_selftest.argtypes = [C.c_int]
    monkeypatch.setattr(binding, "lib", dbg)
    yield binding
    dbg.sh_window_selftest(-1)
    gc.collect()


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _prefill(sh, q, k, v, starts, lengths, kc, vc, window, out, work):
    win = sh._Window(sh._CODE_OF[q.dtype], q.shape[2], q.shape[1], k.shape[1], window, 0, 0.0)
    rows = lambda x: C.byref(sh._Rows(x.data_ptr(), x.stride(0), x.stride(1)))
    cache = sh._WindowCache(kc.data_ptr(), vc.data_ptr(), *kc.stride()[:3])
    return sh.lib.sh_window_prefill(C.byref(win), q.shape[0], len(starts) - 1, rows(q), rows(k), rows(v), starts.data_ptr(), lengths.data_ptr(),
                                    C.byref(cache), rows(out), work.data_ptr(), work.numel(), torch.cuda.current_stream().cuda_stream)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64)])
def test_a_lost_item_leaves_the_rows_of_others_alone(shb, dtype, d):
    """Few rows over many keys, dealt out and merged.  The CTA that should have listed the first key head's item gives up, so its entry
    in the workspace is whatever lay there: here rows behind the tensor's end, where the memory is this test's own.  The call is
    reported, nothing behind the end is written, the other heads come out as usual, and the next call is whole."""
    sh, dt = shb, DT[dtype]
    gen = torch.Generator(device="cuda").manual_seed(51)
    rnd = lambda *shape: torch.randn(*shape, generator=gen, device="cuda").to(dt)
    n, hk, g, window, ctx = 40, 4, 4, 4000, 4000
    q, k, v = rnd(n, hk * g, d), rnd(n, hk, d), rnd(n, hk, d)
    kc, vc = rnd(1, hk, window, d), rnd(1, hk, window, d)
    starts, lengths = _i32([0, n]), _i32([ctx])
    win = sh._Window(sh._CODE_OF[dt], d, hk * g, hk, window, 0, 0.0)
    need = sh.lib.sh_window_prefill_workspace_bytes(C.byref(win), n, 1, 1)
    assert need > 0
    memory = torch.full((20 * n, hk * g, d), 7.0, dtype=dt, device="cuda")
    out = memory[:n]
    whole = torch.empty_like(q)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    assert _prefill(sh, q, k, v, starts, lengths, kc, vc, window, whole, work) == sh.SH_OK
    sh.window_status()
    for entry in ([3, 2 * n, n, 0], [3, n - 1, 16 * n, 0], [1 << 30, (1 << 30) + 5, 1 << 30, 0], [4, -n, n, 0]):
        memory.fill_(7.0)
        work.view(torch.int32).view(-1, 4).copy_(_i32(entry).expand(need // 16, 4))
        assert sh.lib.sh_window_selftest(0) == sh.SH_OK
        assert _prefill(sh, q, k, v, starts, lengths, kc, vc, window, out, work) == sh.SH_OK
        with pytest.raises(sh.ShError) as e:
            sh.window_status()
        assert e.value.status == sh.SH_EDEVICE
        assert (memory[n:] == 7).all()
        assert torch.equal(out[:, g:], whole[:, g:])
        assert (out[:, :g] == 7).all()
        assert sh.lib.sh_window_selftest(-1) == sh.SH_OK
        assert _prefill(sh, q, k, v, starts, lengths, kc, vc, window, out, work) == sh.SH_OK
        sh.window_status()
        assert torch.equal(out, whole) and (memory[n:] == 7).all()


def test_rows_computed_again_do_not_run_out_the_waits(shb):
    """An infinite value that every row sees sends every row through the slow path: a warp's rows take longer than the waits of this
    build last, while the other warps wait for its next item.  All rows come out."""
    sh, dt, d, n = shb, torch.float16, 64, 160000
    gen = torch.Generator(device="cuda").manual_seed(52)
    q, k, v = (torch.randn(n, 1, d, generator=gen, device="cuda").to(dt) for _ in range(3))
    starts = _i32([0, n])
    clean = v.clone()
    v[0, 0, 3] = float("inf")
    out = sh.window_prefill(q, k, v, starts, window=1 << 20)
    sh.window_status()
    assert torch.isposinf(out[:, 0, 3]).all()
    assert torch.isfinite(out[:, 0, :3]).all() and torch.isfinite(out[:, 0, 4:]).all()
    clean[0, 0, 3] = 0
    for i in (0, 1, 255, 256, 70001, n - 257, n - 1):
        want, vmax, smax = ref.attend_ref(q[i:i + 1], [i], k[:i + 1], clean[:i + 1], 1 << 20, 0)
        got = out[i:i + 1].clone()
        got[0, 0, 3] = want[0, 0, 3]
        tol = ref.attend_tolerance(want, vmax, smax, dt)
        tol[0, 0, 3] = 1.0
        ref.check(got, want, tol)
