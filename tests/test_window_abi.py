"""Host side of the query/key preparation and the window cache: the entry points' argument checks (no device call is made: every
call below is refused, or has nothing to do)."""
import copy
import ctypes as C

import pytest

FAKE = 1 << 20      # an aligned address that is never dereferenced


def _sh():
    from paper_2305_17118_b200 import binding as sh
    return sh


def _args(sh):
    rows = lambda heads: sh._Rows(FAKE, heads * 64, 64)
    return dict(w=sh._Window(sh.SH_F16, 64, 4, 2, 8, 2, 0.0), q=rows(4), k=rows(2), v=rows(2), out=rows(4), starts=FAKE, lengths=FAKE,
                cache=sh._WindowCache(FAKE, FAKE, 2 * 10 * 64, 10 * 64, 64), tokens=4, n=3, rope=None, positions=None, axis=0,
                work=None, work_bytes=0)


def _rope(sh, **kw):
    r = sh._Rope(sh.SH_F16, 64, 64, 1, (C.c_int * 3)(32, 0, 0), 0, 0, 1e-6, FAKE, None, None)
    for name, value in kw.items():
        setattr(r, name, (C.c_int * 3)(*value) if name == "sections" else value)
    return r


def _calls(sh, a):
    ref = lambda x: None if x is None else C.byref(x)
    lib = sh.lib
    return dict(
        prefill=lambda: lib.sh_window_prefill(ref(a["w"]), a["tokens"], a["n"], ref(a["q"]), ref(a["k"]), ref(a["v"]), a["starts"],
                                              a["lengths"], ref(a["cache"]), ref(a["out"]), a["work"], a["work_bytes"], None),
        append=lambda: lib.sh_window_append(ref(a["w"]), a["tokens"], a["n"], ref(a["k"]), ref(a["v"]), a["starts"], a["lengths"],
                                            ref(a["cache"]), None),
        decode=lambda: lib.sh_window_decode(ref(a["w"]), a["n"], ref(a["q"]), ref(a["k"]), ref(a["v"]), a["lengths"], ref(a["cache"]),
                                            ref(a["rope"]), a["positions"], a["axis"], ref(a["out"]), a["work"], a["work_bytes"], None))


ALL, CHUNK = ("prefill", "append", "decode"), ("prefill", "append")


@pytest.mark.parametrize("which,change", [
    (ALL, dict(w=None)), (ALL, dict(w__dtype=3)), (ALL, dict(w__dtype=-1)), (ALL, dict(w__head_dim=96)), (ALL, dict(w__window=0)),
    (ALL, dict(w__sinks=-1)), (ALL, dict(w__window=1 << 30)), (ALL, dict(w__q_heads=3)), (ALL, dict(w__kv_heads=0)),
    (ALL, dict(w__scale=-1.0)), (ALL, dict(w__scale=float("nan"))), (ALL, dict(w__scale=float("inf"))), (ALL, dict(n=-1)),
    (CHUNK, dict(tokens=-1)), (CHUNK, dict(tokens=1 << 30)), (CHUNK, dict(starts=None)), (CHUNK, dict(starts=FAKE + 2)),
    (ALL, dict(lengths=None)), (("append", "decode"), dict(cache=None)), (("prefill",), dict(cache=None)), (ALL, dict(k=None)),
    (("prefill", "decode"), dict(q=None)), (("prefill", "decode"), dict(out=None)), (ALL, dict(k__data=FAKE + 8)), (ALL, dict(v__data=None)),
    (ALL, dict(k__head_stride=0)), (ALL, dict(k__token_stride=68)), (ALL, dict(v__token_stride=-64)), (ALL, dict(v__token_stride=1 << 38)),
    (("prefill", "decode"), dict(out__token_stride=128)), (ALL, dict(cache__k=FAKE + 4)), (ALL, dict(cache__slot_stride=32)),
    (ALL, dict(cache__head_stride=64)), (ALL, dict(cache__sequence_stride=640)), (ALL, dict(cache__sequence_stride=0)),
    (("decode",), dict(positions=FAKE)),
])
def test_window_calls_refuse(which, change):
    sh = _sh()
    a = copy.copy(_args(sh))
    for name, value in change.items():
        if "__" in name:
            setattr(a[name.split("__")[0]], name.split("__")[1], value)
        else:
            a[name] = value
    calls = _calls(sh, a)
    for name in which:
        assert calls[name]() == sh.SH_EINVAL, name


@pytest.mark.parametrize("change", [
    dict(dtype=3), dict(head_dim=32), dict(rot_dim=8), dict(rot_dim=80), dict(rot_dim=-16), dict(axes=0), dict(axes=4),
    dict(sections=(31, 0, 0)), dict(axes=2, sections=(40, -8, 0)), dict(spread=1), dict(spread=2), dict(adjacent_pairs=2), dict(eps=-1.0),
    dict(eps=float("nan")), dict(eps=float("inf")), dict(inv_freq_dev=None), dict(inv_freq_dev=FAKE + 1), dict(q_weight_dev=FAKE + 8),
    dict(k_weight_dev=FAKE + 2),
])
def test_rope_calls_refuse(change):
    sh = _sh()
    a = _args(sh)
    r = _rope(sh, **change)
    q = C.byref(a["q"])
    assert sh.lib.sh_qk_norm_rope(C.byref(r), 4, 4, 0, q, None, FAKE, 0, q, None, None) == sh.SH_EINVAL
    a["rope"] = r
    assert _calls(sh, a)["decode"]() == sh.SH_EINVAL


def test_rope_calls_refuse_rows_and_positions():
    sh = _sh()
    a = _args(sh)
    r, q, k = _rope(sh), C.byref(a["q"]), C.byref(a["k"])
    call = sh.lib.sh_qk_norm_rope
    assert call(None, 4, 4, 0, q, None, FAKE, 0, q, None, None) == sh.SH_EINVAL
    assert call(C.byref(r), 4, 4, 2, q, k, FAKE, 0, q, None, None) == sh.SH_EINVAL        # k without k_out
    assert call(C.byref(r), 4, 4, 2, q, None, FAKE, 0, q, None, None) == sh.SH_EINVAL     # k heads without k
    assert call(C.byref(r), 4, 4, 0, q, k, FAKE, 0, q, k, None) == sh.SH_EINVAL
    assert call(C.byref(r), 4, 4, 0, q, None, None, 0, q, None, None) == sh.SH_EINVAL     # no positions
    assert call(C.byref(r), 4, 4, 0, q, None, FAKE + 1, 0, q, None, None) == sh.SH_EINVAL
    assert call(C.byref(r), -1, 4, 0, q, None, FAKE, 0, q, None, None) == sh.SH_EINVAL
    assert call(C.byref(r), 4, 0, 0, q, None, FAKE, 0, q, None, None) == sh.SH_EINVAL
    narrow = sh._Rows(FAKE, 128, 64)                                                      # tokens share elements
    assert call(C.byref(r), 4, 4, 0, q, None, FAKE, 0, C.byref(narrow), None, None) == sh.SH_EINVAL
    three = _rope(sh, axes=3, sections=(16, 8, 8))
    assert call(C.byref(three), 4, 4, 0, q, None, FAKE, -4, q, None, None) == sh.SH_EINVAL
    a["rope"] = three                                                                     # several axes need positions
    assert _calls(sh, a)["decode"]() == sh.SH_EINVAL
    a["rope"] = _rope(sh, dtype=sh.SH_BF16)                                               # another type than the cache's
    assert _calls(sh, a)["decode"]() == sh.SH_EINVAL


def test_decode_workspace():
    sh = _sh()
    a = _args(sh)
    size = sh.lib.sh_window_decode_workspace_bytes
    need = size(C.byref(a["w"]), 3)
    assert 0 < need < 1 << 21
    a["work"], a["work_bytes"] = FAKE, need - 1
    assert _calls(sh, a)["decode"]() == sh.SH_ENOMEM
    a["work"], a["work_bytes"] = FAKE + 4, need
    assert _calls(sh, a)["decode"]() == sh.SH_EINVAL
    assert size(C.byref(a["w"]), 1000) == 0 and size(C.byref(a["w"]), 0) == 0 and size(None, 3) == 0
    a["w"].dtype = sh.SH_F32
    assert size(C.byref(a["w"]), 3) == 0


def test_prefill_workspace():
    sh = _sh()
    a = _args(sh)
    size = sh.lib.sh_window_prefill_workspace_bytes
    assert size(C.byref(a["w"]), 4, 3, 1) == 0                       # a window of 8: nothing to split
    a["w"].window = 8000
    a["cache"] = sh._WindowCache(FAKE, FAKE, 2 * 8002 * 64, 8002 * 64, 64)
    need = size(C.byref(a["w"]), 4, 3, 1)
    assert 1 << 20 < need < 1 << 25 and size(C.byref(a["w"]), 4, 3, 0) == 0 and size(C.byref(a["w"]), 1 << 20, 3, 1) == 0
    assert size(C.byref(a["w"]), 0, 3, 1) == 0 and size(C.byref(a["w"]), 4, 0, 1) == 0 and size(None, 4, 3, 1) == 0
    a["work"], a["work_bytes"] = FAKE, need - 1
    assert _calls(sh, a)["prefill"]() == sh.SH_ENOMEM
    a["work"], a["work_bytes"] = FAKE + 8, need
    assert _calls(sh, a)["prefill"]() == sh.SH_EINVAL
    a["w"].dtype = sh.SH_F32
    assert size(C.byref(a["w"]), 4, 3, 1) == 0


def test_calls_with_nothing_to_do_succeed():
    sh = _sh()
    a = _args(sh)
    a["n"] = 0
    assert all(call() == sh.SH_OK for call in _calls(sh, a).values())
    a = _args(sh)
    a["tokens"] = 0
    calls = _calls(sh, a)
    assert calls["prefill"]() == sh.SH_OK and calls["append"]() == sh.SH_OK
    q = C.byref(a["q"])
    assert sh.lib.sh_qk_norm_rope(C.byref(_rope(sh)), 0, 4, 0, q, None, FAKE, 0, q, None, None) == sh.SH_OK


def test_wrappers_refuse_tensors_on_the_host():
    import torch
    sh = _sh()
    x = torch.zeros(2, 2, 64)
    for call in (lambda: sh.qk_norm_rope(x, None, torch.zeros(2, dtype=torch.int32), None), lambda: sh.Rope(torch.zeros(32)),
                 lambda: sh.window_prefill(x, x, x, torch.zeros(3, dtype=torch.int32), window=4),
                 lambda: sh.window_append(x, x, None, None, None, None, window=4),
                 lambda: sh.window_decode(x, x, x, None, None, None, window=4)):
        with pytest.raises(ValueError):
            call()
