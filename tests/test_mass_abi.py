"""Host side of the shared contexts and the cache with accumulated weights: the entry points' argument checks (no device call is made: every
call below is refused, or has nothing to do) and the wrappers' own."""
import ctypes as C

import pytest
import torch

FAKE = 1 << 20      # an aligned address that is never dereferenced
HUGE = 1 << 40


def _sh():
    from paper_2305_17118_b200 import binding as sh
    return sh


def _args(sh):
    rows = lambda heads: sh._Rows(FAKE, heads * 64, 64)
    cache = lambda at, slots: sh._WindowCache(at, at, 2 * slots * 64, slots * 64, 64)
    return dict(a=sh._Attention(sh.SH_F16, 64, 4, 2, 10, 0.0), q=rows(4), k=rows(2), v=rows(2), out=rows(4), starts=FAKE, lengths=FAKE, seen=FAKE,
                cache=cache(FAKE, 10), rec=sh._Records(FAKE, FAKE, 20, 10), prior=None, prior_dtype=sh.SH_F16, prior_lse=None, out_dtype=sh.SH_F16,
                lse=FAKE, clear=0, tokens=4, n=3, keep=6, recent=2, into=None, into_rec=None, into_slots=0, left=FAKE + 4096, work=FAKE, work_bytes=HUGE)


def _calls(sh, x):
    ref = lambda v: None if v is None else C.byref(v)
    lib = sh.lib
    return dict(
        context=lambda: lib.sh_context_attention(ref(x["a"]), x["tokens"], x["n"], ref(x["q"]), ref(x["cache"]), x["starts"], x["lengths"], ref(x["out"]),
                                                 x["out_dtype"], x["lse"], x["clear"], x["work"], x["work_bytes"], None),
        prefill=lambda: lib.sh_mass_prefill(ref(x["a"]), x["tokens"], x["n"], ref(x["q"]), ref(x["k"]), ref(x["v"]), x["starts"], x["lengths"], x["seen"],
                                            ref(x["cache"]), ref(x["rec"]), ref(x["prior"]), x["prior_dtype"], x["prior_lse"], ref(x["out"]), x["work"],
                                            x["work_bytes"], None),
        decode=lambda: lib.sh_mass_decode(ref(x["a"]), x["n"], ref(x["q"]), ref(x["k"]), ref(x["v"]), x["lengths"], x["seen"], ref(x["cache"]),
                                          ref(x["rec"]), ref(x["prior"]), x["prior_dtype"], x["prior_lse"], ref(x["out"]), x["work"], x["work_bytes"], None),
        evict=lambda: lib.sh_mass_evict(ref(x["a"]), x["n"], x["lengths"], ref(x["cache"]), ref(x["rec"]), x["keep"], x["recent"], ref(x["into"]),
                                        ref(x["into_rec"]), x["into_slots"], x["left"], x["work"], x["work_bytes"], None))


ALL, MASS, STEPS, TOKENS = ("context", "prefill", "decode", "evict"), ("prefill", "decode", "evict"), ("prefill", "decode"), ("context", "prefill")


@pytest.mark.parametrize("which,change", [
    (ALL, dict(a=None)), (ALL, dict(a__dtype=3)), (ALL, dict(a__dtype=-1)), (ALL, dict(a__head_dim=96)), (ALL, dict(a__slots=0)),
    (ALL, dict(a__slots=1 << 30)), (ALL, dict(a__q_heads=3)), (ALL, dict(a__kv_heads=0)), (ALL, dict(a__scale=-1.0)),
    (ALL, dict(a__scale=float("nan"))), (ALL, dict(a__scale=float("inf"))), (ALL, dict(n=-1)), (TOKENS, dict(tokens=-1)),
    (TOKENS, dict(tokens=1 << 30)), (TOKENS, dict(starts=FAKE + 2)), (("prefill",), dict(starts=None)), (("context",), dict(starts=None)),
    (MASS, dict(lengths=None)), (("context",), dict(lengths=FAKE + 1)), (STEPS, dict(seen=None)), (STEPS, dict(seen=FAKE + 2)),
    (ALL, dict(cache=None)), (MASS, dict(rec=None)), (MASS, dict(rec__mass=None)), (MASS, dict(rec__positions=FAKE + 2)),
    (MASS, dict(rec__head_stride=9)), (MASS, dict(rec__sequence_stride=19)), (MASS, dict(rec__sequence_stride=-20)), (STEPS, dict(k=None)),
    (STEPS, dict(v__data=None)), (ALL[:3], dict(q=None)), (ALL[:3], dict(out=None)), (ALL[:3], dict(q__data=FAKE + 8)),
    (ALL[:3], dict(q__token_stride=68)), (ALL[:3], dict(out__token_stride=128)), (ALL, dict(cache__k=FAKE + 4)), (ALL, dict(cache__slot_stride=32)),
    (MASS, dict(cache__head_stride=64)), (MASS, dict(cache__sequence_stride=640)), (ALL, dict(cache__sequence_stride=0)),
    (("context",), dict(out_dtype=2)), (("context",), dict(clear=2)), (("context",), dict(lse=None)), (("context",), dict(lse=FAKE + 2)), (("context",), dict(out_dtype=0, out__head_stride=66)),
    (STEPS, dict(prior_lse=FAKE)), (MASS, dict(work=None)), (ALL, dict(work=FAKE + 8)),
    (("evict",), dict(keep=0)), (("evict",), dict(keep=11)), (("evict",), dict(recent=-1)), (("evict",), dict(recent=7)), (("evict",), dict(left=None)),
    (("evict",), dict(left=FAKE + 4)), (("evict",), dict(into_rec="rec")), (("evict",), dict(into="cache")),
    (("evict",), dict(into="cache", into_rec="spare", into_slots=10)), (("evict",), dict(into="other", into_rec="spare", into_slots=5)),
    (("evict",), dict(into="other", into_rec="rec", into_slots=10)),
    (("evict",), dict(into="other", into_rec="spare", into_slots=1 << 30)),
])
def test_calls_refuse(which, change):
    sh = _sh()
    x = _args(sh)
    x["spare"] = sh._Records(FAKE * 6, FAKE * 7, 20, 10)
    x["other"] = sh._WindowCache(FAKE * 4, FAKE * 4, 2 * 10 * 64, 10 * 64, 64)
    for name, value in change.items():
        if "__" in name:
            setattr(x[name.split("__")[0]], name.split("__")[1], value)
        else:
            x[name] = x[value] if name.startswith("into") and isinstance(value, str) else value
    calls = _calls(sh, x)
    for name in which:
        assert calls[name]() == sh.SH_EINVAL, name


@pytest.mark.parametrize("change", [dict(prior_dtype=2), dict(prior_dtype=3), dict(prior_lse=None), dict(prior_lse=FAKE + 2), dict(prior__data=FAKE + 8),
                                    dict(prior__token_stride=68), dict(prior_dtype=0, prior__head_stride=66)])
def test_priors_refuse(change):
    sh = _sh()
    x = _args(sh)
    x["prior"], x["prior_lse"] = sh._Rows(FAKE, 256, 64), FAKE
    for name, value in change.items():
        if "__" in name:
            setattr(x["prior"], name.split("__")[1], value)
        else:
            x[name] = value
    calls = _calls(sh, x)
    assert calls["prefill"]() == sh.SH_EINVAL and calls["decode"]() == sh.SH_EINVAL


def test_workspaces():
    sh = _sh()
    x = _args(sh)
    a, lib = C.byref(x["a"]), sh.lib
    x["a"].slots = 9000
    x["cache"] = sh._WindowCache(FAKE, FAKE, 2 * 9000 * 64, 9000 * 64, 64)
    x["rec"] = sh._Records(FAKE, FAKE, 18000, 9000)
    sizes = dict(prefill=lib.sh_mass_prefill_workspace_bytes(a, 4, 3), decode=lib.sh_mass_decode_workspace_bytes(a, 3),
                 evict=lib.sh_mass_evict_workspace_bytes(a, 3, 6, 1), context=lib.sh_context_attention_workspace_bytes(a, 3, 3, 0))
    x["tokens"] = 4
    for name, need in sizes.items():
        assert 0 < need < 1 << 24, name
        x["work_bytes"] = need - 1
        if name == "context":
            x["starts"], x["tokens"] = None, 3
        assert _calls(sh, x)[name]() == sh.SH_ENOMEM, name
    assert lib.sh_mass_prefill_workspace_bytes(a, 0, 3) == 0 and lib.sh_mass_prefill_workspace_bytes(None, 4, 3) == 0
    assert lib.sh_mass_decode_workspace_bytes(a, 0) == 0 and lib.sh_mass_decode_workspace_bytes(None, 3) == 0
    assert lib.sh_mass_evict_workspace_bytes(a, 3, 0, 1) == 0 and lib.sh_mass_evict_workspace_bytes(a, 3, 9001, 1) == 0
    assert lib.sh_mass_evict_workspace_bytes(a, 3, 11, 0) > 0
    x["a"].slots = 9
    assert lib.sh_context_attention_workspace_bytes(a, 3, 3, 0) == 0          # little to read: nothing is dealt out
    assert lib.sh_context_attention_workspace_bytes(a, 0, 3, 1) == 0 and lib.sh_context_attention_workspace_bytes(None, 4, 3, 1) == 0


def test_calls_with_nothing_to_do_succeed():
    sh = _sh()
    x = _args(sh)
    x["n"] = 0
    assert all(call() == sh.SH_OK for call in _calls(sh, x).values())
    x = _args(sh)
    x["tokens"] = 0
    calls = _calls(sh, x)
    assert calls["context"]() == sh.SH_OK and calls["prefill"]() == sh.SH_OK


def test_wrappers_refuse_tensors_on_the_host():
    sh = _sh()
    x, c = torch.zeros(2, 2, 64), torch.zeros(2, 2, 5, 64)
    m, i, p = torch.zeros(2, 2, 5), torch.zeros(2, dtype=torch.int32), torch.zeros(2, 2, 5, dtype=torch.int32)
    for call in (lambda: sh.context_attention(x, c, c), lambda: sh.mass_prefill(x, x, x, torch.zeros(3, dtype=torch.int32), i, c, c, m, p, i),
                 lambda: sh.mass_decode(x, x, x, i, c, c, m, p, i), lambda: sh.mass_evict(c, c, m, p, i, keep=2)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("change", [dict(budget=0), dict(recent=-1), dict(recent=11), dict(spare=0), dict(head_dim=96), dict(dtype="int4"),
                                    dict(kv_heads=3), dict(sequences=0), dict(scale=0.0), dict(budget=1 << 30)])
def test_mass_cache_refuses(change):
    sh = _sh()
    args = dict(sequences=2, q_heads=4, kv_heads=2, head_dim=64, budget=10, recent=2, spare=4, dtype="f16", device="cpu")
    with pytest.raises(ValueError):
        sh.MassCache(**{**args, **change})


def test_mass_cache_checks_its_prefix():
    sh = _sh()
    args = dict(sequences=2, q_heads=4, kv_heads=2, head_dim=64, budget=10, recent=2, spare=4, dtype="f16", device="cpu")
    t = lambda *shape, dtype=torch.float16: torch.zeros(shape, dtype=dtype)
    good = t(1, 2, 7, 64)
    cache = sh.MassCache(**args, prefix=(good, good))
    assert cache.first == 7 and cache.seen.tolist() == [7, 7] and cache.lengths.tolist() == [0, 0]
    for prefix in (good, (good,), (good, good, good), (good, None), (t(2, 2, 7, 64),) * 2, (t(1, 4, 7, 64),) * 2, (t(1, 2, 7, 128),) * 2,
                   (good, t(1, 2, 6, 64)), (t(1, 2, 7, 64, dtype=torch.bfloat16),) * 2, (good.transpose(2, 3).contiguous().transpose(2, 3),) * 2):
        with pytest.raises(ValueError):
            sh.MassCache(**args, prefix=prefix)
