"""Query/key preparation and the window cache on the GPU, against 64-bit definitions over full histories."""
import pytest
import torch

import window_reference as ref

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _sh():
    from paper_2305_17118_b200 import binding as sh
    return sh


def _rnd(gen, *shape, dtype, scale=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------------------ norm and rotation
def _rope(sh, gen, d, dtype, rot, sections, spread=False, adjacent=False, qn=True, kn=True, eps=1e-6):
    inv = (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))).float().cuda()
    w = lambda on: _rnd(gen, d, dtype=dtype, scale=0.3) + 1 if on else None
    return sh.Rope(inv, q_weight=w(qn), k_weight=w(kn), eps=eps, sections=sections, spread=spread, adjacent=adjacent)


def _check_rope(x, got, weight, pos, r):
    want, mag = ref.rope_ref(x, weight, pos, r.inv_freq, r.eps, r.sections, r.spread, r.adjacent)
    ref.check(got, want, ref.rope_tolerance(want, mag, x.dtype))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d,rot,sections,spread,adjacent,qn,kn", [
    (128, 128, None, False, False, True, True),
    (128, 96, (16, 16, 16), True, True, True, False),
    (128, 64, (8, 20, 4), False, False, False, True),
    (128, 32, (6, 10), False, True, False, False),
    (128, 0, None, False, False, True, True),
    (64, 64, (12, 10, 10), True, False, True, True),
    (64, 48, None, False, True, True, False),
    (64, 16, (0, 8, 0), False, False, False, False),
])
def test_norm_and_rotation(dtype, d, rot, sections, spread, adjacent, qn, kn):
    sh, gen, dt = _sh(), _gen(1), DT[dtype]
    for t, hq, hk in ((1, 1, 1), (7, 6, 2), (131, 9, 3)):
        packed = _rnd(gen, t, hq + 2 * hk, d, dtype=dt, scale=2.0)
        q, k = packed[:, :hq], packed[:, hq:hq + hk]
        r = _rope(sh, gen, d, dt, rot, sections, spread, adjacent, qn, kn)
        pos = torch.randint(0, 1 << 20, (r.axes, t), generator=gen, device="cuda", dtype=torch.int32)
        before = packed.clone()
        qo, ko = sh.qk_norm_rope(q, k, pos if r.axes > 1 else pos[0], r)
        _check_rope(q, qo, r.q_weight, pos, r)
        _check_rope(k, ko, r.k_weight, pos, r)
        assert torch.equal(packed, before)
        # in place, inside the packed rows: same bits, v untouched
        sh.qk_norm_rope(q, k, pos, r, q_out=q, k_out=k)
        assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(packed[:, hq + hk:], before[:, hq + hk:])


def test_rotation_keeps_the_phase_of_far_positions():
    sh, gen = _sh(), _gen(2)
    q = _rnd(gen, 5, 3, 128, dtype=torch.float32)
    r = _rope(sh, gen, 128, torch.float32, 128, None, qn=False, kn=False)
    pos = _i32([0, 1, (1 << 30) - 1, 1 << 30, 123456789])
    got, none = sh.qk_norm_rope(q, None, pos, r)
    assert none is None
    _check_rope(q, got, None, pos, r)


def test_rotation_layouts_and_large_token_counts():
    """Heads outermost, strided outputs with gaps, and more tokens than one wave of warps; gaps stay as they were."""
    sh, gen, dt = _sh(), _gen(3), torch.bfloat16
    q = _rnd(gen, 5, 301, 128, dtype=dt).transpose(0, 1)
    k = _rnd(gen, 2, 301, 128, dtype=dt).transpose(0, 1)
    out = torch.full((301, 9, 144), 5.0, dtype=dt, device="cuda")
    r = _rope(sh, gen, 128, dt, 128, None)
    pos = torch.arange(301, device="cuda", dtype=torch.int32)
    sh.qk_norm_rope(q, k, pos, r, q_out=out[:, :5, :128], k_out=out[:, 6:8, 16:])
    _check_rope(q, out[:, :5, :128], r.q_weight, pos, r)
    _check_rope(k, out[:, 6:8, 16:], r.k_weight, pos, r)
    assert (out[:, 5] == 5).all() and (out[:, 8] == 5).all() and (out[:, :5, 128:] == 5).all() and (out[:, 6:8, :16] == 5).all()
    x = _rnd(gen, 20011, 3, 64, dtype=torch.float16)
    r = _rope(sh, gen, 64, torch.float16, 64, None)
    pos = torch.arange(20011, device="cuda", dtype=torch.int32)
    got, _ = sh.qk_norm_rope(x, None, pos, r)
    _check_rope(x, got, r.q_weight, pos, r)
    assert sh.qk_norm_rope(x[:0], None, pos[:0], r)[0].shape == (0, 3, 64)


# ------------------------------------------------------------------------------------------------ prompts
def _history(gen, lens, ctx, hk, d, dt):
    """Full keys and values of every sequence, cached tokens first."""
    return [(_rnd(gen, c + n, hk, d, dtype=dt), _rnd(gen, c + n, hk, d, dtype=dt)) for n, c in zip(lens, ctx)]


def _caches(hist, ctx, hk, d, window, sinks, dt, fill):
    kc = torch.full((len(ctx), hk, sinks + window, d), fill, dtype=dt, device="cuda")
    vc = kc.clone()
    for i, c in enumerate(ctx):
        for slot, pos in ref.slots_ref(max(c, 0), window, sinks).items():
            kc[i, :, slot], vc[i, :, slot] = hist[i][0][pos], hist[i][1][pos]
    return kc, vc


def _prefill_case(dtype, d, hk, g, window, sinks, lens, ctx, seed=5, pad=3, fill=float("nan"), hot=1.0):
    sh, gen, dt = _sh(), _gen(seed), DT[dtype]
    hist = _history(gen, lens, ctx, hk, d, dt)
    kc, vc = _caches(hist, ctx, hk, d, window, sinks, dt, fill)
    total = sum(lens) + pad
    k, v = torch.full((2, total, hk, d), fill, dtype=dt, device="cuda")
    q = _rnd(gen, total, hk * g, d, dtype=dt, scale=hot)
    starts = [0]
    for (hk_, hv_), n, c in zip(hist, lens, ctx):
        k[starts[-1]:starts[-1] + n], v[starts[-1]:starts[-1] + n] = hk_[c:], hv_[c:]
        starts.append(starts[-1] + n)
    out = torch.full((total, hk * g, d), 7.0, dtype=dt, device="cuda")
    before = kc.clone(), vc.clone()
    sh.window_prefill(q, k, v, _i32(starts), window=window, sinks=sinks, lengths=_i32(ctx), k_cache=kc, v_cache=vc, out=out)
    torch.cuda.synchronize()
    same = lambda a, b: torch.equal(a.view(torch.int8), b.view(torch.int8))
    assert same(kc, before[0]) and same(vc, before[1])
    assert (out[starts[-1]:] == 7).all()
    for i, (n, c) in enumerate(zip(lens, ctx)):
        if n == 0:
            continue
        rows = slice(starts[i], starts[i + 1])
        want, vmax, smax = ref.attend_ref(q[rows], range(c, c + n), *hist[i], window, sinks)
        ref.check(out[rows], want, ref.attend_tolerance(want, vmax, smax, dt), f"sequence {i}")
    if not any(ctx):      # the same prompts without a cache: the same bits
        fresh = torch.full_like(out, 7.0)
        sh.window_prefill(q, k, v, _i32(starts), window=window, sinks=sinks, out=fresh)
        assert torch.equal(fresh, out)
    sh.window_append(k, v, _i32(starts), _i32(ctx), kc, vc, window=window, sinks=sinks)
    for i, (n, c) in enumerate(zip(lens, ctx)):
        live = ref.slots_ref(c + n, window, sinks)
        for slot in range(sinks + window):
            for cache, old, h in ((kc, before[0], hist[i][0]), (vc, before[1], hist[i][1])):
                if slot in live and (live[slot] >= c or slot in ref.slots_ref(c, window, sinks)):
                    assert torch.equal(cache[i, :, slot], h[live[slot]]), (i, slot)
                else:
                    assert same(cache[i, :, slot], old[i, :, slot])


SHAPES = [
    # hk, g, window, sinks, lens, ctx
    (1, 1, 1, 0, (1, 5), (0, 3)),
    (2, 4, 16, 4, (1, 0, 33, 7), (0, 9, 50, 20)),
    (1, 3, 130, 1, (129, 300), (0, 0)),
    (3, 1, 70, 130, (65, 260, 1), (128, 100, 1000)),
    (2, 7, 64, 0, (100, 64, 1, 2), (64, 63, 65, 0)),
    (1, 8, 500, 5, (20, 3), (505, 2000)),
    (2, 2, 257, 3, (400, 2), (1, 259)),
    (1, 16, 40, 2, (19,), (0,)),
    (1, 71, 33, 2, (5, 3), (0, 77)),
    (1, 130, 20, 1, (4, 2), (0, 30)),
]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s[:4])))
def test_prompt_chunks(dtype, d, shape):
    """Ragged chunks over rings before, at and after their first wrap; slots that hold no token, rows behind the last sequence and
    the chunk's padding are NaN."""
    _prefill_case(dtype, d, *shape)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_prompt_chunks_with_large_logits_and_many_sequences(dtype):
    _prefill_case(dtype, 128, 1, 2, 90, 2, (40, 300), (0, 200), seed=8, hot=12.0)
    _prefill_case(dtype, 64, 1, 1, 20, 1, [1 + i % 3 for i in range(700)], [(i * 11) % 50 for i in range(700)], seed=10)
    lens = [(i * 7) % 11 for i in range(75)]
    _prefill_case(dtype, 64, 1, 2, 24, 2, lens, [(i * 13) % 70 for i in range(75)], seed=9)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hk,g,window,sinks,lens,ctx", [
    (1, 2, 2000, 4, (1, 5, 0, 140), (2500, 3, 9, 1000)),       # parts without a tile, and all of them in use
    (2, 3, 1200, 0, (70,), (5000,)),
    (1, 71, 1500, 130, (3, 1), (1630, 64)),
    (1, 130, 2500, 0, (2,), (2400,)),
    (1, 4, 1100, 1, (1500,), (0,)),                            # a chunk that looks at itself alone
])
def test_few_rows_over_many_keys(dtype, d, hk, g, window, sinks, lens, ctx):
    """Few rows over a long context: the key tiles of a query tile go to several CTAs, whose results are merged."""
    import ctypes as C
    sh = _sh()
    w = sh._Window(sh.DTYPE_CODE[dtype], d, hk * g, hk, window, sinks, 0.0)
    assert sh.lib.sh_window_prefill_workspace_bytes(C.byref(w), sum(lens), len(lens), 1) > 0
    _prefill_case(dtype, d, hk, g, window, sinks, lens, ctx, seed=41, pad=0, fill=0.0)
    _prefill_case(dtype, d, hk, g, window, sinks, lens, ctx, seed=42, hot=8.0)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_few_rows_with_infinite_values_idle_sequences_and_without_a_workspace(dtype):
    """With and without a workspace the same result: infinite values come out in their element alone, a key that is NaN makes the
    rows that see it NaN, keys and values out of sight matter to nobody, idle sequences keep their rows, a replayed graph repeats."""
    import ctypes as C
    sh, gen, dt = _sh(), _gen(43), DT[dtype]
    hk, g, d, window, t, n, inf = 2, 3, 128, 2000, 2100, 40, float("inf")
    hist = _history(gen, [n, n], [t, t], hk, d, dt)
    vals = hist[0][1].clone()
    hist[0][1][1500, 1, 17], hist[0][1][t + 20, 0, 3], hist[0][1][50, 0, 9] = inf, -inf, inf      # (position 50 has left the window)
    kc, vc = _caches(hist, [t, t], hk, d, window, 0, dt, 0.0)
    k, v = (torch.cat([h[x][t:] for h in hist]) for x in (0, 1))
    q = _rnd(gen, 2 * n, hk * g, d, dtype=dt)
    starts, lengths = _i32([0, n, 2 * n]), _i32([t, -1])
    args = dict(window=window, lengths=lengths, k_cache=kc, v_cache=vc)
    with_work = torch.full_like(q, 7.0)
    sh.window_prefill(q, k, v, starts, out=with_work, **args)
    without = torch.full_like(q, 7.0)
    win = sh._Window(sh.DTYPE_CODE[dtype], d, hk * g, hk, window, 0, 0.0)
    rows = lambda x: C.byref(sh._Rows(x.data_ptr(), x.stride(0), x.stride(1)))
    cache = sh._WindowCache(kc.data_ptr(), vc.data_ptr(), *kc.stride()[:3])
    assert sh.lib.sh_window_prefill(C.byref(win), 2 * n, 2, rows(q), rows(k), rows(v), starts.data_ptr(), lengths.data_ptr(), C.byref(cache),
                                    rows(without), None, 0, torch.cuda.current_stream().cuda_stream) == sh.SH_OK
    replayed, graph = torch.full_like(q, 7.0), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sh.window_prefill(q, k, v, starts, out=replayed, **args)
    for _ in range(3):
        graph.replay()
    assert torch.equal(replayed, with_work)
    want, vmax, smax = ref.attend_ref(q[:n], range(t, t + n), hist[0][0], vals, window, 0)
    tol = ref.attend_tolerance(want, vmax, smax, dt)
    expect = torch.zeros(n, hk * g, d, dtype=torch.float64)
    expect[:, g:, 17], expect[20:, :g, 3] = inf, -inf
    for out in (with_work, without):
        assert (out[n:] == 7).all()
        got = out[:n].double().cpu()
        assert torch.equal(torch.where(torch.isinf(got), got, 0.0), expect)
        ref.check(torch.where(torch.isinf(got), want, got), want, tol)
    kc[0, 0, (t - 30) % window, 5] = float("nan")
    sh.window_prefill(q, k, v, starts, out=with_work, **args)
    assert torch.isnan(with_work[:n, :g]).all() and not torch.isnan(with_work[:n, g:]).any()


@pytest.mark.parametrize("dtype,hk,g,d", [("bf16", 8, 4, 128), ("f16", 16, 1, 128), ("bf16", 4, 7, 64), ("f32", 4, 2, 64)])
def test_prompts_that_fill_the_device(dtype, hk, g, d):
    """Many tiles on every SM, short and long sequences mixed: every row against a definition in 64 bits, and run after run the same."""
    sh, gen, dt = _sh(), _gen(14), DT[dtype]
    lens, ctx, window, sinks = (1, 200, 777, 1500, 0, 130, 640), (0, 100, 0, 700, 5, 3000, 650), 640, 4
    hist = _history(gen, lens, ctx, hk, d, dt)
    kc, vc = _caches(hist, ctx, hk, d, window, sinks, dt, 0.0)
    k, v = (torch.cat([h[x][c:] for h, c in zip(hist, ctx)]) for x in (0, 1))
    q = _rnd(gen, sum(lens), hk * g, d, dtype=dt)
    starts = [sum(lens[:i]) for i in range(len(lens) + 1)]
    args = dict(window=window, sinks=sinks, lengths=_i32(ctx), k_cache=kc, v_cache=vc)
    out = sh.window_prefill(q, k, v, _i32(starts), **args)
    for _ in range(12):
        assert torch.equal(sh.window_prefill(q, k, v, _i32(starts), **args), out)
    for i, (n, c) in enumerate(zip(lens, ctx)):
        if n == 0:
            continue
        keys, vals = (x.double().repeat_interleave(g, 1).transpose(0, 1) for x in hist[i])      # [hq, c + n, d]
        qs = q[starts[i]:starts[i + 1]].double().transpose(0, 1)
        see = ref.visible(torch.arange(c, c + n)[:, None], torch.arange(c + n)[None], window, sinks).cuda()
        logits = (qs @ keys.transpose(1, 2) * d ** -0.5).masked_fill(~see, float("-inf"))
        want = (torch.softmax(logits, -1) @ vals).transpose(0, 1).cpu()
        vmax = vals.abs().amax((1, 2)).view(1, -1, 1).cpu()
        smax = (qs.abs().amax((1, 2)) * keys.abs().sum(-1).amax(-1) * d ** -0.5).view(1, -1, 1).cpu()
        ref.check(out[starts[i]:starts[i + 1]], want, ref.attend_tolerance(want, vmax, smax, dt), f"sequence {i}")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_tokens_out_of_sight_never_matter(dtype, bad):
    """A key or value that is not finite reaches the queries that see it and no other."""
    sh, gen, dt = _sh(), _gen(11), DT[dtype]
    n, window, sinks, hk, g, d = 300, 40, 3, 2, 2, 128
    q, k, v = _rnd(gen, n, hk * g, d, dtype=dt), _rnd(gen, n, hk, d, dtype=dt), _rnd(gen, n, hk, d, dtype=dt)
    starts = _i32([0, n])
    clean = sh.window_prefill(q, k, v, starts, window=window, sinks=sinks)
    at = 150
    for which in (0, 1):
        k2, v2 = k.clone(), v.clone()
        (k2, v2)[which][at, 1] = bad
        out = sh.window_prefill(q, k2, v2, starts, window=window, sinks=sinks)
        sees = ref.visible(torch.arange(n), torch.tensor(at), window, sinks).cuda()
        assert torch.equal(out[:, :g], clean[:, :g])                 # the other key head
        got, want = out[~sees, g:].double().cpu(), clean[~sees, g:].double().cpu()
        assert torch.isfinite(got).all()
        tol = 4 * ref.half_step(dt) * v.double().abs().max().item()      # (another kernel path may serve such rows)
        assert (got - want).abs().max() <= tol
        if which == 1:
            assert not torch.isfinite(out[sees, g:]).any()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_prompt_layouts(dtype):
    """Views of a packed projection, heads outermost, caches with the slot dimension outside the heads, strided outputs."""
    sh, gen, dt = _sh(), _gen(12), DT[dtype]
    n, hq, hk, d, window, sinks, c = 150, 6, 2, 64, 48, 3, 100
    hist = _history(gen, [n], [c], hk, d, dt)
    kc, vc = _caches(hist, [c], hk, d, window, sinks, dt, 0.0)
    q = _rnd(gen, n, hq, d, dtype=dt)
    k, v = hist[0][0][c:], hist[0][1][c:]
    args = dict(window=window, sinks=sinks, lengths=_i32([c]))
    plain = sh.window_prefill(q, k, v, _i32([0, n]), k_cache=kc, v_cache=vc, **args)
    packed = torch.cat([q, k, v], 1)
    heads_out = lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)
    slots_out = lambda x: x.transpose(1, 2).contiguous().transpose(1, 2)
    out = torch.full((hq, n, d + 16), 5.0, dtype=dt, device="cuda")
    sh.window_prefill(packed[:, :hq], packed[:, hq:hq + hk], packed[:, hq + hk:], _i32([0, n]), k_cache=slots_out(kc), v_cache=slots_out(vc),
                      out=out[:, :, :d].transpose(0, 1), **args)
    assert torch.equal(out[:, :, :d].transpose(0, 1), plain) and (out[:, :, d:] == 5).all()
    got = sh.window_prefill(heads_out(q), heads_out(k), heads_out(v), _i32([0, n]), k_cache=kc, v_cache=vc, **args)
    assert torch.equal(got, plain)
    k2, v2 = slots_out(kc), slots_out(vc)
    sh.window_append(packed[:, hq:hq + hk], packed[:, hq + hk:], _i32([0, n]), _i32([c]), k2, v2, window=window, sinks=sinks)
    sh.window_append(k, v, _i32([0, n]), _i32([c]), kc, vc, window=window, sinks=sinks)
    assert torch.equal(k2, kc) and torch.equal(v2, vc)


def test_starts_that_make_no_sense_stay_inside_the_tensors():
    """Offsets outside the tensor or decreasing are clamped: neighbouring memory keeps its contents."""
    sh, gen, dt = _sh(), _gen(13), torch.bfloat16
    n, d = 40, 64
    guard = torch.full((3 * n, 2, d), 3.0, dtype=dt, device="cuda")
    q, k, v = (_rnd(gen, n, 2, d, dtype=dt) for _ in range(3))
    cache = torch.zeros(3, 2, 12, d, dtype=dt, device="cuda")
    for starts in ([0, 50, 1 << 30, 5], [-7, 20, 10, 90], [30, 20, 10, 0]):
        sh.window_prefill(q, k, v, _i32(starts), window=10, sinks=2, lengths=_i32([0, 3, 5]), k_cache=cache, v_cache=cache.clone(),
                          out=guard[n:2 * n])
        sh.window_append(k, v, _i32(starts), _i32([0, 3, 5]), cache, cache.clone(), window=10, sinks=2)
    torch.cuda.synchronize()
    assert (guard[:n] == 3).all() and (guard[2 * n:] == 3).all()


# ------------------------------------------------------------------------------------------------ single tokens
def _decode_case(dtype, d, hk, g, window, sinks, ctx, rope=False, seed=21, hot=1.0):
    sh, gen, dt = _sh(), _gen(seed), DT[dtype]
    n = len(ctx)
    hist = _history(gen, [1] * n, [max(c, 0) for c in ctx], hk, d, dt)
    kc, vc = _caches(hist, ctx, hk, d, window, sinks, dt, float("nan"))
    packed = _rnd(gen, n, hk * (g + 2), d, dtype=dt, scale=hot)
    q, k, v = packed[:, :hk * g], packed[:, hk * g:hk * (g + 1)], packed[:, hk * (g + 1):]
    r = _rope(sh, gen, d, dt, d // 2, None) if rope else None
    out = torch.full((n, hk * g, d), 7.0, dtype=dt, device="cuda")
    before = kc.clone(), vc.clone()
    sh.window_decode(q, k, v, _i32(ctx), kc, vc, window=window, sinks=sinks, rope=r, out=out)
    same = lambda a, b: torch.equal(a.view(torch.int8), b.view(torch.int8))
    qq = q
    if rope:
        pos = _i32([max(c, 0) for c in ctx])
        qq, _ = ref.rope_ref(q, r.q_weight, pos, r.inv_freq, r.eps, r.sections, False, False)
        kk, mag = ref.rope_ref(k, r.k_weight, pos, r.inv_freq, r.eps, r.sections, False, False)
    for i, c in enumerate(ctx):
        if c < 0:
            assert (out[i] == 7).all() and same(kc[i], before[0][i]) and same(vc[i], before[1][i])
            continue
        slot = c if c < sinks else sinks + (c - sinks) % window
        stored = kc[i, :, slot]
        if rope:
            ref.check(stored, kk[i], ref.rope_tolerance(kk[i], mag[i], dt), "stored key")
        else:
            assert torch.equal(stored, k[i])
        assert torch.equal(vc[i, :, slot], v[i])
        others = [s for s in range(sinks + window) if s != slot]
        assert same(kc[i][:, others], before[0][i][:, others]) and same(vc[i][:, others], before[1][i][:, others])
        hist[i][0][c], hist[i][1][c] = stored, v[i]
        want, vmax, smax = ref.attend_ref(qq[i:i + 1], [c], *hist[i], window, sinks)
        ref.check(out[i:i + 1], want, ref.attend_tolerance(want, vmax, smax, dt), f"sequence {i} at {c}")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hk,g,window,sinks,rope", [(1, 1, 1, 0, False), (2, 4, 24, 4, True), (3, 1, 150, 2, False), (1, 7, 33, 0, True),
                                                    (2, 8, 100, 130, False), (1, 2, 600, 1, False), (1, 20, 65, 3, True), (5, 3, 17, 16, False)])
def test_single_tokens(dtype, d, hk, g, window, sinks, rope):
    """Lengths before, at and after each border of the cache, idle slots among them; slots that hold no token are NaN."""
    s, w = sinks, window
    ctx = sorted({0, 1, max(s - 1, 0), s, s + 1, s + w - 1, s + w, s + w + 1, s + 2 * w, 3 * w + 17}) + [-1]
    _decode_case(dtype, d, hk, g, window, sinks, ctx, rope)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d,rot,sections,spread,adjacent,qn,kn", [
    (128, 128, (24, 20, 20), False, False, True, True),
    (128, 96, (16, 16, 16), True, True, False, True),
    (64, 64, (12, 20), False, True, True, False),
    (64, 32, (6, 5, 5), True, False, False, False),
])
def test_single_tokens_prepared_in_the_same_launch(dtype, d, rot, sections, spread, adjacent, qn, kn):
    """Every form of the preparation inside the step, with positions of their own: the stored key is the prepared one, and the output is
    that of the prepared query over what is stored."""
    sh, gen, dt = _sh(), _gen(29), DT[dtype]
    n, hk, g, window, sinks, c = 3, 2, 5, 40, 3, 57
    hist = _history(gen, [1] * n, [c] * n, hk, d, dt)
    kc, vc = _caches(hist, [c] * n, hk, d, window, sinks, dt, float("nan"))
    q, k, v = _rnd(gen, n, hk * g, d, dtype=dt), _rnd(gen, n, hk, d, dtype=dt), _rnd(gen, n, hk, d, dtype=dt)
    r = _rope(sh, gen, d, dt, rot, sections, spread, adjacent, qn, kn)
    pos = torch.randint(0, 1 << 20, (len(sections), n), generator=gen, device="cuda", dtype=torch.int32)
    out = sh.window_decode(q, k, v, _i32([c] * n), kc, vc, window=window, sinks=sinks, rope=r, positions=pos)
    args = (pos, r.inv_freq, r.eps, r.sections, spread, adjacent)
    want_q, _ = ref.rope_ref(q, r.q_weight, *args)
    want_k, mag = ref.rope_ref(k, r.k_weight, *args)
    slot = sinks + (c - sinks) % window
    for i in range(n):
        stored = kc[i, :, slot]
        ref.check(stored, want_k[i], ref.rope_tolerance(want_k[i], mag[i], dt), "stored key")
        hist[i][0][c], hist[i][1][c] = stored, v[i]
        want, vmax, smax = ref.attend_ref(want_q[i:i + 1], [c], *hist[i], window, sinks)
        ref.check(out[i:i + 1], want, ref.attend_tolerance(want, vmax, smax, dt))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_other_scales_and_rows_before_the_first_sequence(dtype):
    sh, gen, dt = _sh(), _gen(30), DT[dtype]
    q, k, v = _rnd(gen, 90, 4, 64, dtype=dt), _rnd(gen, 90, 2, 64, dtype=dt), _rnd(gen, 90, 2, 64, dtype=dt)
    out = torch.full_like(q, 7.0)
    sh.window_prefill(q, k, v, _i32([5, 70, 80]), window=30, sinks=1, scale=0.31, out=out)
    assert (out[:5] == 7).all() and (out[80:] == 7).all()
    for a, b in ((5, 70), (70, 80)):
        want, vmax, smax = ref.attend_ref(q[a:b], range(b - a), k[a:b], v[a:b], 30, 1, scale=0.31)
        ref.check(out[a:b], want, ref.attend_tolerance(want, vmax, smax, dt))
    kc, vc = torch.zeros(1, 2, 31, 64, dtype=dt, device="cuda"), torch.zeros(1, 2, 31, 64, dtype=dt, device="cuda")
    sh.window_append(k, v, _i32([5, 70]), _i32([0]), kc, vc, window=30, sinks=1)
    step = sh.window_decode(q[70:71], k[70:71], v[70:71], _i32([65]), kc, vc, window=30, sinks=1, scale=0.31)
    want, vmax, smax = ref.attend_ref(q[70:71], [65], k[5:71], v[5:71], 30, 1, scale=0.31)
    ref.check(step, want, ref.attend_tolerance(want, vmax, smax, dt))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_single_tokens_over_long_axes_and_large_batches(dtype):
    _decode_case(dtype, 128, 2, 4, 5000, 4, [20011], rope=True)              # one sequence: the axis is split
    _decode_case(dtype, 64, 1, 1, 3001, 0, [2500, 7000, -1], seed=22)
    _decode_case(dtype, 128, 1, 11, 9000, 3, [9100], seed=25, rope=True)
    _decode_case(dtype, 64, 3, 2, 20000, 0, [-1, 19999, 3], seed=27)
    _decode_case(dtype, 128, 4, 2, 30, 2, [(i * 37) % 90 for i in range(190)], seed=23)
    _decode_case(dtype, 128, 2, 2, 200, 2, [500, 150], seed=24, hot=12.0)    # one key takes nearly all the weight


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_long_axes_with_infinite_values_and_without_a_workspace(dtype):
    """The axis is split over the device (a second launch merges) or, without a workspace, over a cluster: the same result; values
    that are infinite come out in their element alone."""
    import ctypes as C
    sh, gen, dt = _sh(), _gen(28), DT[dtype]
    hk, g, d, window, t, inf = 2, 3, 128, 8000, 8100, float("inf")
    hist = _history(gen, [1], [t], hk, d, dt)
    hist[0][1][5000, 1, 17], hist[0][1][t, 0, 3], hist[0][1][50, 0, 9] = inf, -inf, inf      # (position 50 has left the window)
    kc, vc = _caches(hist, [t], hk, d, window, 0, dt, float("nan"))
    q, k, v = _rnd(gen, 1, hk * g, d, dtype=dt), hist[0][0][t:], hist[0][1][t:]
    outs = []
    for work in (True, False):
        k2, v2 = kc.clone(), vc.clone()
        if work:
            out = sh.window_decode(q, k, v, _i32([t]), k2, v2, window=window)
        else:
            out, lengths = torch.zeros_like(q), _i32([t])
            win = sh._Window(sh.DTYPE_CODE[dtype], d, hk * g, hk, window, 0, 0.0)
            rows = lambda x: C.byref(sh._Rows(x.data_ptr(), x.stride(0), x.stride(1)))
            cache = sh._WindowCache(k2.data_ptr(), v2.data_ptr(), *k2.stride()[:3])
            assert sh.lib.sh_window_decode(C.byref(win), 1, rows(q), rows(k), rows(v), lengths.data_ptr(), C.byref(cache), None, None, 0,
                                           rows(out), None, 0, torch.cuda.current_stream().cuda_stream) == sh.SH_OK
        outs.append(out.double().cpu())
    vals = hist[0][1].clone()
    vals[torch.isinf(vals)] = 0
    want, vmax, smax = ref.attend_ref(q, [t], hist[0][0], vals, window, 0)
    tol = ref.attend_tolerance(want, vmax, smax, dt)
    expect = torch.zeros(hk * g, d, dtype=torch.float64)
    expect[g:, 17], expect[:g, 3] = inf, -inf
    for out in outs:
        assert torch.equal(torch.where(torch.isinf(out[0]), out[0], 0.0), expect)
        ref.check(torch.where(torch.isinf(out), want, out), want, tol)


def test_cache_offsets_pass_32_bits():
    """A cache of more than 2^31 elements: equal keys give the mean of the values, which are zero but for some far rows."""
    sh, dt, d = _sh(), torch.float16, 128
    window = (1 << 24) + 77
    kc = torch.zeros(1, 1, window, d, dtype=dt, device="cuda")
    vc = torch.zeros_like(kc)
    t = window - 1
    marks = [0, 5, window // 2, window - 40, window - 2]
    for i, m in enumerate(marks):
        vc[0, 0, m, i] = 60000.0
    q = torch.zeros(1, 2, d, dtype=dt, device="cuda")
    k = torch.zeros(1, 1, d, dtype=dt, device="cuda")
    v = torch.zeros(1, 1, d, dtype=dt, device="cuda")
    out = sh.window_decode(q, k, v, _i32([t]), kc, vc, window=window)
    want = torch.zeros(d, dtype=torch.float64)
    want[:len(marks)] = 60000.0 / window
    for h in range(2):
        # 60000 / 2^24 lies among the subnormal fp16 numbers, whose step is 2^-24
        assert ((out[0, h].double().cpu() - want).abs() <= 2.0 ** -25 + want * 2.0 ** -11).all()
    out = sh.window_prefill(q, k, v, _i32([0, 1]), window=window, lengths=_i32([t]), k_cache=kc, v_cache=vc)
    for h in range(2):
        assert ((out[0, h].double().cpu() - want).abs() <= 2.0 ** -25 + want * 2.0 ** -10).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_infinite_values_in_sight_come_out(dtype):
    """An infinite value that a query sees makes that element of its output infinite, and no other element."""
    sh, gen, dt = _sh(), _gen(26), DT[dtype]
    n, d, g, inf = 200, 128, 3, float("inf")
    q, k, v = _rnd(gen, n, g, d, dtype=dt), _rnd(gen, n, 1, d, dtype=dt), _rnd(gen, n, 1, d, dtype=dt)
    v[120, 0, 17] = inf
    v[130, 0, 40] = -inf
    out = sh.window_prefill(q, k, v, _i32([0, n]), window=60, sinks=1)
    kc, vc = torch.zeros(1, 1, 61, d, dtype=dt, device="cuda"), torch.zeros(1, 1, 61, d, dtype=dt, device="cuda")
    sh.window_append(k[:-1], v[:-1], _i32([0, n - 1]), _i32([0]), kc, vc, window=60, sinks=1)
    late = v.clone()
    late[150, 0, 17], late[n - 1, 0, 99] = inf, inf
    sh.window_append(k[:-1], late[:-1], _i32([0, n - 1]), _i32([0]), kc, vc, window=60, sinks=1)
    step = sh.window_decode(q[-1:], k[-1:], late[-1:], _i32([n - 1]), kc, vc, window=60, sinks=1)
    for i in range(n):
        want = torch.zeros(d)
        want[17] = inf if 120 <= i < 180 else 0
        want[40] = -inf if 130 <= i < 190 else 0
        for h in range(g):
            got = out[i, h].float().cpu()
            assert torch.equal(torch.where(torch.isinf(got), got, 0.0), want) and not torch.isnan(got).any(), i
    want = torch.zeros(d)
    want[17], want[99] = inf, inf
    for h in range(g):
        got = step[0, h].float().cpu()
        assert torch.equal(torch.where(torch.isinf(got), got, 0.0), want) and not torch.isnan(got).any()


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_a_served_batch_from_prompts_to_tokens(dtype):
    """WindowCache: prompts in two rounds of ragged chunks, then tokens, one sequence idle; raw projections in, compared with
    attention over the full history of rotated keys."""
    sh, gen, dt = _sh(), _gen(31), DT[dtype]
    n, hq, hk, d, window, sinks = 3, 4, 2, 64, 37, 3
    r = _rope(sh, gen, d, dt, 64, None)
    cache = sh.WindowCache(n, hq, hk, d, window, sinks, dtype=dt, rope=r)
    cache.lengths[2] = -1
    hist = [[], []]
    for lens in ([50, 20], [30, 1], None, None, None):
        if lens is not None:
            starts = [0, lens[0], sum(lens), sum(lens) + 2]
            rows = [slice(starts[i], starts[i + 1]) for i in range(2)]
        else:
            rows = [slice(i, i + 1) for i in range(2)]
        total = sum(lens) + 5 if lens is not None else 3
        packed = _rnd(gen, total, hq + 2 * hk, d, dtype=dt)
        q, k, v = packed[:, :hq], packed[:, hq:hq + hk], packed[:, hq + hk:]
        out = cache.prefill(q, k, v, _i32(starts)) if lens is not None else cache.decode(q, k, v)
        for i in range(2):
            c = len(hist[i])
            m = rows[i].stop - rows[i].start
            pos = torch.arange(c, c + m, device="cuda", dtype=torch.int32)
            qr, kr = sh.qk_norm_rope(q[rows[i]], k[rows[i]], pos, r)
            hist[i] += list(zip(kr, v[rows[i]]))
            keys, vals = torch.stack([x for x, _ in hist[i]]), torch.stack([x for _, x in hist[i]])
            if lens is None:      # the step's query is not rounded between the rotation and the attention
                qr, _ = ref.rope_ref(q[rows[i]], r.q_weight, pos, r.inv_freq, r.eps, r.sections, False, False)
            want, vmax, smax = ref.attend_ref(qr, range(c, c + m), keys, vals, window, sinks)
            # the fused step may round a key the other way when it lies at a tie, within the fp32 error of the norm: one step of one key
            tie = ref.half_step(dt) * 2 * smax * 2 * vmax if lens is None else 0.0
            ref.check(out[rows[i]], want, ref.attend_tolerance(want, vmax, smax, dt) + tie)
        assert cache.lengths.tolist() == [len(hist[0]), len(hist[1]), -1]


def test_prepared_rows_feed_the_budgeted_cache():
    """qk_norm_rope writes what Handle.prefill and Handle.decode_step take; with a budget beyond the stream the result is full
    causal attention, which is also the window cache's with a window beyond the stream."""
    sh, gen, dt = _sh(), _gen(32), torch.float16
    n, heads, d = 90, 4, 128
    packed = _rnd(gen, n + 1, 3 * heads, d, dtype=dt)
    r = _rope(sh, gen, d, dt, 128, None)
    pos = torch.arange(n + 1, device="cuda", dtype=torch.int32)
    q, k = sh.qk_norm_rope(packed[:, :heads], packed[:, heads:2 * heads], pos, r)
    v = packed[:, 2 * heads:].contiguous()
    h = sh.Handle(B=128, r=8, w=64, m=16, heads=heads, head_dim=d, dtype="f16")
    out = torch.empty(n, heads, d, dtype=torch.float32, device="cuda")
    h.prefill(q[:n], k[:n], v[:n], out=out)
    step = h.decode_step(q[n], k[n], v[n])
    cache = sh.WindowCache(1, heads, heads, d, 200, 0, dtype="f16")
    got = cache.prefill(q[:n], k[:n], v[:n], _i32([0, n]))
    got1 = cache.decode(q[n:], k[n:], v[n:])
    want, vmax, smax = ref.attend_ref(q, range(n + 1), k, v, 1 << 20, 0)
    tol = ref.attend_tolerance(want, vmax, smax, dt)
    ref.check(out, want[:n], 2e-3 + tol[:n])
    ref.check(step[None], want[n:], 2e-3 + tol[n:])
    ref.check(got, want[:n], tol[:n])
    ref.check(got1, want[n:], tol[n:])


@pytest.fixture(autouse=True)
def _no_wait_gave_up():
    yield
    _sh().window_status()


def test_graphs_streams_and_calls_at_once():
    """Captured calls replay on new inputs; two graphs and an eager call run at once on three streams with the same results."""
    sh, gen, dt = _sh(), _gen(33), torch.bfloat16
    n, hq, hk, d, window, sinks = 4, 8, 2, 128, 700, 4
    r = _rope(sh, gen, d, dt, 128, None)
    long = 30000                                     # a window over which one sequence spreads out
    mk = lambda: dict(lk=_rnd(gen, 1, hk, long, d, dtype=dt), lv=_rnd(gen, 1, hk, long, d, dtype=dt), lo=torch.empty(1, hq, d, dtype=dt, device="cuda"),
                      ll=_i32([70001]), p=_rnd(gen, n, hq + 2 * hk, d, dtype=dt), kc=_rnd(gen, n, hk, window + sinks, d, dtype=dt),
                      vc=_rnd(gen, n, hk, window + sinks, d, dtype=dt), x=_rnd(gen, 200, hq + 2 * hk, d, dtype=dt),
                      out=torch.empty(n, hq, d, dtype=dt, device="cuda"), xo=torch.zeros(200, hq, d, dtype=dt, device="cuda"),
                      lengths=_i32([900, 5, -1, 704]), starts=_i32([0, 150, 150, 160, 190]))

    def work(s):
        pk = s["p"]
        sh.window_prefill(s["x"][:, :hq], s["x"][:, hq:hq + hk], s["x"][:, hq + hk:], s["starts"], window=window, sinks=sinks,
                          lengths=s["lengths"], k_cache=s["kc"], v_cache=s["vc"], out=s["xo"])
        sh.window_decode(pk[:, :hq], pk[:, hq:hq + hk], pk[:, hq + hk:], s["lengths"], s["kc"], s["vc"], window=window, sinks=sinks, rope=r,
                         out=s["out"])
        sh.window_decode(pk[:1, :hq], pk[:1, hq:hq + hk], pk[:1, hq + hk:], s["ll"], s["lk"], s["lv"], window=long, out=s["lo"])

    a, b, c = mk(), mk(), mk()
    want = []
    for s in (a, b, c):
        t = {x: y.clone() for x, y in s.items()}
        work(t)
        want.append(t)
    torch.cuda.synchronize()
    graphs = []
    for s in (a, b):
        t = {x: torch.zeros_like(y) for x, y in s.items()}
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            work(t)                                  # warm-up outside the capture, on the inputs of nobody
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            work(t)
        for x in t:
            t[x].copy_(s[x])
        graphs.append((g, t))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    eager = {x: y.clone() for x, y in c.items()}
    torch.cuda.synchronize()
    for (g, _), st in zip(graphs, streams):
        with torch.cuda.stream(st):
            g.replay()
    with torch.cuda.stream(streams[2]):
        work(eager)
    torch.cuda.synchronize()
    for got, w in zip([graphs[0][1], graphs[1][1], eager], want):
        live = [0, 1, 3]
        assert torch.equal(got["out"][live], w["out"][live])
        for x in ("xo", "kc", "vc", "lo", "lk", "lv"):
            assert torch.equal(got[x], w[x]), x


FIRST_CALLS = """
import torch
from paper_2305_17118_b200 import binding as sh
torch.manual_seed(5)
for dt, d, axis in ((torch.bfloat16, 128, 30000), (torch.float16, 64, 30000), (torch.bfloat16, 64, 300), (torch.float16, 128, 300), (torch.float32, 64, 300), (torch.float32, 128, 300)):
    q, k, v = torch.randn(40, 8, d, device="cuda").to(dt), torch.randn(40, 2, d, device="cuda").to(dt), torch.randn(40, 2, d, device="cuda").to(dt)
    kc, vc = torch.randn(1, 2, axis, d, device="cuda").to(dt), torch.randn(1, 2, axis, d, device="cuda").to(dt)
    r = sh.Rope(torch.rand(d // 2, device="cuda"), q_weight=torch.ones(d, device="cuda", dtype=dt))
    pos, starts, ln = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (list(range(40)), [0, 40], [70001]))
    def calls(kc, vc):
        a, b = sh.qk_norm_rope(q, k, pos, r)
        c = sh.window_prefill(a, b, v, starts, window=axis, lengths=ln, k_cache=kc, v_cache=vc)
        sh.window_append(b, v, starts, ln, kc, vc, window=axis)
        return c, sh.window_decode(q[:1], k[:1], v[:1], ln + 40, kc, vc, window=axis, rope=r)
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    mine = kc.clone(), vc.clone()
    ln + 40
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):      # the first call of each kernel is captured
        got = calls(*mine)
    mine[0].copy_(kc), mine[1].copy_(vc)
    g.replay()
    torch.cuda.synchronize()
    for x, y in zip(got, calls(kc, vc)):
        assert torch.equal(x, y)
    sh.window_status()
print("same")
"""


def test_the_first_calls_of_a_process_can_be_captured():
    import pathlib
    import subprocess
    import sys
    done = subprocess.run([sys.executable, "-c", FIRST_CALLS], cwd=pathlib.Path(__file__).parent.parent, capture_output=True, text=True, timeout=240)
    assert done.returncode == 0 and done.stdout.strip() == "same", done.stderr[-2000:]


def test_results_on_another_stream_than_the_current_one():
    """New outputs and workspaces belong to the stream of the call, not to the current one, which is kept busy meanwhile."""
    sh, gen, dt = _sh(), _gen(36), torch.bfloat16
    q, k, v = _rnd(gen, 500, 4, 128, dtype=dt), _rnd(gen, 500, 2, 128, dtype=dt), _rnd(gen, 500, 2, 128, dtype=dt)
    kc, vc = _rnd(gen, 1, 2, 20000, 128, dtype=dt), _rnd(gen, 1, 2, 20000, 128, dtype=dt)
    r = _rope(sh, gen, 128, dt, 128, None)
    pos, starts, ln = torch.arange(500, device="cuda", dtype=torch.int32), _i32([0, 300, 480]), _i32([50000])

    def calls(stream):
        a = sh.qk_norm_rope(q, k, pos, r, stream=stream)
        b = sh.window_prefill(q, k, v, starts, window=90, sinks=2, stream=stream)
        c = sh.window_decode(q[:1], k[:1], v[:1], ln, kc, vc, window=20000, rope=r, stream=stream)
        return (*a, b, c)

    want = calls(None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    big = torch.randn(8192, 8192, device="cuda")
    for _ in range(3):
        for _ in range(4):
            big @ big                                # the current stream falls behind
        got = calls(side)
        side.synchronize()
        with torch.cuda.stream(side):
            assert all(torch.equal(x, y) for x, y in zip(got, want))
        del got
    torch.cuda.synchronize()


def test_results_do_not_depend_on_the_run():
    """No atomics whose order could change a result: repeated calls give the same bits."""
    sh, gen, dt = _sh(), _gen(34), torch.bfloat16
    q, k, v = _rnd(gen, 1000, 8, 128, dtype=dt), _rnd(gen, 1000, 2, 128, dtype=dt), _rnd(gen, 1000, 2, 128, dtype=dt)
    kc, vc = _rnd(gen, 1, 2, 5004, 128, dtype=dt), _rnd(gen, 1, 2, 5004, 128, dtype=dt)
    first = None
    for _ in range(4):
        a = sh.window_prefill(q, k, v, _i32([0, 600, 1000]), window=300, sinks=4)
        b = sh.window_decode(q[:1], k[:1], v[:1], _i32([9000]), kc, vc, window=5000, sinks=4)
        if first is None:
            first = a, b
        assert torch.equal(a, first[0]) and torch.equal(b, first[1])


def test_wrappers_refuse_what_the_kernels_cannot_take():
    sh, gen, dt = _sh(), _gen(35), torch.bfloat16
    q, k, v = _rnd(gen, 4, 4, 64, dtype=dt), _rnd(gen, 4, 2, 64, dtype=dt), _rnd(gen, 4, 2, 64, dtype=dt)
    kc, vc = _rnd(gen, 4, 2, 10, 64, dtype=dt), _rnd(gen, 4, 2, 10, 64, dtype=dt)
    ln, st = _i32([0, 1, 2, 3]), _i32([0, 1, 2, 3, 4])
    win = dict(window=8, sinks=2)
    r = _rope(sh, gen, 64, dt, 64, None)
    ok = sh.window_decode(q, k, v, ln, kc, vc, **win)
    assert ok.shape == q.shape
    bad = [
        lambda: sh.window_decode(q, k, v, ln, kc, vc, window=0, sinks=2),
        lambda: sh.window_decode(q, k, v, ln, kc, vc, window=9, sinks=2),
        lambda: sh.window_decode(q, k, v, ln, kc, vc, scale=0.0, **win),
        lambda: sh.window_decode(q[:, :3], k, v, ln, kc, vc, **win),
        lambda: sh.window_decode(q, k, v[:3], ln, kc, vc, **win),
        lambda: sh.window_decode(q, k.float(), v, ln, kc, vc, **win),
        lambda: sh.window_decode(q, k, v, ln.long(), kc, vc, **win),
        lambda: sh.window_decode(q, k, v, ln.cpu(), kc, vc, **win),
        lambda: sh.window_decode(q, k, v, ln[:3], kc, vc, **win),
        lambda: sh.window_decode(q, k, v, ln, kc, vc[:, :, :9], **win),
        lambda: sh.window_decode(q, k, v, ln, kc, vc.transpose(1, 2).contiguous().transpose(1, 2), **win),
        lambda: sh.window_decode(q, k, v, ln, kc, vc, positions=ln, **win),
        lambda: sh.window_decode(q, k, v, ln, kc, vc, rope=_rope(sh, gen, 128, dt, 64, None), **win),
        lambda: sh.window_decode(q, k, v, ln, kc, vc, rope=_rope(sh, gen, 64, dt, 64, (20, 6, 6)), **win),
        lambda: sh.window_decode(q, k, v, ln, kc, vc, out=torch.empty(4, 4, 64, device="cuda"), **win),
        lambda: sh.window_prefill(q.cpu(), k, v, st, **win),
        lambda: sh.window_prefill(q, k, v, st, lengths=ln, **win),
        lambda: sh.window_prefill(q, k, v, st, k_cache=kc, v_cache=vc, **win),
        lambda: sh.window_prefill(q, k, v, st.float(), **win),
        lambda: sh.window_prefill(q[..., ::2], k, v, st, **win),
        lambda: sh.window_append(k, v, st, ln[:2], kc, vc, **win),
        lambda: sh.qk_norm_rope(q, k, ln[:3], r),
        lambda: sh.qk_norm_rope(q, k[:3], ln, r),
        lambda: sh.qk_norm_rope(q, None, ln, r, k_out=k),
        lambda: sh.qk_norm_rope(q.float(), k.float(), ln, r),
        lambda: sh.Rope(r.inv_freq[:12]),
        lambda: sh.Rope(r.inv_freq, sections=(16, 8)),
        lambda: sh.Rope(r.inv_freq, spread=True),
        lambda: sh.Rope(r.inv_freq.half()),
        lambda: sh.WindowCache(0, 4, 2, 64, 8),
        lambda: sh.WindowCache(2, 4, 2, 96, 8),
        lambda: sh.WindowCache(2, 4, 2, 64, 8, dtype="int4"),
        lambda: sh.WindowCache(2, 3, 2, 64, 8),
        lambda: sh.WindowCache(4, 8, 2, 64, 8, dtype=dt).decode(q, k, v),
        lambda: sh.WindowCache(4, 8, 2, 64, 8, dtype=dt).prefill(q, k, v, st),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was taken")
    # refused by the library: misaligned addresses, broadcast rows, outputs that share elements
    wide = _rnd(gen, 4, 4, 72, dtype=dt)
    for call in (lambda: sh.window_decode(wide[..., 3:67], k, v, ln, kc, vc, **win),
                 lambda: sh.window_prefill(q, k[:, :1].expand(4, 2, 64), v, st, **win),
                 lambda: sh.qk_norm_rope(q, None, ln, r, q_out=torch.empty(4, 1, 64, dtype=dt, device="cuda").expand(4, 4, 64)),
                 lambda: sh.qk_norm_rope(q, None, ln, sh.Rope(r.inv_freq, eps=float("nan")))):
        with pytest.raises(sh.ShError) as e:
            call()
        assert e.value.status == sh.SH_EINVAL
