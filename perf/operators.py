"""What the window-cache operators and the query/key preparation are measured on.

Three operators of the serving path:

* ``rope``    - per-head RMS norm of queries and keys and their position rotation (one to three axes), one pass;
* ``prefill`` - attention of a ragged batch of prompt chunks with a sliding window and sink tokens, over a ring cache
  (the context) and the chunk itself; a fresh prompt's rows are appended to the cache as well;
* ``decode``  - one token per sequence over the same cache: (norm, rotation,) append and attention.

A token at position p sees the positions j <= p with j < sinks or j > p - window.  A cache has ``sinks + window`` slots
per sequence and head: position j lives in slot j when j < sinks, else in slot sinks + (j - sinks) % window.
"""
import math

import torch

own = False

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6


# ---------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # the token of one sequence in a decode loop: latency
        dict(name="rope_token", op="rope", tokens=1, q_heads=32, k_heads=8, head_dim=128, dtype="bf16", rot=128, axes=1,
             spread=False, adjacent=False, norm=True, far=100000),
        # the packed projections of a long prompt, 40 query heads as in the OPT-13B-shaped workload, grouped keys
        dict(name="rope_prompt", op="rope", tokens=16384, q_heads=40, k_heads=8, head_dim=128, dtype="bf16", rot=128, axes=1,
             spread=False, adjacent=False, norm=True, far=0),
        # image and text tokens with (time, height, width) positions, odd token count, part of the head rotates
        dict(name="rope_axes", op="rope", tokens=5003, q_heads=28, k_heads=4, head_dim=128, dtype="f16", rot=96, axes=3,
             spread=True, adjacent=True, norm=False, far=2500),
        # one short prompt of a small model
        dict(name="prompt_short", op="prefill", lens="33", ctx="0", pad=0, q_heads=8, kv_heads=2, head_dim=64, dtype="f16",
             window=128, sinks=4),
        # a ragged batch of fresh prompts with padding rows behind it
        dict(name="prompt_ragged", op="prefill", lens="1,300,777,2048,0,1023,4001", ctx="0,0,0,0,0,0,0", pad=42, q_heads=32,
             kv_heads=8, head_dim=128, dtype="bf16", window=1024, sinks=4),
        # a long document in one call
        dict(name="prompt_long", op="prefill", lens="32768", ctx="0", pad=0, q_heads=32, kv_heads=8, head_dim=128, dtype="f16",
             window=4096, sinks=16),
        # chunks that continue sequences whose rings have wrapped (or not yet), one key head per query head
        dict(name="chunk_continued", op="prefill", lens="256,256,256,200,256,17,256,256", ctx="9000,2047,2052,100,50001,4100,1,7777",
             pad=0, q_heads=40, kv_heads=40, head_dim=128, dtype="bf16", window=2048, sinks=4),
        # 32-bit rows, head_dim 64
        dict(name="prompt_f32", op="prefill", lens="700,511", ctx="0,0", pad=0, q_heads=16, kv_heads=16, head_dim=64, dtype="f32",
             window=346, sinks=64),
        # one sequence with a long window: few rows, a long axis; the step starts from raw projections
        dict(name="step_one", op="decode", sequences=1, idle=0, ctx_lo=100000, ctx_hi=100000, q_heads=32, kv_heads=8, head_dim=128,
             dtype="bf16", window=16384, sinks=4, rope=True),
        # a serving batch at different lengths, two slots of it idle
        dict(name="step_batch", op="decode", sequences=128, idle=2, ctx_lo=500, ctx_hi=20000, q_heads=32, kv_heads=8, head_dim=128,
             dtype="bf16", window=4096, sinks=4, rope=True),
        # the OPT-66B-shaped batch under a budget of 410 rows per head
        dict(name="step_budget", op="decode", sequences=128, idle=0, ctx_lo=2048, ctx_hi=2048, q_heads=72, kv_heads=72, head_dim=128,
             dtype="f16", window=406, sinks=4, rope=False),
        # a small 32-bit batch, some sequences just begun
        dict(name="step_f32", op="decode", sequences=5, idle=1, ctx_lo=0, ctx_hi=700, q_heads=12, kv_heads=12, head_dim=64, dtype="f32",
             window=126, sinks=2, rope=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "prefill", "decode"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f16", "f32"])
    d = rng.choice([64, 128, 128])
    kv = rng.choice([1, 2, 4, 5, 8, 12, 40])
    g = rng.choice([1, 1, 2, 3, 4, 7, 8]) if kv <= 8 else 1
    if op == "rope":
        axes = rng.choice([1, 3])
        rot = rng.choice([d, d, d // 2, 3 * d // 4])
        return dict(op="rope", tokens=_log_int(rng, 1, 16384), q_heads=kv * g, k_heads=kv, head_dim=d, dtype=dtype, rot=rot, axes=axes,
                    spread=axes == 3 and rng.random() < 0.5, adjacent=rng.random() < 0.4, norm=rng.random() < 0.7,
                    far=_log_int(rng, 1, 1 << 20))
    window, sinks = _log_int(rng, 16, 4096), rng.choice([0, 1, 4, 16, 130])
    if op == "prefill":
        n = _log_int(rng, 1, 12)
        cap = max(1, (2048 if dtype == "f32" else 16384) // (n * max(1, kv * g // 8)))
        lens = [rng.choice([_log_int(rng, 1, cap), _log_int(rng, 1, cap), cap, 0, 1]) for _ in range(n)]
        if sum(lens) == 0:
            lens[0] = 1
        fresh = rng.random() < 0.5
        ctx = [0 if fresh else rng.choice([0, _log_int(rng, 1, 20000), _log_int(rng, 1, 20000)]) for _ in range(n)]
        return dict(op="prefill", lens=",".join(map(str, lens)), ctx=",".join(map(str, ctx)), pad=rng.choice([0, 0, 3, 130]),
                    q_heads=kv * g, kv_heads=kv, head_dim=d, dtype=dtype, window=window, sinks=sinks)
    n = _log_int(rng, 1, 200)
    window = max(16, min(window * 4, (1 << 20) // (n * kv)))
    lo = _log_int(rng, 1, 40000) - 1
    return dict(op="decode", sequences=n, idle=min(n - 1, rng.choice([0, 0, 1, 5])), ctx_lo=lo, ctx_hi=lo + _log_int(rng, 1, 20000) - 1,
                q_heads=kv * g, kv_heads=kv, head_dim=d, dtype=dtype, window=window, sinks=sinks, rope=rng.random() < 0.5)


def _ints(text):
    return [int(x) for x in text.split(",")]


def _contexts(case):
    """Tokens that each sequence of a decode batch holds (-1: an idle slot), spread over [ctx_lo, ctx_hi]."""
    n, span = case["sequences"], case["ctx_hi"] - case["ctx_lo"]
    c = [case["ctx_lo"] + span * ((i * 7919) % n) // max(1, n - 1) if n > 1 else case["ctx_lo"] for i in range(n)]
    for i in range(case["idle"]):
        c[n - 1 - i] = -1
    return c


# ---------------------------------------------------------------------------------------------------- inputs
def _inv_freq(rot):
    return (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().cuda()


def _sections(rot, axes):
    if axes == 1:
        return (rot // 2,)
    third = rot // 2 // 3
    return (rot // 2 - 2 * third, third, third)


def _rope_setup(g, d, dt, rot, axes, spread, adjacent, norm):
    w = lambda: (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(dt)
    sections = _sections(rot, axes)
    return dict(inv_freq=_inv_freq(rot), sections=sections, spread=spread, adjacent=adjacent,
                axis=torch.tensor(_axis_of_pair(sections, spread, rot // 2)).cuda(),
                q_weight=w() if norm else None, k_weight=w() if norm else None)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, d = DT[case["dtype"]], case["head_dim"]
    rnd = lambda *shape, s=1.0: torch.empty(shape, device="cuda", dtype=dt).normal_(0.0, s, generator=g)
    st = dict(case=case)
    if case["op"] == "rope":
        t, hq, hk = case["tokens"], case["q_heads"], case["k_heads"]
        packed = rnd(t, hq + 2 * hk, d, s=2.0)                       # one projection's output: q, k and v heads of a token
        st["q"], st["k"] = packed[:, :hq], packed[:, hq:hq + hk]
        base = torch.arange(t, device="cuda", dtype=torch.int32) + case["far"]
        if case["axes"] == 3:                                       # rows of an image 64 patches wide
            i = torch.arange(t, device="cuda", dtype=torch.int32)
            st["positions"] = torch.stack([base // 1024, (i // 64) % 16 + case["far"], i % 64 + case["far"]]).contiguous()
        else:
            st["positions"] = base
        st.update(_rope_setup(g, d, dt, case["rot"], case["axes"], case["spread"], case["adjacent"], case["norm"]))
        if own:
            st["rope"] = _own_rope(st)
        return st
    hq, hk, w, s = case["q_heads"], case["kv_heads"], case["window"], case["sinks"]
    if case["op"] == "prefill":
        lens, ctx = _ints(case["lens"]), _ints(case["ctx"])
        n, total = len(lens), sum(lens) + case["pad"]
        packed = rnd(total, hq + 2 * hk, d)
        st["q"], st["k"], st["v"] = packed[:, :hq], packed[:, hq:hq + hk], packed[:, hq + hk:]
        starts = [0]
        for x in lens:
            starts.append(starts[-1] + x)
        st.update(lens=lens, ctx=ctx, starts_host=starts)
        st["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
        st["fresh"] = not any(ctx)
        st["lengths"] = torch.tensor(ctx, dtype=torch.int32, device="cuda")
        st["out"] = torch.full((total, hq, d), 7.0, dtype=dt, device="cuda")
    else:
        ctx = _contexts(case)
        n = case["sequences"]
        packed = rnd(n, hq + 2 * hk, d)
        st["q"], st["k"], st["v"] = packed[:, :hq], packed[:, hq:hq + hk], packed[:, hq + hk:]
        st["ctx"] = ctx
        st["lengths"] = torch.tensor(ctx, dtype=torch.int32, device="cuda")
        st["out"] = torch.full((n, hq, d), 7.0, dtype=dt, device="cuda")
        if case["rope"]:
            st.update(_rope_setup(g, d, dt, d, 1, False, False, True))
            if own:
                st["rope"] = _own_rope(st)
    # every slot holds rows, also those that no present token lives in: what an earlier user of the slot left behind
    st["k_cache"], st["v_cache"] = rnd(n, hk, s + w, d), rnd(n, hk, s + w, d)
    return st


# ---------------------------------------------------------------------------------------------------- the framework's calls
def _own_rope(st):
    from paper_2305_17118_b200 import binding as sh
    return sh.Rope(st["inv_freq"], q_weight=st["q_weight"], k_weight=st["k_weight"], eps=EPS, sections=st["sections"],
                   spread=st["spread"], adjacent=st["adjacent"])


def _own_run(st):
    from paper_2305_17118_b200 import binding as sh
    case = st["case"]
    if case["op"] == "rope":
        return sh.qk_norm_rope(st["q"], st["k"], st["positions"], st["rope"])
    win = dict(window=case["window"], sinks=case["sinks"])
    if case["op"] == "decode":
        sh.window_decode(st["q"], st["k"], st["v"], st["lengths"], st["k_cache"], st["v_cache"], rope=st.get("rope"), out=st["out"], **win)
        return st["out"], st["k_cache"], st["v_cache"]
    if st["fresh"]:
        sh.window_prefill(st["q"], st["k"], st["v"], st["starts"], out=st["out"], **win)
        sh.window_append(st["k"], st["v"], st["starts"], st["lengths"], st["k_cache"], st["v_cache"], **win)
        return st["out"], st["k_cache"], st["v_cache"]
    # the append of a continued chunk overwrites ring rows that the same call reads: it is left to the fresh prompts,
    # so that a pass can be repeated on the same inputs
    sh.window_prefill(st["q"], st["k"], st["v"], st["starts"], lengths=st["lengths"], k_cache=st["k_cache"], v_cache=st["v_cache"],
                      out=st["out"], **win)
    return st["out"]


# ---------------------------------------------------------------------------------------------------- the plain form
def _axis_of_pair(sections, spread, pairs):
    """Axis whose position turns each pair: blocks of the sections' sizes, or dealt out in turn (``spread``)."""
    if len(sections) == 1:
        return [0] * pairs
    if spread:
        return [i % 3 if i < 3 * sections[i % 3] else 0 for i in range(pairs)]
    return [0] * sections[0] + [1] * sections[1] + [2] * sections[2]


def _plain_rotate(x, weight, positions, st):
    """fp32 [t, h, d] from 16- or 32-bit rows: norm, then rotation by angles taken in 64 bits."""
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * weight.float()
    pairs = st["inv_freq"].numel()
    pos = positions if positions.dim() == 2 else positions[None]
    ang = (pos[st["axis"]].double() * st["inv_freq"].double()[:, None]).t()
    c, s = ang.cos().float()[:, None], ang.sin().float()[:, None]
    out = y.clone()
    a, b = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if st["adjacent"] else (slice(0, pairs), slice(pairs, 2 * pairs))
    out[..., a] = y[..., a] * c - y[..., b] * s
    out[..., b] = y[..., a] * s + y[..., b] * c
    return out


def _plain_softmax_pv(s, v):
    s = s - s.amax(-1, keepdim=True)
    p = s.exp()
    return torch.matmul(p, v) / p.sum(-1, keepdim=True)


def _slot_positions(length, sinks, window, device):
    """Position held by each slot of a cache with ``length`` tokens [n] (-1: none)."""
    j = torch.arange(window, device=device)
    c = length[:, None] - sinks                                     # tokens in the ring so far
    ring = torch.where(c > j, j + (c - 1 - j).clamp(min=0) // window * window + sinks, -1)
    s = torch.arange(sinks, device=device).expand(length.shape[0], -1)
    return torch.cat([torch.where(s < length[:, None], s, -1), ring], 1)


def _plain_prefill(st):
    case = st["case"]
    w, s, hk = case["window"], case["sinks"], case["kv_heads"]
    g, d = case["q_heads"] // hk, case["head_dim"]
    dev = st["q"].device
    for i, n in enumerate(st["lens"]):
        if n == 0:
            continue
        r0, c = st["starts_host"][i], st["ctx"][i]
        k, v = st["k"][r0:r0 + n].float().transpose(0, 1), st["v"][r0:r0 + n].float().transpose(0, 1)
        kp = torch.arange(c, c + n, device=dev)
        if c:
            sp = _slot_positions(torch.full((1,), c, device=dev, dtype=torch.int64), s, w, dev)[0]
            live = min(c, s + w)                                     # live slots are the first ones until the ring wraps
            k, v = torch.cat([st["k_cache"][i, :, :live].float(), k], 1), torch.cat([st["v_cache"][i, :, :live].float(), v], 1)
            kp = torch.cat([sp[:live], kp])
        m = min(c, s + w)
        for a in range(0, n, 512):                                   # blocks of queries against the keys that one of them can see
            b = min(n, a + 512)
            lo = m + max(0, a - w + 1)                               # (the context's live slots stay whole)
            head = max(m, min(lo, s))                                # earlier rows of a fresh prompt: its sinks
            if lo <= head or c:
                ks, vs, ps = k[:, :m + b], v[:, :m + b], kp[:m + b]
            else:
                ks, vs = (torch.cat([x[:, :head], x[:, lo:b]], 1) for x in (k, v))
                ps = torch.cat([kp[:head], kp[lo:b]])
            q = st["q"][r0 + a:r0 + b].float().view(b - a, hk, g, d).permute(1, 2, 0, 3)
            qp = torch.arange(c + a, c + b, device=dev)[:, None]
            vis = (ps <= qp) & ((ps < s) | (ps > qp - w))
            sc = torch.matmul(q, ks[:, None].transpose(-1, -2)) * d ** -0.5
            sc = sc.masked_fill(~vis, -math.inf)
            o = _plain_softmax_pv(sc, vs[:, None])
            st["out"][r0 + a:r0 + b] = o.permute(2, 0, 1, 3).reshape(b - a, hk * g, d).to(st["out"].dtype)
    if not st["fresh"]:
        return st["out"]
    for i, n in enumerate(st["lens"]):
        r0 = st["starts_host"][i]
        new = st["k"][r0:r0 + n].transpose(0, 1), st["v"][r0:r0 + n].transpose(0, 1)
        first = max(s, n - w)
        slots = (torch.arange(first, max(first, n), device=dev) - s) % w + s
        for cache, rows in zip((st["k_cache"], st["v_cache"]), new):
            cache[i, :, :min(s, n)] = rows[:, :s]
            if n > first:
                cache[i, :, slots] = rows[:, first:]
    return st["out"], st["k_cache"], st["v_cache"]


def _plain_decode(st):
    case = st["case"]
    w, s, hk = case["window"], case["sinks"], case["kv_heads"]
    g, d = case["q_heads"] // hk, case["head_dim"]
    n = st["lengths"].shape[0]
    length = st["lengths"].long()
    active = length >= 0
    q, k = st["q"].float(), st["k"].float()
    if case["rope"]:
        pos = st["lengths"].clamp(min=0)
        q, k = _plain_rotate(st["q"], st["q_weight"], pos, st), _plain_rotate(st["k"], st["k_weight"], pos, st)
    slot = torch.where(length < s, length, s + (length - s) % w).clamp(min=0)
    rows = torch.arange(n, device=slot.device)
    for cache, new in ((st["k_cache"], k), (st["v_cache"], st["v"])):
        cache[rows, :, slot] = torch.where(active[:, None, None], new.to(cache.dtype), cache[rows, :, slot])
    sp = _slot_positions((length + 1).clamp(min=0), s, w, slot.device)
    vis = sp >= 0
    sc = torch.matmul(q.view(n, hk, g, d), st["k_cache"].float().transpose(-1, -2)) * d ** -0.5
    sc = sc.masked_fill(~vis[:, None, None], -math.inf)
    o = _plain_softmax_pv(sc, st["v_cache"].float()).reshape(n, hk * g, d).to(st["out"].dtype)
    st["out"].copy_(torch.where(active[:, None, None], o, st["out"]))
    return st["out"], st["k_cache"], st["v_cache"]


def run(state):
    if own:
        return _own_run(state)
    case = state["case"]
    if case["op"] == "rope":
        f = lambda x, w: _plain_rotate(x, w, state["positions"], state).to(x.dtype)
        return f(state["q"], state["q_weight"]), f(state["k"], state["k_weight"])
    return _plain_prefill(state) if case["op"] == "prefill" else _plain_decode(state)


# ---------------------------------------------------------------------------------------------------- the cost
def _visible_pairs(n, c, w, s):
    """Visible (query, key) pairs of n queries at positions c .. c + n - 1."""
    full = lambda p: min(p + 1, w) + min(s, max(0, p + 1 - w))
    ramp = min(max(0, w + s - c), n)                                 # positions below w + s are counted one by one
    return sum(full(c + i) for i in range(ramp)) + (n - ramp) * (w + s)


def work(case):
    es, d = DT[case["dtype"]].itemsize, case["head_dim"]
    if case["op"] == "rope":
        rows = case["tokens"] * (case["q_heads"] + case["k_heads"])
        return {"bytes": 2 * rows * d * es + 4 * case["tokens"] * case["axes"], "flops": rows * (4 * d * case["norm"] + 3 * case["rot"])}
    hq, hk, w, s = case["q_heads"], case["kv_heads"], case["window"], case["sinks"]
    if case["op"] == "decode":
        ctx = [c for c in _contexts(case) if c >= 0]
        keys = sum(min(c + 1, w) + min(s, max(0, c + 1 - w)) for c in ctx)
        return {"bytes": (2 * keys * hk + len(ctx) * (2 * hq + 2 * hk)) * d * es, "flops": 4 * d * hq * keys}
    lens, ctx = _ints(case["lens"]), _ints(case["ctx"])
    pairs, rows = 0, 0
    for n, c in zip(lens, ctx):
        if n == 0:
            continue
        pairs += _visible_pairs(n, c, w, s)
        ring = max(0, c - max(s, c - w + 1))                         # context rows in the first query's window, and the sinks
        rows += n * (2 * hq + 2 * hk) + 2 * hk * (ring + min(s, c))
        if not any(ctx):
            rows += 2 * hk * (min(n, s) + min(max(0, n - s), w))     # the rows appended to the cache
    return {"bytes": rows * d * es, "flops": 4 * d * hq * pairs}


# ---------------------------------------------------------------------------------------------------- the definition in 64 bits
def _exact_turn(x, weight, positions, st):
    y = x.double()
    if weight is not None:
        y = y / ((y ** 2).sum(-1, keepdim=True) / y.shape[-1] + EPS) ** 0.5 * weight.double()
    f = st["inv_freq"].double()
    pairs = len(f)
    if positions.dim() == 1:
        positions = positions.expand(3, -1)
    sec = st["sections"]
    out = y.clone()
    for i in range(pairs):
        if len(sec) == 1:
            ax = 0
        elif st["spread"]:
            ax = i % 3 if i < 3 * sec[i % 3] else 0
        else:
            ax = 0 if i < sec[0] else 1 if i < sec[0] + sec[1] else 2
        z = torch.polar(torch.ones_like(positions[ax], dtype=torch.float64), positions[ax].double() * f[i])[:, None]
        a, b = (2 * i, 2 * i + 1) if st["adjacent"] else (i, i + pairs)
        r = torch.complex(y[..., a], y[..., b]) * z
        out[..., a], out[..., b] = r.real, r.imag
    return out


def _exact_attend(q, qpos, keys, vals, kpos, w, s):
    """q [t, hq, d], keys and vals [hk, m, d] in 64 bits; kpos[m] (-1: no token)."""
    t, hq, d = q.shape
    g = hq // keys.shape[0]
    out = torch.empty_like(q)
    see = (kpos[None] >= 0) & (kpos[None] <= qpos[:, None]) & ((kpos[None] < s) | (qpos[:, None] - kpos[None] < w))
    for h in range(hq):
        logit = (q[:, h] @ keys[h // g].t()) / math.sqrt(d)
        logit = torch.where(see, logit, torch.full_like(logit, -math.inf))
        out[:, h] = torch.exp(logit - torch.logsumexp(logit, 1, keepdim=True)) @ vals[h // g]
    return out


def exact(case, seed):
    if work(case)["flops"] > 4e12:
        return None
    st = prepare(case, seed)
    if case["op"] == "rope":
        return (_exact_turn(st["q"], st["q_weight"], st["positions"], st), _exact_turn(st["k"], st["k_weight"], st["positions"], st))
    w, s = case["window"], case["sinks"]
    out, kc, vc = st["out"].double(), st["k_cache"].double(), st["v_cache"].double()
    where = lambda p: p if p < s else s + (p - s) % w
    q, k, v = st["q"].double(), st["k"].double(), st["v"].double()
    if case["op"] == "decode":
        if case["rope"]:
            pos = st["lengths"].clamp(min=0)
            q, k = _exact_turn(st["q"], st["q_weight"], pos, st), _exact_turn(st["k"], st["k_weight"], pos, st)
        for i, c in enumerate(st["ctx"]):
            if c < 0:
                continue
            kc[i, :, where(c)], vc[i, :, where(c)] = k[i], v[i]
            held = torch.full((s + w,), -1, dtype=torch.int64)
            first = max(s, c + 1 - w)
            old = torch.cat([torch.arange(0, min(s, c + 1)), torch.arange(first, max(first, c + 1))])
            held[torch.where(old < s, old, s + (old - s) % w)] = old
            held = held.to(q.device)
            out[i] = _exact_attend(q[i:i + 1], torch.tensor([c], device=q.device), kc[i], vc[i], held, w, s)[0]
        return out, kc, vc
    for i, (n, c) in enumerate(zip(st["lens"], st["ctx"])):
        r0 = st["starts_host"][i]
        held = torch.cat([torch.arange(0, min(s, c)), torch.arange(max(s, c - w), max(s, c - w, c))]).to(q.device)
        at = torch.where(held < s, held, s + (held - s) % w)
        for a in range(0, n, 1024):
            b = min(n, a + 1024)
            new = torch.arange(a, b, device=q.device) + c
            j0 = max(0, a - w + 1)                                   # earlier tokens of the chunk: out of every window here,
            js = torch.cat([torch.arange(0, min(j0, max(0, s - c))), torch.arange(j0, b)]).to(q.device)      # but for the sinks
            keys = torch.cat([kc[i][:, at], k[r0 + js].transpose(0, 1)], 1)
            vals = torch.cat([vc[i][:, at], v[r0 + js].transpose(0, 1)], 1)
            out[r0 + a:r0 + b] = _exact_attend(q[r0 + a:r0 + b], new, keys, vals, torch.cat([held, js + c]), w, s)
    if not st["fresh"]:
        return out
    for i, n in enumerate(st["lens"]):
        r0 = st["starts_host"][i]
        keep = torch.cat([torch.arange(0, min(s, n)), torch.arange(max(s, n - w), max(s, n - w, n))]).to(q.device)
        to = torch.where(keep < s, keep, s + (keep - s) % w)
        kc[i][:, to], vc[i][:, to] = k[r0 + keep].transpose(0, 1), v[r0 + keep].transpose(0, 1)
    return out, kc, vc
