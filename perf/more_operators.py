"""What shared contexts and the cache with accumulated weights are measured on.

Four operators of the serving path:

* ``context`` - attention of tokens to a context that they share and that is complete: a prefix that a whole batch has in common, or each
  sequence's own encoder states (cross attention).  Every token of context i sees its ``lengths[i]`` rows.
* ``prompt``  - prompt chunks over a cache that keeps, for every row, the attention weight it has received so far (its mass): the chunk is
  stored, attends causally over the cache and itself, and every row's mass grows by the weights that the chunk's tokens give it.
* ``step``    - the same for one token per sequence.  Where a batch also shares a prefix, the softmax goes over both: the prefix is attended
  to for all sequences at once, and the step continues from that result.
* ``evict``   - of each (sequence, key head), keep the rows with the largest mass and the newest ones, in place or into a smaller cache.

A mass row is added up over the query heads that share a key head.  Slots 0 .. lengths[i] - 1 of a cache are live, in any order.
"""
import math

import torch

own = False

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # one decoder token of a few sequences over their encoder states: latency
        dict(name="cross_tokens", op="context", contexts=3, counts="1,1,1", rows=700, lo=33, hi=700, q_heads=8, kv_heads=8, head_dim=64,
             dtype="f16"),
        # a decoding batch, every sequence over its own encoder states, as many key heads as query heads
        dict(name="cross_batch", op="context", contexts=128, counts="1", rows=1500, lo=200, hi=1500, q_heads=20, kv_heads=20, head_dim=64,
             dtype="bf16"),
        # decoder prompts over encoder states of another length, one sequence without tokens and one without states
        dict(name="cross_prompts", op="context", contexts=7, counts="448,1,200,0,333,511,97", rows=1500, lo=0, hi=1500, q_heads=16,
             kv_heads=16, head_dim=64, dtype="f16"),
        # a batch that shares a long system prompt, grouped heads
        dict(name="prefix_batch", op="context", contexts=1, counts="256", rows=16384, lo=16001, hi=16001, q_heads=32, kv_heads=8,
             head_dim=128, dtype="bf16"),
        # the first tokens of a small 32-bit batch
        dict(name="step_f32", op="step", sequences=5, idle=1, lo=0, hi=120, slots=130, q_heads=12, kv_heads=12, head_dim=64, dtype="f32",
             prefix=0),
        # the OPT-66B-shaped batch under a budget of 410 rows and the 64 tokens that come in between two evictions
        dict(name="step_budget", op="step", sequences=128, idle=0, lo=410, hi=473, slots=474, q_heads=72, kv_heads=72, head_dim=128,
             dtype="f16", prefix=0),
        # a long budget, grouped heads, sequences of different lengths that continue one shared prefix
        dict(name="step_shared", op="step", sequences=64, idle=2, lo=100, hi=4090, slots=4096, q_heads=32, kv_heads=8, head_dim=128,
             dtype="bf16", prefix=5000),
        # a ragged batch of fresh prompts
        dict(name="prompt_ragged", op="prompt", counts="1,300,777,2048,0,1023", held="0,0,0,0,0,0", slots=2048, q_heads=32, kv_heads=8,
             head_dim=128, dtype="bf16"),
        # a long document in one call
        dict(name="prompt_long", op="prompt", counts="16384", held="0", slots=16500, q_heads=32, kv_heads=8, head_dim=128, dtype="f16"),
        # chunks that continue 32-bit caches
        dict(name="chunk_f32", op="prompt", counts="64,17,200", held="500,0,31", slots=600, q_heads=12, kv_heads=12, head_dim=64, dtype="f32"),
        # prompts brought down to a budget, into the cache that decoding uses
        dict(name="evict_prompts", op="evict", sequences=8, lo=1500, hi=32768, slots=32768, keep=2048, recent=256, into=True, kv_heads=8,
             head_dim=128, dtype="bf16"),
        # the OPT-66B-shaped batch when its 64 spare slots have filled up
        dict(name="evict_steps", op="evict", sequences=128, lo=474, hi=474, slots=474, keep=410, recent=64, into=False, kv_heads=72,
             head_dim=128, dtype="f16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["context", "context", "step", "step", "prompt", "evict"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f16", "f32"])
    d = rng.choice([64, 128, 128])
    kv = rng.choice([1, 2, 4, 5, 8, 12, 40])
    g = rng.choice([1, 1, 2, 3, 4, 7, 8, 16]) if kv <= 8 else 1
    heads = dict(q_heads=kv * g, kv_heads=kv, head_dim=d, dtype=dtype)
    if op == "context":
        rows = _log_int(rng, 1, 20000)
        if rng.random() < 0.5:                                       # one token of each sequence, or a batch that shares a prefix
            n = max(1, min(_log_int(rng, 1, 256), (1 << 22) // (rows * kv)))
            return dict(op=op, contexts=n, counts="1", rows=rows, lo=_log_int(rng, 1, rows), hi=rows, **heads)
        n = _log_int(rng, 1, 8)
        cap = max(1, min(4000, (1 << (24 if dtype == "f32" else 27)) // (n * rows * max(1, kv * g // 8))))
        counts = [rng.choice([_log_int(rng, 1, cap), _log_int(rng, 1, cap), 0, 1]) for _ in range(n)]
        if sum(counts) < 2:
            counts[0] = 2
        return dict(op=op, contexts=n, counts=",".join(map(str, counts)), rows=rows, lo=rng.choice([0, 1, _log_int(rng, 1, rows)]), hi=rows, **heads)
    if op == "step":
        n = _log_int(rng, 1, 200)
        slots = max(2, min(_log_int(rng, 16, 16000), (1 << 22) // (n * kv)))
        lo = _log_int(rng, 1, slots) - 1
        return dict(op=op, sequences=n, idle=min(n - 1, rng.choice([0, 0, 1, 5])), lo=lo, hi=rng.randint(lo, slots - 1), slots=slots,
                    prefix=rng.choice([0, 0, min(_log_int(rng, 1, 8000), (1 << 22) // (n * kv))]), **heads)
    if op == "prompt":
        n = _log_int(rng, 1, 8)
        cap = max(2, (1024 if dtype == "f32" else 8192) // (n * max(1, kv * g // 8)))
        counts = [rng.choice([_log_int(rng, 1, cap), _log_int(rng, 1, cap), cap, 0, 1]) for _ in range(n)]
        if sum(counts) == 0:
            counts[0] = 2
        fresh = rng.random() < 0.5
        held = [0 if fresh else rng.choice([0, _log_int(rng, 1, 4000)]) for _ in range(n)]
        return dict(op=op, counts=",".join(map(str, counts)), held=",".join(map(str, held)),
                    slots=max(a + b for a, b in zip(counts, held)) + rng.choice([0, 1, 77]), **heads)
    heads.pop("q_heads")
    n = _log_int(rng, 1, 128)
    slots = max(8, min(_log_int(rng, 8, 32768), (1 << 22) // (n * kv)))
    keep = max(1, min(slots - 1, _log_int(rng, 1, slots)))
    return dict(op="evict", sequences=n, lo=_log_int(rng, 1, slots) - 1, hi=slots, slots=slots, keep=keep,
                recent=rng.choice([0, min(keep, 1), keep // 4, keep]), into=rng.random() < 0.5, **heads)


def _ints(text):
    return [int(x) for x in text.split(",")]


def _spread(n, lo, hi):
    """n lengths over [lo, hi], in no order."""
    return [lo + (hi - lo) * ((i * 7919) % n) // (n - 1) if n > 1 else hi for i in range(n)]


def _counts(case):
    """Tokens of each context."""
    counts = _ints(case["counts"])
    return counts * case["contexts"] if len(counts) == 1 and case["contexts"] > 1 else counts


def _held(case):
    """Live rows of each sequence of a step (-1: an idle slot of the batch)."""
    held = _spread(case["sequences"], case["lo"], case["hi"])
    return held[:len(held) - case["idle"]] + [-1] * case["idle"]


# ---------------------------------------------------------------------------------------------------- inputs
def _starts(counts):
    starts = [0]
    for x in counts:
        starts.append(starts[-1] + x)
    return starts


def _ints_on_gpu(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, d, hk = DT[case["dtype"]], case["head_dim"], case["kv_heads"]
    rnd = lambda *shape: torch.empty(shape, device="cuda", dtype=dt).normal_(0.0, 1.0, generator=g)
    st = dict(case=case)
    if case["op"] == "context":
        counts, n = _counts(case), case["contexts"]
        hq, total = case["q_heads"], sum(counts)
        st["counts"], st["each"] = counts, counts == [1] * n
        st["q"] = rnd(total, hq, d)
        st["k"], st["v"] = rnd(n, hk, case["rows"], d), rnd(n, hk, case["rows"], d)
        st["lengths"] = _ints_on_gpu(_spread(n, case["lo"], case["hi"]))
        st["starts"] = _ints_on_gpu(_starts(counts))
        return st
    if case["op"] == "evict":
        n, slots = case["sequences"], case["slots"]
        st["k"], st["v"] = rnd(n, hk, slots, d), rnd(n, hk, slots, d)
        st["lengths"] = _ints_on_gpu(_spread(n, case["lo"], case["hi"]))
        # what rows have received so far: a few much, most of them little, some the same
        heavy = torch.empty(n, hk, slots, device="cuda").normal_(0.0, 2.0, generator=g).exp()
        st["mass_now"] = (heavy * 64).floor() / 64
        # the rows that survived earlier evictions in some order, behind them the tokens that have come since
        order = torch.rand(n, hk, slots, device="cuda", generator=g).argsort(-1)
        late = torch.arange(slots, device="cuda")
        st["positions_now"] = torch.where(late < case["keep"], order, late + slots).to(torch.int32)
        st["mass"], st["positions"] = st["mass_now"].clone(), st["positions_now"].clone()
        if case["into"]:
            st["into"] = (rnd(n, hk, case["keep"], d), rnd(n, hk, case["keep"], d), torch.zeros(n, hk, case["keep"], device="cuda"),
                          torch.zeros(n, hk, case["keep"], dtype=torch.int32, device="cuda"))
        return st
    hq, slots = case["q_heads"], case["slots"]
    if case["op"] == "step":
        held = _held(case)
        n = total = case["sequences"]
        if case["prefix"]:
            st["prefix_k"], st["prefix_v"] = rnd(1, hk, case["prefix"], d), rnd(1, hk, case["prefix"], d)
    else:
        counts, held = _ints(case["counts"]), _ints(case["held"])
        n, total = len(counts), sum(counts)
        st["counts"], st["starts"] = counts, _ints_on_gpu(_starts(counts))
    packed = rnd(total, hq + 2 * hk, d)                              # one projection's output: q, k and v heads of a token
    st["q"], st["k"], st["v"] = packed[:, :hq], packed[:, hq:hq + hk], packed[:, hq + hk:]
    st["held"] = held
    st["lengths"] = _ints_on_gpu(held)
    st["seen"] = st["lengths"].clamp(min=0) * 3 + 7                  # tokens so far: most of them were evicted
    # every slot holds something, also those that no row lives in: what an earlier user of the slot left behind
    st["k_cache"], st["v_cache"] = rnd(n, hk, slots, d), rnd(n, hk, slots, d)
    st["mass"] = torch.empty(n, hk, slots, device="cuda").normal_(0.0, 1.0, generator=g).exp()
    st["positions"] = torch.arange(slots, dtype=torch.int32, device="cuda").expand(n, hk, slots).contiguous()
    st["out"] = torch.full((total, hq, d), 7.0, dtype=dt, device="cuda")
    return st


# ---------------------------------------------------------------------------------------------------- the framework's calls
def _own_run(st):
    from paper_2305_17118_b200 import binding as sh
    case = st["case"]
    if case["op"] == "context":
        return sh.context_attention(st["q"], st["k"], st["v"], None if st["each"] or len(st["counts"]) == 1 else st["starts"], st["lengths"])
    if case["op"] == "evict":
        if case["into"]:
            return (sh.mass_evict(st["k"], st["v"], st["mass"], st["positions"], st["lengths"], keep=case["keep"], recent=case["recent"],
                                  into=st["into"]), *st["into"])
        st["mass"].copy_(st["mass_now"])                             # the records as they are when the spare slots have filled up again
        st["positions"].copy_(st["positions_now"])
        left = sh.mass_evict(st["k"], st["v"], st["mass"], st["positions"], st["lengths"], keep=case["keep"], recent=case["recent"])
        return left, st["k"], st["v"], st["mass"], st["positions"]
    if case["op"] == "step":
        prior = sh.context_attention(st["q"], st["prefix_k"], st["prefix_v"], partial=True) if case["prefix"] else None
        sh.mass_decode(st["q"], st["k"], st["v"], st["lengths"], st["k_cache"], st["v_cache"], st["mass"], st["positions"], st["seen"],
                       prior=prior, out=st["out"])
    else:
        sh.mass_prefill(st["q"], st["k"], st["v"], st["starts"], st["lengths"], st["k_cache"], st["v_cache"], st["mass"], st["positions"],
                        st["seen"], out=st["out"])
    return st["out"], st["k_cache"], st["v_cache"], st["mass"], st["positions"]


# ---------------------------------------------------------------------------------------------------- the plain form
def _padded(x, counts):
    """Rows [tokens, heads, d] as [sequences, heads, longest, d] in fp32, and the (sequence, place) of each token."""
    seq = torch.repeat_interleave(torch.arange(len(counts), device=x.device), torch.tensor(counts, device=x.device))
    first = torch.tensor(_starts(counts)[:-1], device=x.device)
    place = torch.arange(x.shape[0], device=x.device) - first[seq]
    y = torch.zeros(len(counts), x.shape[1], max(counts), x.shape[2], device=x.device)
    y[seq, :, place] = x.float()
    return y, seq, place


def _plain_context(st):
    case = st["case"]
    n, hk, d = case["contexts"], case["kv_heads"], case["head_dim"]
    q, seq, place = _padded(st["q"], st["counts"])
    g, longest = q.shape[1] // hk, q.shape[2]
    s = torch.matmul(q.reshape(n, hk, g * longest, d), st["k"].float().transpose(-1, -2)) * d ** -0.5
    live = torch.arange(case["rows"], device=s.device) < st["lengths"][:, None]
    s.masked_fill_(~live[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True).clamp(min=-3e38)                  # (a context without rows)
    p = (s - top).exp()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, torch.where(live[:, None, :, None], st["v"].float(), 0.0)) / total.clamp(min=1e-37)
    lse = total.log() + top
    return o.view(n, hk * g, longest, d)[seq, :, place].to(st["q"].dtype), lse.view(n, hk * g, longest)[seq, :, place]


def _plain_step(st):
    case = st["case"]
    n, hk, d, slots = case["sequences"], case["kv_heads"], case["head_dim"], case["slots"]
    hq = case["q_heads"]
    active = st["lengths"] >= 0
    rows, at = torch.arange(n, device=st["q"].device)[active], st["lengths"][active].long()
    for cache, new in ((st["k_cache"], st["k"]), (st["v_cache"], st["v"])):
        cache[rows, :, at] = new[rows]
    st["positions"][rows, :, at] = st["seen"][rows, None]
    st["mass"][rows, :, at] = 0.0
    q = st["q"].float().view(n, hk, hq // hk, d)
    s = torch.matmul(q, st["k_cache"].float().transpose(-1, -2)) * d ** -0.5
    live = (torch.arange(slots, device=s.device) <= st["lengths"][:, None])[:, None, None]
    s = s.masked_fill(~live, -math.inf)
    v = st["v_cache"].float()
    if case["prefix"]:
        s = torch.cat([s, torch.matmul(q, st["prefix_k"].float().transpose(-1, -2)) * d ** -0.5], -1)
        v = torch.cat([v, st["prefix_v"].float().expand(n, -1, -1, -1)], 2)
    p = (s - s.amax(-1, keepdim=True).clamp(min=-3e38)).exp()
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-37)
    o = torch.matmul(p, v).view(n, hq, d).to(st["out"].dtype)
    st["out"].copy_(torch.where(active[:, None, None], o, st["out"]))
    st["mass"].add_(torch.where(live[:, :, 0], p[..., :slots].sum(2), 0.0))
    return st["out"], st["k_cache"], st["v_cache"], st["mass"], st["positions"]


def _plain_prompt(st):
    case = st["case"]
    hk, d, slots, counts = case["kv_heads"], case["head_dim"], case["slots"], st["counts"]
    g, n = case["q_heads"] // hk, len(counts)
    q, seq, place = _padded(st["q"], counts)
    longest = q.shape[2]
    held = st["lengths"].long()
    at = held[seq] + place
    for cache, new in ((st["k_cache"], st["k"]), (st["v_cache"], st["v"])):
        cache[seq, :, at] = new
    st["positions"][seq, :, at] = (st["seen"][seq] + place.to(torch.int32))[:, None]
    st["mass"][seq, :, at] = 0.0
    span = max(a + b for a, b in zip(counts, st["held"]))            # no sequence has rows behind it
    token, count = torch.arange(longest, device=q.device), torch.tensor(counts, device=q.device)
    sees = torch.arange(span, device=q.device) <= (held[:, None] + token)[..., None]
    for h in range(hk):                                              # a key head at a time: all scores together would not fit
        s = torch.matmul(q[:, h * g:(h + 1) * g], st["k_cache"][:, h, None, :span].float().transpose(-1, -2)) * d ** -0.5
        s.masked_fill_(~sees[:, None], -math.inf)
        p = s.sub_(s.amax(-1, keepdim=True)).exp_()
        p.div_(p.sum(-1, keepdim=True))
        o = torch.matmul(p, st["v_cache"][:, h, None, :span].float())
        st["out"][:, h * g:(h + 1) * g] = o[seq, :, place].to(st["out"].dtype)
        p.mul_((token < count[:, None])[:, None, :, None])
        st["mass"][:, h, :span] += p.sum((1, 2))
    return st["out"], st["k_cache"], st["v_cache"], st["mass"], st["positions"]


def _take(x, idx):
    return torch.gather(x, 2, idx[..., None].expand(-1, -1, -1, x.shape[3])) if x.dim() == 4 else torch.gather(x, 2, idx)


def _plain_evict(st):
    case = st["case"]
    slots, keep = case["slots"], case["keep"]
    if not case["into"]:
        st["mass"].copy_(st["mass_now"])
        st["positions"].copy_(st["positions_now"])
    slot = torch.arange(slots, device=st["k"].device).expand_as(st["mass"])
    live = slot < st["lengths"][:, None, None]
    pos = torch.where(live, st["positions"], -1)
    worth = torch.where(pos > pos.amax(-1, keepdim=True) - case["recent"], math.inf, st["mass"]).masked_fill_(~live, -math.inf)
    order = torch.sort(worth, dim=-1, descending=True, stable=True).indices      # among equal ones the lowest slot first
    stays = torch.zeros_like(live).scatter_(2, order[..., :keep], True) & live
    left = st["lengths"].clamp(max=keep)
    if case["into"]:
        idx = torch.where(stays, slot, slots).sort(-1).values[..., :keep]
        there = idx < slots
        for src, dst in zip((st["k"], st["v"], st["mass"], st["positions"]), st["into"]):
            new = _take(src, idx.clamp(max=slots - 1))
            dst.copy_(torch.where(there[..., None] if dst.dim() == 4 else there, new, dst))
        return left, *st["into"]
    most = min(keep, slots - keep)
    hole = torch.where(~stays & live, slot, slots)[..., :keep].sort(-1).values[..., :most]
    move = torch.where(stays, slot, slots)[..., keep:].sort(-1).values[..., :most]
    real = (hole < slots) & (move < slots)
    hole, move = torch.where(real, hole, 0), torch.where(real, move, 0)
    seq, head, i = real.nonzero(as_tuple=True)
    for x in (st["k"], st["v"], st["mass"], st["positions"]):
        x[seq, head, hole[seq, head, i]] = x[seq, head, move[seq, head, i]]
    return left, st["k"], st["v"], st["mass"], st["positions"]


def run(state):
    if own:
        return _own_run(state)
    return {"context": _plain_context, "step": _plain_step, "prompt": _plain_prompt, "evict": _plain_evict}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------------- the cost
def work(case):
    es, d, hk = DT[case["dtype"]].itemsize, case["head_dim"], case["kv_heads"]
    if case["op"] == "context":
        counts, lengths = _counts(case), _spread(case["contexts"], case["lo"], case["hi"])
        pairs = sum(a * b for a, b in zip(counts, lengths))
        rows = 2 * hk * sum(b for a, b in zip(counts, lengths) if a)
        return {"bytes": (rows + 2 * case["q_heads"] * sum(counts)) * d * es + 4 * case["q_heads"] * sum(counts), "flops": 4 * d * case["q_heads"] * pairs}
    if case["op"] == "evict":
        lengths = _spread(case["sequences"], case["lo"], case["hi"])
        moved = sum(min(n, case["keep"]) if case["into"] else min(max(0, n - case["keep"]), case["keep"]) for n in lengths)
        return {"bytes": hk * (8 * sum(lengths) + moved * (4 * d * es + 8)), "flops": 0}
    if case["op"] == "step":
        held = [c for c in _held(case) if c >= 0]
        new, keys, pairs = len(held), sum(held), sum(held) + len(held) * (1 + case["prefix"])
        rows = 2 * hk * (keys + 2 * new + (case["prefix"] if new else 0))
    else:
        counts, held = _ints(case["counts"]), _ints(case["held"])
        new = sum(counts)
        keys = sum(b for a, b in zip(counts, held) if a)
        pairs = sum(a * b + a * (a + 1) // 2 for a, b in zip(counts, held))
        rows = 2 * hk * (keys + 2 * new)
    # keys and values of the cache are read, the new ones read and stored, queries read, outputs written, masses read and written
    return {"bytes": (rows + 2 * case["q_heads"] * new) * d * es + hk * (8 * keys + 8 * new), "flops": 4 * d * case["q_heads"] * pairs}


# ---------------------------------------------------------------------------------------------------- the definition in 64 bits
def _exact_attend(q, keys, vals, sees=None):
    """q [t, d] over keys and vals [m, d] in 64 bits: (outputs [t, d], log of the sum of exponentials [t], weights [t, m])."""
    logit = q @ keys.t() / math.sqrt(q.shape[1])
    if sees is not None:
        logit = torch.where(sees, logit, torch.full_like(logit, -math.inf))
    lse = torch.logsumexp(logit, 1)
    w = torch.exp(logit - lse[:, None])
    return w @ vals, lse, w


def exact(case, seed):
    w = work(case)
    if w["flops"] > 4e12:
        return None
    st = prepare(case, seed)
    if case["op"] == "evict":
        return _exact_evict(st)
    g = case["q_heads"] // case["kv_heads"]
    q, k, v = st["q"].double(), st["k"], st["v"]
    if case["op"] == "context":
        out, lse = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
        a = 0
        for i, (count, length) in enumerate(zip(st["counts"], st["lengths"].tolist())):
            for h in range(case["q_heads"] if length > 0 and count > 0 else 0):
                out[a:a + count, h], lse[a:a + count, h], _ = _exact_attend(q[a:a + count, h], k[i, h // g, :length].double(), v[i, h // g, :length].double())
            a += count
        return out, lse
    out, kc, vc, mass, positions = st["out"].double(), st["k_cache"].double(), st["v_cache"].double(), st["mass"].double(), st["positions"]
    counts = [1] * case["sequences"] if case["op"] == "step" else st["counts"]
    prefix = case.get("prefix", 0)
    a = 0
    for i, (count, held) in enumerate(zip(counts, st["held"])):
        if held >= 0 and count:
            end, dev = held + count, q.device
            kc[i, :, held:end], vc[i, :, held:end] = k[a:a + count].transpose(0, 1).double(), v[a:a + count].transpose(0, 1).double()
            positions[i, :, held:end] = int(st["seen"][i]) + torch.arange(count, dtype=torch.int32, device=dev)
            mass[i, :, held:end] = 0
            sees = torch.arange(end, device=dev)[None] <= torch.arange(held, end, device=dev)[:, None]
            if prefix:
                sees = torch.cat([sees, torch.ones(count, prefix, dtype=torch.bool, device=dev)], 1)
            for h in range(case["q_heads"]):
                keys, vals = kc[i, h // g, :end], vc[i, h // g, :end]
                if prefix:
                    keys, vals = torch.cat([keys, st["prefix_k"][0, h // g].double()]), torch.cat([vals, st["prefix_v"][0, h // g].double()])
                out[a:a + count, h], _, weights = _exact_attend(q[a:a + count, h], keys, vals, sees)
                mass[i, h // g, :end] += weights[:, :end].sum(0)
        a += count
    return out, kc, vc, mass, positions


def _exact_evict(st):
    """Counted row by row instead of sorted: a row stays if fewer than `keep` rows go before it."""
    case = st["case"]
    keep, recent = case["keep"], case["recent"]
    k, v, mass, pos = st["k"], st["v"], st["mass"], st["positions"]
    if case["sequences"] * case["kv_heads"] > 1500 and case["slots"] > 2000:
        return None
    lengths = st["lengths"].tolist()
    left = torch.tensor([min(n, keep) for n in lengths], dtype=torch.int32, device=k.device)
    for i, n in enumerate(lengths):
        for h in range(case["kv_heads"]) if n > 0 else []:
            m, p = mass[i, h, :n].double(), pos[i, h, :n].long()
            new = p > int(p.max()) - recent
            m = torch.where(new, torch.full_like(m, math.inf), m)
            up, inverse, many = torch.unique(m, return_inverse=True, return_counts=True)
            heavier = (many.flip(0).cumsum(0).flip(0) - many)[inverse]
            before = torch.zeros(n, dtype=torch.int64, device=k.device)
            by = torch.argsort(inverse * n + torch.arange(n, device=k.device))
            group = inverse[by]
            before[by] = torch.arange(n, device=k.device) - (many.cumsum(0) - many)[group]
            stays = heavier + before < keep
            kept = stays.nonzero()[:, 0]
            if case["into"]:
                for src, dst in zip((k, v, mass, pos), st["into"]):
                    dst[i, h, :len(kept)] = src[i, h, kept]
            else:
                holes, moved = (~stays).nonzero()[:, 0], kept[kept >= keep]
                holes = holes[holes < keep]
                for x in (k, v, mass, pos):
                    x[i, h, holes] = x[i, h, moved].clone()
    out = st["into"] if case["into"] else (k, v, mass, pos)
    return left, out[0].double(), out[1].double(), out[2].double(), out[3]
