"""Shared contexts and the cache with accumulated weights as they are used: the cache object, captured graphs, streams, large and far
tensors, many sequences, values that are not finite."""
import pytest
import torch

import mass_reference as mr
import window_reference as ref
from test_gpu_mass import DT, INF, NAN, PROMPT, STEP, _check_context, _check_sequence, _i32, _rnd, _same, _sh

pytestmark = pytest.mark.gpu


def _state(n, hk, slots, d, dt):
    return [torch.zeros(n, hk, slots, d, dtype=dt, device="cuda"), torch.zeros(n, hk, slots, d, dtype=dt, device="cuda"),
            torch.zeros(n, hk, slots, device="cuda"), torch.zeros(n, hk, slots, dtype=torch.int32, device="cuda")]


@pytest.mark.parametrize("dtype,rope,shared", [("bf16", True, True), ("f16", False, True), ("f32", True, False)])
def test_mass_cache(dtype, rope, shared):
    """The object against the calls that it stands for, bit by bit: prompts longer than the cache, a chunk that fits, steps with evictions."""
    sh, rnd, dt = _sh(), _rnd(5), DT[dtype]
    n, hk, g, d, budget, recent, spare, p = 3, 2, 2, 64, 24, 6, 8, 19
    rp = sh.Rope(10000.0 ** (-torch.arange(0, d, 2, device="cuda").float() / d), rnd(d, dtype=dt), rnd(d, dtype=dt)) if rope else None
    prefix = (rnd(1, hk, p, d, dtype=dt), rnd(1, hk, p, d, dtype=dt)) if shared else None
    first = p if shared else 0
    cache = sh.MassCache(n, hk * g, hk, d, budget, recent, spare, dtype=dtype, rope=rp, prefix=prefix, scale=0.3)
    cache.lengths[2] = -1
    state = _state(n, hk, budget + spare, d, dt)
    lengths, seen = _i32([0, 0, -1]), _i32([first] * n)

    def prepared(q, k, pos):
        if rope:
            q, k = sh.qk_norm_rope(q, k, pos, rp)
        return q, k, sh.context_attention(q, *prefix, scale=0.3, partial=True) if shared else None

    for counts in ([70, 11, 0], [5, 8, 0], [30, 2, 3]):                # the second fits into the spare slots
        starts, total = [0], sum(counts)
        for x in counts:
            starts.append(starts[-1] + x)
        q, k, v = rnd(total, hk * g, d, dtype=dt), rnd(total, hk, d, dtype=dt), rnd(total, hk, d, dtype=dt)
        got = cache.prefill(q, k, v, _i32(starts), longest=max(counts))
        pos = torch.cat([seen[i] + torch.arange(counts[i], dtype=torch.int32, device="cuda") for i in range(n)])
        q, k, prior = prepared(q, k, pos)
        grown = lengths + torch.where(lengths < 0, 0, _i32(counts))
        if max(counts) > spare:
            whole = _state(n, hk, budget + max(counts), d, dt)
            held = sh.mass_evict(*state, lengths, keep=budget, recent=recent, into=whole)
            out = sh.mass_prefill(q, k, v, _i32(starts), held, *whole, seen, prior=prior, scale=0.3)
            lengths = sh.mass_evict(*whole, held + torch.where(held < 0, 0, _i32(counts)), keep=budget, recent=recent, into=state)
        else:
            out = sh.mass_prefill(q, k, v, _i32(starts), lengths, *state, seen, prior=prior, scale=0.3)
            lengths = grown
        seen += torch.where(lengths < 0, 0, _i32(counts))
        assert torch.equal(got, out) and torch.equal(cache.lengths, lengths) and torch.equal(cache.seen, seen)
    since = 0                                                          # tokens since the last eviction
    for step in range(3 * spare + 1):
        q, k, v = rnd(n, hk * g, d, dtype=dt), rnd(n, hk, d, dtype=dt), rnd(n, hk, d, dtype=dt)
        got = cache.decode(q, k, v)
        if since == spare:
            sh.mass_evict(*state, lengths, keep=budget, recent=recent, left=lengths)
            since = 0
        q, k, prior = prepared(q, k, seen)
        out = sh.mass_decode(q, k, v, lengths, *state, seen, prior=prior, scale=0.3)
        active = (lengths >= 0).to(torch.int32)
        lengths, seen, since = lengths + active, seen + active, since + 1
        assert torch.equal(got, out) and torch.equal(cache.lengths, lengths) and torch.equal(cache.seen, seen)
    for a, b in zip((cache.k, cache.v, cache.mass, cache.positions), state):
        for i, c in enumerate(lengths.tolist()):
            assert torch.equal(a[i, :, :max(c, 0)], b[i, :, :max(c, 0)])
    for i in range(2):
        for h in range(hk):
            held = cache.positions[i, h, :int(lengths[i])].tolist()
            assert len(set(held)) == len(held) and set(range(int(seen[i]) - recent, int(seen[i]))) <= set(held) and min(held) >= first


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_steps(dtype):
    """Two graphs of a whole step, each with its own tensors, replayed at once on two streams with lengths that move on; against eager calls."""
    sh, dt = _sh(), DT[dtype]
    n, hk, g, d, slots, keep = 4, 2, 4, 128, 300, 290
    sides = []
    for side in range(2):
        rnd = _rnd(side)
        s = dict(k=rnd(n, hk, slots, d, dtype=dt), v=rnd(n, hk, slots, d, dtype=dt), mass=rnd(n, hk, slots, dtype=torch.float32).abs(),
                 positions=torch.arange(slots, dtype=torch.int32, device="cuda").expand(n, hk, slots).contiguous(), lengths=_i32([295, 3, 299, -1]),
                 seen=_i32([300, 3, 400, 0]), q=rnd(n, hk * g, d, dtype=dt), kn=rnd(n, hk, d, dtype=dt), vn=rnd(n, hk, d, dtype=dt),
                 pk=rnd(1, hk, 600, d, dtype=dt), pv=rnd(1, hk, 600, d, dtype=dt), out=torch.zeros(n, hk * g, d, dtype=dt, device="cuda"))
        sides.append(s)

    def step(s):
        prior = sh.context_attention(s["q"], s["pk"], s["pv"], partial=True)
        sh.mass_decode(s["q"], s["kn"], s["vn"], s["lengths"], s["k"], s["v"], s["mass"], s["positions"], s["seen"], prior=prior, out=s["out"])
        active = (s["lengths"] >= 0).to(torch.int32)
        s["lengths"] += active
        s["seen"] += active
        sh.mass_evict(s["k"], s["v"], s["mass"], s["positions"], s["lengths"], keep=keep, recent=20, left=s["lengths"])

    want = [{name: x.clone() for name, x in s.items()} for s in sides]
    for w in want:
        for _ in range(6):
            step(w)
    streams, graphs = [torch.cuda.Stream(), torch.cuda.Stream()], []
    torch.cuda.synchronize()
    for s, stream in zip(sides, streams):
        keepsake = {name: x.clone() for name, x in s.items()}
        with torch.cuda.stream(stream):
            step(s)
            for name, x in s.items():
                x.copy_(keepsake[name])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step(s)
        graphs.append(graph)
    torch.cuda.synchronize()
    for _ in range(6):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for s, w in zip(sides, want):
        for name in s:
            assert torch.equal(s[name], w[name]), name


def test_captured_prompts_on_a_stream_of_their_own():
    sh, rnd, dt = _sh(), _rnd(9), torch.float16
    n, hk, g, d, slots = 3, 1, 4, 64, 2500
    total = 40
    q, k, v = rnd(total, hk * g, d, dtype=dt), rnd(total, hk, d, dtype=dt), rnd(total, hk, d, dtype=dt)
    kc, vc = rnd(n, hk, slots, d, dtype=dt), rnd(n, hk, slots, d, dtype=dt)
    starts, lengths, seen = _i32([0, 0, 0, 0]), _i32([0, 0, 0]), _i32([0, 0, 0])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    new = [kc.clone(), vc.clone(), torch.zeros(n, hk, slots, device="cuda"), torch.zeros(n, hk, slots, dtype=torch.int32, device="cuda")]
    out = torch.zeros_like(q)
    torch.cuda.synchronize()
    call = lambda: sh.mass_prefill(q, k, v, starts, lengths, *new, seen, out=out, stream=side)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    for counts, held in (([40, 0, 0], [2400, 7, 0]), ([1, 20, 19], [0, 2480, 1000]), ([3, 3, 34], [2497, -1, 5])):
        at = [0]
        for c in counts:
            at.append(at[-1] + c)
        starts.copy_(_i32(at)), lengths.copy_(_i32(held)), seen.copy_(_i32([max(c, 0) for c in held]))
        for x, y in zip(new, (kc, vc)):
            x.copy_(y)
        new[2].fill_(0.5), new[3].fill_(-3), out.fill_(7)
        old = [x.clone() for x in new]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, (c, rows) in enumerate(zip(held, counts)):
            a, b = at[i], at[i + 1]
            if rows == 0 or c < 0:
                assert (out[a:b] == 7).all() and all(_same(x[i], y[i]) for x, y in zip(new, old))
            else:
                _check_sequence(old, new, i, c, rows, q[a:b], k[a:b], v[a:b], out[a:b], max(c, 0), g, dt, PROMPT)


def _big(q, keys, vals, held, dt, prior=None):
    """All rows of one sequence in 64 bits on the device, a head at a time: differences over tolerances of outputs and masses are returned as
    functions of what is to be compared."""
    t, hq, d = q.shape
    m, hk = keys.shape[:2]
    g, half = hq // hk, ref.half_step(dt)
    sees = torch.arange(m, device="cuda")[None] <= held + torch.arange(t, device="cuda")[:, None]
    chain = (m / 16 + 64) * 2.0 ** -23
    out, tol, mass, mass_tol = [], [], torch.zeros(hk, m, dtype=torch.float64, device="cuda"), torch.zeros(hk, m, dtype=torch.float64, device="cuda")
    for h in range(hq):
        qq, k, v = q[:, h].double(), keys[:, h // g].double(), vals[:, h // g].double()
        s = (qq @ k.T * d ** -0.5).masked_fill(~sees, -INF)
        size = ((qq.abs() @ k.abs().T) * d ** -0.5).masked_fill(~sees, 0).amax(1, keepdim=True)
        lse = torch.logsumexp(s, 1, keepdim=True)
        p = torch.exp(s - lse)
        e = ((d + 8) * 2.0 ** -23 + half ** 2) * size + 2.0 ** -21
        o, vol = p @ v, p @ v.abs()
        tl = ref.rounding(o, dt) + (e + chain) * (vol + o.abs()) + half * vol
        if dt == torch.float16:
            tl = tl + 2.0 ** -32 * p.amax(1, keepdim=True) * (sees.double() @ v.abs()) + 2.0 ** -24
        out.append(o), tol.append(tl)
        mass[h // g] += p.sum(0)
        mass_tol[h // g] += (p * (2 * e + chain + 8 * 2.0 ** -24 * lse.abs() + 2.0 ** -21)).sum(0)
    mass_tol += (t * g + 8) * 2.0 ** -24 * mass + 2.0 ** -23 * mass
    return torch.stack(out, 1), torch.stack(tol, 1), mass, mass_tol


@pytest.mark.parametrize("dtype,d,hk,g,counts,held", [
    ("bf16", 128, 4, 4, [2048, 1, 777, 0, 300], [0, 0, 0, 0, 0]), ("f16", 128, 8, 1, [1500], [700]), ("f16", 64, 2, 8, [513, 1025], [0, 63]),
    ("bf16", 64, 1, 16, [900, 130], [2000, 0]), ("bf16", 128, 1, 7, [700], [129]), ("f16", 64, 1, 130, [60], [65]),
])
def test_prompts_that_fill_the_device(dtype, d, hk, g, counts, held):
    """Every row, twice: the second run gives the same bits (no sum depends on an order of arrival)."""
    sh, rnd, dt, n = _sh(), _rnd(d + g), DT[dtype], len(counts)
    slots = max(a + b for a, b in zip(counts, held)) + 3
    starts = [0]
    for c in counts:
        starts.append(starts[-1] + c)
    q, k, v = (rnd(starts[-1], x, d, dtype=dt) for x in (hk * g, hk, hk))
    kc, vc = rnd(n, hk, slots, d, dtype=dt), rnd(n, hk, slots, d, dtype=dt)
    runs = []
    for _ in range(2):
        new = [kc.clone(), vc.clone(), torch.full((n, hk, slots), 0.25, device="cuda"), torch.zeros(n, hk, slots, dtype=torch.int32, device="cuda")]
        out = sh.mass_prefill(q, k, v, _i32(starts), _i32(held), *new, _i32(held))
        runs.append((out, *new))
    assert all(torch.equal(a, b) for a, b in zip(*runs))
    out, kn, vn, mass, _ = runs[0]
    for i, (c, rows) in enumerate(zip(held, counts)):
        if rows == 0:
            continue
        end = c + rows
        want, tol, got, got_tol = _big(q[starts[i]:starts[i + 1]], kn[i, :, :end].transpose(0, 1), vn[i, :, :end].transpose(0, 1), c, dt)
        assert ((out[starts[i]:starts[i + 1]].double() - want).abs() <= tol).all()
        before = torch.where(torch.arange(end, device="cuda") < c, 0.25, 0.0).double()
        assert ((mass[i, :, :end].double() - got - before).abs() <= got_tol + 2.0 ** -24).all()
        assert (mass[i, :, end:] == 0.25).all()


def test_many_sequences():
    """More sequences than a warp looks at in one go, most of them short, some without tokens."""
    sh, rnd, dt, hk, g, d, slots, n = _sh(), _rnd(1), torch.bfloat16, 2, 2, 64, 40, 333
    counts = [(i * 7) % 5 for i in range(n)]
    held = [(i * 13) % 36 for i in range(n)]
    starts = [0]
    for c in counts:
        starts.append(starts[-1] + c)
    q, k, v = (rnd(starts[-1], x, d, dtype=dt) for x in (hk * g, hk, hk))
    new = [rnd(n, hk, slots, d, dtype=dt), rnd(n, hk, slots, d, dtype=dt), torch.ones(n, hk, slots, device="cuda"),
           torch.arange(slots, dtype=torch.int32, device="cuda").expand(n, hk, slots).contiguous()]
    old = [x.clone() for x in new]
    out = sh.mass_prefill(q, k, v, _i32(starts), _i32(held), *new, _i32(held))
    ctx, lse = sh.context_attention(q, old[0], old[1], _i32(starts), _i32(held))
    left = sh.mass_evict(*new, _i32(held), keep=10, recent=2)
    assert left.tolist() == [min(c, 10) for c in held]
    again = [x.clone() for x in old]
    sh.mass_prefill(q, k, v, _i32(starts), _i32(held), *again, _i32(held), out=out)
    for i in list(range(0, n, 29)) + [n - 1]:
        a, b = starts[i], starts[i + 1]
        if a < b:
            _check_sequence(old, again, i, held[i], b - a, q[a:b], k[a:b], v[a:b], out[a:b], held[i], g, dt, PROMPT)
            if held[i]:
                _check_context(q, old[0][i:i + 1], old[1][i:i + 1], [(a, b)], [held[i]], ctx, lse, dt, PROMPT)
        for h in range(hk):
            _, holes, moved = mr.evict(again[2][i, h, :held[i]].tolist(), again[3][i, h, :held[i]].tolist(), 10, 2)
            want = again[0][i, h].clone()
            want[holes] = again[0][i, h][moved]
            assert torch.equal(new[0][i, h, :held[i]], want[:held[i]])


@pytest.mark.parametrize("dtype,kind", [("bf16", "few"), ("f16", "few"), ("f32", "few"), ("bf16", "steps"), ("f16", "steps"), ("f32", "steps"), ("bf16", "prompts"), ("f16", "prompts"), ("f32", "prompts")])
def test_values_that_are_not_finite(dtype, kind):
    """An infinite value in sight shows in its element alone; what is out of sight does not show at all; a query that is not finite spoils its own
    rows and the masses that it gives, nothing else."""
    sh, rnd, dt, hk, g, d, slots = _sh(), _rnd(2), DT[dtype], 2, 2, 64, 80 if kind == "few" else 300
    counts, held = ([70, 40, 3], [130, 0, 64]) if kind == "prompts" else ([1, 1, 1], [79, 64, 1] if kind == "few" else [200, 64, 1])
    starts = [0]
    for c in counts:
        starts.append(starts[-1] + c)
    total = starts[-1]
    q, k, v = (rnd(total, x, d, dtype=dt) for x in (hk * g, hk, hk))
    state = [rnd(3, hk, slots, d, dtype=dt), rnd(3, hk, slots, d, dtype=dt), torch.ones(3, hk, slots, device="cuda"), torch.zeros(3, hk, slots, dtype=torch.int32, device="cuda")]
    for i, c in enumerate(held):
        state[0][i, :, c:], state[1][i, :, c:], state[2][i, :, c:] = NAN, NAN, NAN
    if held[0]:
        state[1][0, 0, 5, 7] = INF                               # sequence 0, key head 0: element 7 of its two query heads
    if kind == "prompts":
        v[starts[0] + 60, 1, 9] = -INF                           # seen by its last ten tokens only
    q[starts[2], 3, 0] = NAN                                     # the first token of sequence 2, its last head
    clean = [x.clone() for x in state]
    clean[1][0, 0, 5, 7] = 0
    qc, vc = q.clone(), v.clone()
    qc[starts[2], 3, 0] = 0
    if kind == "prompts":
        vc[starts[0] + 60, 1, 9] = 0

    def run(q, v, state):
        out = torch.zeros_like(q)
        if kind != "prompts":
            sh.mass_decode(q, k, v, _i32(held), *state, _i32(held), out=out)
        else:
            sh.mass_prefill(q, k, v, _i32(starts), _i32(held), *state, _i32(held), out=out)
        return out

    out, want = run(q, v, state), run(qc, vc, clean)
    spoiled = torch.zeros_like(out, dtype=torch.bool)
    if held[0]:
        spoiled[starts[0]:starts[1], :2, 7] = True
        assert (out[starts[0]:starts[1], :2, 7] == INF).all()
    if kind == "prompts":
        spoiled[starts[0] + 60:starts[1], 2:, 9] = True
        assert (out[starts[0] + 60:starts[1], 2:, 9] == -INF).all()
    spoiled[starts[2], 3] = True
    assert out[starts[2], 3].isnan().all()
    near = (out.double() - want.double()).abs() <= 4 * torch.finfo(dt).eps * want.double().abs().clamp(min=0.05)
    assert (near | spoiled).all()
    # Masses do not depend on the values, so both runs lie within one bound of the same definition.  (Not the same bits: a row that is computed
    # again adds its products in another order.)  Sequence 2: of the key head that the spoiled query does not read.
    for i in range(3):
        end, a, b = held[i] + counts[i], starts[i], starts[i + 1]
        x = mr.attend(qc[a:b], clean[0][i, :, :end].transpose(0, 1), clean[1][i, :, :end].transpose(0, 1),
                      torch.arange(end)[None] <= torch.arange(held[i], end)[:, None])
        tol = 2 * mr.mass_tolerance(x, g, dt, (torch.arange(end) < held[i]).double()[:, None]).T
        near = (state[2][i, :, :end].double().cpu() - clean[2][i, :, :end].double().cpu()).abs() <= tol
        assert (near if i < 2 else near[:1]).all()
    assert state[2][2, 1, :held[2] + 1].isnan().all()


def test_far_offsets():
    """Rows that lie more than 2^32 bytes apart, for every call that takes a cache."""
    sh, rnd, dt, hk, g, d, slots = _sh(), _rnd(4), torch.bfloat16, 2, 2, 128, 60
    far = (1 << 32) // 2 + 1024                                  # elements between key heads
    keys, values = (torch.empty(far * 2, dtype=dt, device="cuda") for _ in range(2))
    view = lambda x: x.as_strided((2, hk, slots, d), (slots * d, far, d, 1))
    near = [rnd(2, hk, slots, d, dtype=dt), rnd(2, hk, slots, d, dtype=dt)]
    kc, vc = view(keys), view(values)
    kc.copy_(near[0]), vc.copy_(near[1])
    q, k, v = (rnd(6, x, d, dtype=dt) for x in (hk * g, hk, hk))
    held, starts = _i32([40, 50]), _i32([0, 4, 6])
    mass = rnd(2, hk, slots, dtype=torch.float32).abs()
    pos = torch.arange(slots, dtype=torch.int32, device="cuda").expand(2, hk, slots).contiguous()
    got = []
    for kk, vv in (near, (kc, vc)):
        m, p = mass.clone(), pos.clone()
        a = sh.mass_prefill(q, k, v, starts, held, kk, vv, m, p, held)
        ln = held + _i32([4, 2])
        b = sh.mass_decode(q[:2], k[:2], v[:2], ln, kk, vv, m, p, ln)
        c = sh.context_attention(q, kk, vv, starts, held)
        e = sh.context_attention(q[:2], kk, vv, lengths=held)
        ln = sh.mass_evict(kk, vv, m, p, ln + 1, keep=33, recent=5)
        got.append((a, b, *c, *e, ln, m, p, kk.clone(), vv.clone()))
    for x, y in zip(*got):
        assert torch.equal(x, y)


def test_nothing_to_do():
    sh, dt = _sh(), torch.float16
    e = lambda *s: torch.empty(*s, dtype=dt, device="cuda")
    out, lse = sh.context_attention(e(0, 4, 64), e(3, 2, 5, 64), e(3, 2, 5, 64), _i32([0, 0, 0, 0]))
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    m, p = torch.zeros(2, 2, 5, device="cuda"), torch.zeros(2, 2, 5, dtype=torch.int32, device="cuda")
    k, v = e(2, 2, 5, 64).zero_(), e(2, 2, 5, 64).zero_()
    before = [x.clone() for x in (k, v, m, p)]
    sh.mass_prefill(e(0, 4, 64), e(0, 2, 64), e(0, 2, 64), _i32([0, 0, 0]), _i32([1, 2]), k, v, m, p, _i32([1, 2]))
    sh.mass_decode(e(2, 4, 64).zero_(), e(2, 2, 64).zero_(), e(2, 2, 64).zero_(), _i32([-1, 5]), k, v, m, p, _i32([1, 2]))
    assert sh.mass_evict(k, v, m, p, _i32([-1, 0]), keep=2).tolist() == [-1, 0]
    assert all(torch.equal(a, b) for a, b in zip((k, v, m, p), before))
    sh.window_status()


def test_wrappers_refuse():
    sh, dt = _sh(), torch.float16
    z = lambda *s: torch.zeros(*s, dtype=dt, device="cuda")
    q, k, c, m, p, i = z(2, 4, 64), z(2, 2, 64), z(2, 2, 5, 64), torch.zeros(2, 2, 5, device="cuda"), torch.zeros(2, 2, 5, dtype=torch.int32, device="cuda"), _i32([1, 1])
    ok = dict(q=q, k=k, v=k, lengths=i, k_cache=c, v_cache=c.clone(), mass=m, positions=p, seen=i)
    bad = [dict(q=q.float()), dict(k=z(2, 3, 64)), dict(v=z(2, 2, 128)), dict(lengths=i.long()), dict(lengths=_i32([1])), dict(k_cache=z(2, 1, 5, 64)),
           dict(v_cache=z(2, 2, 6, 64)), dict(mass=m.double()), dict(mass=m.transpose(0, 1)), dict(positions=p.long()), dict(positions=p[:, :, :4]),
           dict(mass=torch.zeros(2, 2, 10, device="cuda")[:, :, ::2]), dict(seen=i.float()), dict(scale=-1.0), dict(out=z(2, 4, 64).float()),
           dict(prior=q), dict(prior=(q, torch.zeros(2, 5, device="cuda"))), dict(prior=(q, torch.zeros(2, 4, device="cuda", dtype=torch.float64))),
           dict(prior=(z(2, 3, 64), torch.zeros(2, 4, device="cuda")))]
    for change in bad:
        with pytest.raises(ValueError):
            sh.mass_decode(**{**ok, **change})
        with pytest.raises(ValueError):
            sh.mass_prefill(**{**ok, "starts": _i32([0, 1, 2]), **change})
    for args in (dict(keep=0), dict(keep=6), dict(keep=2, recent=3), dict(keep=2, into=(c, c)), dict(keep=2, left=i.long()),
                 dict(keep=2, into=(z(2, 2, 1, 64), z(2, 2, 1, 64), torch.zeros(2, 2, 1, device="cuda"), torch.zeros(2, 2, 1, dtype=torch.int32, device="cuda")))):
        with pytest.raises(ValueError):
            sh.mass_evict(c, c.clone(), m, p, i, **args)
    for args in ((q, z(3, 2, 5, 64), z(3, 2, 5, 64)), (q, c, c, _i32([0, 2])), (q, c, z(2, 2, 5, 128)), (q, z(2, 3, 5, 64), z(2, 3, 5, 64))):
        with pytest.raises(ValueError):
            sh.context_attention(*args)
    with pytest.raises(sh.ShError):                              # a stride that is no multiple of 16 bytes
        odd = torch.zeros(2 * 2 * 5 * 68, dtype=dt, device="cuda").as_strided((2, 2, 5, 64), (2 * 5 * 68, 5 * 68, 68, 1))
        sh.context_attention(q, odd, odd)


@pytest.mark.parametrize("n,hk,d,slots,keep,recent", [(40, 32, 64, 100, 70, 10), (5, 1, 128, 200, 150, 60), (76, 1, 64, 47000, 500, 100), (3, 1, 64, 380000, 9000, 50)])
def test_eviction_of_other_shapes(n, hk, d, slots, keep, recent):
    """Many short caches, which move their own rows; long ones whose keys do not fit into shared memory."""
    sh, rnd, dt = _sh(), _rnd(slots), torch.float16
    state = [rnd(n, hk, slots, d, dtype=dt), rnd(n, hk, slots, d, dtype=dt), (rnd(n, hk, slots, dtype=torch.float32) * 8).round() / 8,
             torch.rand(n, hk, slots, device="cuda").argsort(-1).to(torch.int32)]
    held = [slots - (i * 37) % (slots // 2) for i in range(n)]
    old = [x.clone() for x in state]
    lengths = _i32(held)
    left = sh.mass_evict(*state, lengths, keep=keep, recent=recent)
    assert left.tolist() == [min(c, keep) for c in held]
    assert sh.mass_evict(*[x.clone() for x in old], lengths, keep=keep, recent=recent, left=lengths).tolist() == left.tolist()
    for i in sorted({0, n // 2, n - 1}):
        for h in sorted({0, hk - 1}):
            _, holes, moved = mr.evict(old[2][i, h, :held[i]].tolist(), old[3][i, h, :held[i]].tolist(), keep, recent)
            for x, y in zip(old, state):
                want = x[i, h].clone()
                want[holes] = x[i, h][moved]
                assert torch.equal(y[i, h], want)


@pytest.mark.parametrize("dtype,g", [("f16", 4), ("bf16", 9), ("f32", 3)])
def test_steps_of_many_sequences(dtype, g):
    """More units than run at once: the weights are added by a launch of their own."""
    sh, rnd, dt, n, hk, d, slots = _sh(), _rnd(g), DT[dtype], 900, 2, 64, 600
    q, k, v = (rnd(n, x, d, dtype=dt) for x in (hk * g, hk, hk))
    held = [(i * 71) % slots if i % 10 else -1 for i in range(n)]
    old = [rnd(n, hk, slots, d, dtype=dt), rnd(n, hk, slots, d, dtype=dt), torch.ones(n, hk, slots, device="cuda"), torch.zeros(n, hk, slots, dtype=torch.int32, device="cuda")]
    new = [x.clone() for x in old]
    out = sh.mass_decode(q, k, v, _i32(held), *new, _i32([max(c, 0) for c in held]))
    for i in (0, 1, 2, 333, 511, 899):
        if held[i] < 0:
            assert (out[i] == 0).all() and all(torch.equal(x[i], y[i]) for x, y in zip(new, old))
        else:
            _check_sequence(old, new, i, held[i], 1, q[i:i + 1], k[i:i + 1], v[i:i + 1], out[i:i + 1], held[i], g, dt, STEP)
