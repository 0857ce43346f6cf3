"""Attention over shared contexts and the cache with accumulated weights against their 64-bit definitions (bounds: mass_reference)."""
import pytest
import torch

import mass_reference as mr
import window_reference as ref

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
STEP, PROMPT = dict(parts=2, lift=15), dict(parts=1, lift=7)
NAN, INF = float("nan"), float("inf")


def _sh():
    from paper_2305_17118_b200 import binding as sh
    return sh


def _rnd(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *shape, dtype: torch.randn(*shape, generator=g, device="cuda").to(dtype)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _check_context(q, k, v, ranges, lengths, out, lse, dtype, kind, scale=None):
    """ranges: (first, end) of each context's tokens."""
    for i, (a, b) in enumerate(ranges):
        n = min(max(lengths[i], 0), k.shape[2])
        if a == b:
            continue
        if n == 0:
            assert (out[a:b] == 0).all() and (lse[a:b] == -INF).all()
            continue
        x = mr.attend(q[a:b], k[i, :, :n].transpose(0, 1), v[i, :, :n].transpose(0, 1), torch.ones(b - a, n, dtype=torch.bool), scale)
        ref.check(out[a:b], x["out"], mr.out_tolerance(x, dtype, out_dtype=out.dtype, **kind), f"context {i}")
        ref.check(lse[a:b], x["lse"], mr.lse_tolerance(x, dtype), f"lse of context {i}")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d,hk,g,rows,lengths", [
    (64, 2, 1, 1, [1, 1, 0]), (128, 1, 4, 17, [17, 16, 1, -1]), (64, 3, 7, 200, [200, 3, 129]), (128, 2, 16, 1031, [1031, 400]),
    (64, 8, 8, 65, [65] * 40),
])
def test_one_token_of_each_context(dtype, d, hk, g, rows, lengths):
    sh, rnd, dt, n = _sh(), _rnd(rows + g), DT[dtype], len(lengths)
    q, k, v = rnd(n, hk * g, d, dtype=dt), rnd(n, hk, rows, d, dtype=dt), rnd(n, hk, rows, d, dtype=dt)
    for i, x in enumerate(lengths):                              # what lies behind a context is not looked at
        k[i, :, max(x, 0):], v[i, :, max(x, 0):] = NAN, INF
    for partial in (False, True):
        out, lse = sh.context_attention(q, k, v, lengths=_i32(lengths), partial=partial)
        assert out.dtype == (torch.float32 if partial else dt)
        _check_context(q, k, v, [(i, i + 1) for i in range(n)], lengths, out, lse, dt, STEP)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d,hk,g,rows,counts,lengths", [
    (64, 2, 1, 5, [3, 0, 2], [5, 4, 1]), (128, 2, 4, 64, [33, 1, 70], [64, 63, 65]), (64, 1, 7, 130, [40, 0, 0, 19], [0, 130, 5, 129]),
    (128, 1, 16, 300, [17, 30], [300, 1]), (64, 4, 3, 4000, [2, 1], [4000, 3999]),
])
def test_prompts_over_contexts(dtype, d, hk, g, rows, counts, lengths):
    """Ragged tokens, views of a packed projection, contexts laid out [rows, heads], rows that belong to nobody."""
    sh, rnd, dt, n = _sh(), _rnd(rows + g), DT[dtype], len(counts)
    before, behind = 3, 2
    total = before + sum(counts) + behind
    q = rnd(total, hk * g + 5, d, dtype=dt)[:, 2:2 + hk * g]
    k, v = rnd(n, rows, hk, d, dtype=dt).transpose(1, 2), rnd(n, rows, hk, d, dtype=dt).transpose(1, 2)
    q[:before], q[total - behind:] = NAN, NAN
    for i, x in enumerate(lengths):
        k[i, :, x:], v[i, :, x:] = INF, NAN
    starts = [before]
    for c in counts:
        starts.append(starts[-1] + c)
    out, lse = torch.full((total, hk * g, d), 7.0, dtype=dt, device="cuda"), torch.full((total, hk * g), 7.0, device="cuda")
    sh.context_attention(q, k, v, _i32(starts), _i32(lengths), out=out, lse=lse, scale=0.2)
    _check_context(q, k, v, list(zip(starts, starts[1:])), lengths, out, lse, dt, PROMPT, 0.2)
    for x in (out, lse):
        assert (x[:before] == 7).all() and (x[total - behind:] == 7).all()
    fresh = sh.context_attention(q, k, v, _i32(starts), _i32(lengths), scale=0.2)
    part = sh.context_attention(q, k, v, _i32(starts), _i32(lengths), scale=0.2, partial=True)
    _check_context(q, k, v, list(zip(starts, starts[1:])), lengths, *part, dt, PROMPT, 0.2)
    assert torch.equal(fresh[0][before:total - behind], out[before:total - behind]) and (fresh[0][:before] == 0).all() and (fresh[1][:before] == -INF).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d,hk,g,rows,tokens", [(128, 2, 4, 700, 33), (64, 1, 1, 20000, 5), (128, 1, 8, 9000, 2), (64, 2, 2, 129, 300)])
def test_a_shared_prefix(dtype, d, hk, g, rows, tokens):
    sh, rnd, dt = _sh(), _rnd(rows), DT[dtype]
    q, k, v = rnd(tokens, hk * g, d, dtype=dt), rnd(1, hk, rows, d, dtype=dt), rnd(1, hk, rows, d, dtype=dt)
    for lengths in ([rows], [rows - 7], [0]):
        for partial in (False, True):
            out, lse = sh.context_attention(q, k, v, lengths=_i32(lengths), partial=partial)
            _check_context(q, k, v, [(0, tokens)], lengths, out, lse, dt, PROMPT)
    whole = sh.context_attention(q, k, v)
    again = sh.context_attention(q, k, v, starts=_i32([0, tokens]))
    assert torch.equal(whole[0], again[0]) and torch.equal(whole[1], again[1])


def _cache(rnd, n, hk, slots, d, dt, held, poison=True):
    """A cache whose records lie in a wider tensor; slots that hold nothing hold NaN."""
    k, v = rnd(n, hk, slots, d, dtype=dt), rnd(n, hk, slots, d, dtype=dt)
    mass = rnd(n, hk + 1, slots + 3, dtype=torch.float32).abs()[:, 1:, 1:slots + 1]
    positions = torch.zeros(n, hk + 1, slots + 3, dtype=torch.int32, device="cuda")[:, 1:, 1:slots + 1]
    for i, c in enumerate(held):
        if poison:
            k[i, :, max(c, 0):], v[i, :, max(c, 0):], mass[i, :, max(c, 0):] = NAN, INF, NAN
        for h in range(hk):
            positions[i, h, :max(c, 0)] = torch.randperm(max(c, 0), device="cuda").to(torch.int32) * 2
    return k, v, mass, positions


def _same(a, b):
    return torch.equal(a.nan_to_num(nan=-77.0), b.nan_to_num(nan=-77.0))


def _check_sequence(old, new, i, c, rows, q, kn, vn, out, seen, g, dt, kind, prior=None, scale=None):
    """Sequence i, which held c rows, has taken `rows` new ones."""
    k, v, mass, positions = new
    end, hk = c + rows, k.shape[1]
    assert torch.equal(k[i, :, c:end], kn.transpose(0, 1)) and torch.equal(v[i, :, c:end], vn.transpose(0, 1))
    for now, was in zip(new, old):                               # everything else is as it was
        if now is not mass:
            assert _same(now[i, :, :c], was[i, :, :c])
        assert _same(now[i, :, end:], was[i, :, end:])
    assert torch.equal(positions[i, :, c:end], (seen + torch.arange(rows, dtype=torch.int32, device="cuda")).expand(hk, rows))
    sees = torch.arange(end)[None] <= torch.arange(c, end)[:, None]
    x = mr.attend(q, k[i, :, :end].transpose(0, 1), v[i, :, :end].transpose(0, 1), sees, scale, prior)
    ref.check(out, x["out"], mr.out_tolerance(x, dt, **kind), f"sequence {i}")
    before = old[2][i].T.double().cpu()[:end].clone()
    before[c:] = 0
    ref.check(mass[i, :, :end].T, before + mr.mass_of(x, g), mr.mass_tolerance(x, g, dt, before), f"mass of sequence {i}")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d,hk,g,slots,held", [
    (64, 2, 1, 1, [0, 0]), (128, 1, 4, 33, [32, 0, -1, 17, 33]), (64, 3, 7, 200, [199, 3, 128, 127]), (128, 2, 16, 900, [899, 400]),
    (64, 8, 2, 70, [69] * 40), (64, 1, 1, 6000, [5900]),
])
def test_single_tokens(dtype, d, hk, g, slots, held):
    """Types, head layouts, idle sequences, full caches, few rows over a long axis; with and without a shared prefix before them."""
    sh, rnd, dt, n = _sh(), _rnd(slots + g), DT[dtype], len(held)
    packed = rnd(n, hk * (g + 2), d, dtype=dt)
    q, kn, vn = packed[:, :hk * g], packed[:, hk * g:hk * (g + 1)], packed[:, hk * (g + 1):]
    seen = _i32([max(c, 0) * 2 + 5 for c in held])
    pk, pv = rnd(1, hk, 50, d, dtype=dt), rnd(1, hk, 50, d, dtype=dt)
    for prior in (None, sh.context_attention(q, pk, pv, partial=True), sh.context_attention(q, pk, pv)):
        old = _cache(_rnd(slots), n, hk, slots, d, dt, held)
        new = tuple(x.clone() for x in old[:2]) + _cache(_rnd(slots), n, hk, slots, d, dt, held)[2:]
        new[3].copy_(old[3])
        out = torch.full((n, hk * g, d), 7.0, dtype=dt, device="cuda")
        assert sh.mass_decode(q, kn, vn, _i32(held), *new, seen, prior=prior, out=out) is out
        for i, c in enumerate(held):
            if not 0 <= c < slots:
                assert (out[i] == 7).all() and all(_same(a[i], b[i]) for a, b in zip(new, old))
                continue
            pr = None if prior is None else tuple(x[i:i + 1] for x in prior)
            _check_sequence(old, new, i, c, 1, q[i:i + 1], kn[i:i + 1], vn[i:i + 1], out[i:i + 1], int(seen[i]), g, dt, STEP, pr)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d,hk,g,slots,counts,held", [
    (64, 2, 1, 9, [1, 0, 9], [0, 3, 0]), (128, 1, 4, 200, [130, 7, 30, 5], [0, 190, 171, -1]), (64, 2, 7, 150, [64, 65], [64, 1]),
    (128, 1, 16, 90, [33], [50]), (64, 1, 2, 3000, [20, 3], [2900, 0]), (64, 4, 1, 700, [513, 129, 127], [0, 0, 511]),
])
def test_prompts(dtype, d, hk, g, slots, counts, held):
    """Ragged chunks over caches, sequences without tokens or room or that are idle, rows of nobody; with and without a prefix."""
    sh, rnd, dt, n = _sh(), _rnd(slots + g), DT[dtype], len(held)
    before, behind = 2, 3
    starts = [before]
    for c in counts:
        starts.append(starts[-1] + c)
    total = starts[-1] + behind
    packed = rnd(total, hk * (g + 2), d, dtype=dt)
    packed[:before], packed[total - behind:] = NAN, NAN
    q, kn, vn = packed[:, :hk * g], packed[:, hk * g:hk * (g + 1)], packed[:, hk * (g + 1):]
    seen = _i32([max(c, 0) * 2 + 5 for c in held])
    pk, pv = rnd(1, hk, 50, d, dtype=dt), rnd(1, hk, 50, d, dtype=dt)
    for prior in (None, sh.context_attention(q, pk, pv, partial=True), sh.context_attention(q, pk, pv)):
        old = _cache(_rnd(slots), n, hk, slots, d, dt, held)
        new = tuple(x.clone() for x in old[:2]) + _cache(_rnd(slots), n, hk, slots, d, dt, held)[2:]
        new[3].copy_(old[3])
        out = torch.full((total, hk * g, d), 7.0, dtype=dt, device="cuda")
        sh.mass_prefill(q, kn, vn, _i32(starts), _i32(held), *new, seen, prior=prior, out=out)
        assert (out[:before] == 7).all() and (out[total - behind:] == 7).all()
        for i, (c, rows) in enumerate(zip(held, counts)):
            a, b = starts[i], starts[i + 1]
            if c < 0 or c + rows > slots or rows == 0:
                assert (out[a:b] == 7).all() and all(_same(x[i], y[i]) for x, y in zip(new, old))
                continue
            pr = None if prior is None else tuple(x[a:b] for x in prior)
            _check_sequence(old, new, i, c, rows, q[a:b], kn[a:b], vn[a:b], out[a:b], int(seen[i]), g, dt, PROMPT, pr)


def _records(rnd, n, hk, slots, held, odd):
    mass = (rnd(n, hk, slots, dtype=torch.float32) * 4).round() / 4       # many equal ones
    if odd:
        mass[..., ::7], mass[..., 1::5], mass[..., 2::11], mass[..., 3::13] = NAN, -0.0, 0.0, INF
    positions = torch.stack([torch.stack([torch.randperm(slots, device="cuda") for _ in range(hk)]) for _ in range(n)]).to(torch.int32)
    return mass, positions


@pytest.mark.parametrize("odd", [False, True])
@pytest.mark.parametrize("dtype,d,hk,slots,held,keep,recent", [
    ("f16", 64, 1, 2, [2, 1, 0, -1], 1, 0), ("f32", 64, 3, 40, [40, 39, 20, 21, 5], 20, 20), ("bf16", 128, 2, 474, [474, 411, 410, 100], 410, 64),
    ("f16", 128, 1, 3000, [3000, 2999, 1500], 100, 1), ("f32", 128, 2, 515, [515, 514], 512, 3), ("bf16", 64, 1, 50000, [50000, 49999], 600, 17),
])
def test_eviction(dtype, d, hk, slots, held, keep, recent, odd):
    sh, rnd, dt, n = _sh(), _rnd(slots), DT[dtype], len(held)
    k, v = rnd(n, hk, slots, d, dtype=dt), rnd(n, hk, slots, d, dtype=dt)
    mass, positions = _records(rnd, n, hk, slots, held, odd)
    src = (k, v, mass, positions)
    own = tuple(x.clone() for x in src)
    room = keep + 3
    into = (torch.full((n, hk, room, d), 7.0, dtype=dt, device="cuda"), torch.full((n, hk, room, d), 8.0, dtype=dt, device="cuda"),
            torch.full((n, hk, room), 9.0, device="cuda"), torch.full((n, hk, room), 10, dtype=torch.int32, device="cuda"))
    lengths = _i32(held)
    left = sh.mass_evict(*src, lengths, keep=keep, recent=recent, into=into)
    assert left.tolist() == [min(c, keep) for c in held] and lengths.tolist() == held
    assert all(_same(a, b) for a, b in zip(src, own))
    assert sh.mass_evict(*own, lengths, keep=keep, recent=recent, left=lengths) is lengths and lengths.tolist() == left.tolist()
    for i, c in enumerate(held):
        for h in range(hk):
            stay, holes, moved = mr.evict(mass[i, h, :max(c, 0)].tolist(), positions[i, h, :max(c, 0)].tolist(), keep, recent)
            at = torch.tensor(stay, dtype=torch.int64, device="cuda")
            for x, y, fill in zip(src, into, (7, 8, 9, 10)):
                assert _same(y[i, h, :len(stay)], x[i, h, at]) and (y[i, h, len(stay):] == fill).all()
            for x, y in zip(src, own):
                want = x[i, h].clone()
                want[holes] = x[i, h, moved]
                assert _same(y[i, h], want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_run_together(dtype):
    """A batch shares a prefix, reads prompts, and decodes with evictions: every step against what its cache really holds."""
    sh, rnd, dt = _sh(), _rnd(3), DT[dtype]
    n, hk, g, d, slots, keep, recent = 3, 2, 2, 64, 48, 40, 8
    pk, pv = rnd(1, hk, 33, d, dtype=dt), rnd(1, hk, 33, d, dtype=dt)
    state = [torch.zeros(n, hk, slots, d, dtype=dt, device="cuda"), torch.zeros(n, hk, slots, d, dtype=dt, device="cuda"),
             torch.zeros(n, hk, slots, device="cuda"), torch.zeros(n, hk, slots, dtype=torch.int32, device="cuda")]
    counts = [48, 5, 30]
    starts = _i32([0, 48, 53, 83])
    lengths, seen = _i32([0, 0, 0]), _i32([0, 0, 0])
    old = [x.clone() for x in state]
    q, kn, vn = rnd(83, hk * g, d, dtype=dt), rnd(83, hk, d, dtype=dt), rnd(83, hk, d, dtype=dt)
    prior = sh.context_attention(q, pk, pv, partial=True)
    out = sh.mass_prefill(q, kn, vn, starts, lengths, *state, seen, prior=prior)
    a = 0
    for i, c in enumerate(counts):
        _check_sequence(old, state, i, 0, c, q[a:a + c], kn[a:a + c], vn[a:a + c], out[a:a + c], 0, g, dt, PROMPT, tuple(x[a:a + c] for x in prior))
        a += c
    lengths += _i32(counts)
    seen += _i32(counts)
    held = list(counts)
    for step in range(20):
        if max(held) == slots:
            was, before = [x.clone() for x in state], list(held)
            sh.mass_evict(*state, lengths, keep=keep, recent=recent, left=lengths)
            held = [min(c, keep) for c in held]
            assert lengths.tolist() == held
            for i in range(n):
                for h in range(hk):
                    _, holes, moved = mr.evict(was[2][i, h, :before[i]].tolist(), was[3][i, h, :before[i]].tolist(), keep, recent)
                    for x, y in zip(was, state):
                        want = x[i, h].clone()
                        want[holes] = x[i, h, moved]
                        assert torch.equal(y[i, h], want)
                    newest = set(range(int(seen[i]) - min(recent, held[i]), int(seen[i])))
                    assert newest <= set(state[3][i, h, :held[i]].tolist())
        q, kn, vn = rnd(n, hk * g, d, dtype=dt), rnd(n, hk, d, dtype=dt), rnd(n, hk, d, dtype=dt)
        prior = sh.context_attention(q, pk, pv, partial=True)
        old = [x.clone() for x in state]
        out = sh.mass_decode(q, kn, vn, lengths, *state, seen, prior=prior)
        for i in range(n):
            _check_sequence(old, state, i, held[i], 1, q[i:i + 1], kn[i:i + 1], vn[i:i + 1], out[i:i + 1], int(seen[i]), g, dt, STEP,
                            tuple(x[i:i + 1] for x in prior))
        lengths += 1
        seen += 1
        held = [c + 1 for c in held]
