"""Calls of the shared contexts and of the cache with accumulated weights that lie at the edge of what they take."""
import pytest
import torch

from test_gpu_mass import DT, INF, NAN, PROMPT, STEP, _check_sequence, _i32, _rnd, _same, _sh

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("partial", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_no_contexts(dtype, partial):
    """A batch without contexts: all rows belong to nobody."""
    sh, dt, tokens = _sh(), DT[dtype], 6
    q, k = _rnd(1)(tokens, 4, 64, dtype=dt), torch.empty(0, 2, 5, 64, dtype=dt, device="cuda")
    odt = torch.float32 if partial else dt
    for at in (0, 3, tokens):
        for lengths in (None, _i32([])):
            # (whoever asks for memory of these sizes next gets it as it is here)
            left = [torch.full((tokens, 4, 64), 7.0, dtype=odt, device="cuda"), torch.full((tokens, 4), 7.0, device="cuda")]
            del left
            out, lse = sh.context_attention(q, k, k, _i32([at]), lengths, partial=partial)
            assert out.dtype is odt and (out == 0).all() and (lse == -INF).all()
    out, lse = torch.full((tokens, 4, 64), 7.0, dtype=odt, device="cuda"), torch.full((tokens, 4), 7.0, device="cuda")
    sh.context_attention(q, k, k, _i32([2]), partial=partial, out=out, lse=lse)
    assert (out == 7).all() and (lse == 7).all()


def _step(cache, rnd, dt, g, n):
    """One token of each sequence, every one against what its cache really holds."""
    hk, slots, d = cache.k.shape[1:]
    q, k, v = rnd(n, hk * g, d, dtype=dt), rnd(n, hk, d, dtype=dt), rnd(n, hk, d, dtype=dt)
    held, seen = cache.lengths.tolist(), cache.seen.tolist()
    old = [x.clone() for x in (cache.k, cache.v, cache.mass, cache.positions)]
    out = cache.decode(q, k, v)
    for i, c in enumerate(held):
        if 0 <= c < slots:
            _check_sequence(old, (cache.k, cache.v, cache.mass, cache.positions), i, c, 1, q[i:i + 1], k[i:i + 1], v[i:i + 1], out[i:i + 1], seen[i], g, dt, STEP)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("longest,counts,lengths", [(20, [33, 5, 0], [0, 5, 0]), (35, [70, 5, 0], [0, 5, 0])])
def test_a_chunk_without_room_is_not_counted(dtype, longest, counts, lengths):
    """A `longest` that is too small: whoever the kernels leave out is not taken to hold rows.  (In the cache itself, in one of the chunk's size.)"""
    sh, rnd, dt, n, hk, g, d = _sh(), _rnd(longest), DT[dtype], 3, 2, 2, 64
    cache = sh.MassCache(n, hk * g, hk, d, 24, 6, 8, dtype=dtype)
    for x in (cache.k, cache.v, cache.mass):                              # what an earlier user has left
        x.fill_(NAN)
    starts, total = [0, counts[0], counts[0] + counts[1], sum(counts)], sum(counts)
    q, k, v = (rnd(total, x, d, dtype=dt) for x in (hk * g, hk, hk))
    out = cache.prefill(q, k, v, _i32(starts), longest=longest)
    assert (out[:counts[0]] == 0).all() and out[counts[0]:].isfinite().all()
    assert cache.lengths.tolist() == lengths and cache.seen.tolist() == lengths
    for _ in range(3):
        _step(cache, rnd, dt, g, n)
    cache.evict()
    assert cache.lengths.tolist() == [x + 3 for x in lengths]


def test_replayed_steps_stop_at_the_last_slot():
    """A captured step that is replayed past the spare slots: full sequences take no part and stay as they are."""
    sh, rnd, dt, n, hk, g, d = _sh(), _rnd(1), torch.bfloat16, 2, 2, 2, 64
    cache = sh.MassCache(n, hk * g, hk, d, 24, 6, 8, dtype="bf16")
    q, k, v = (rnd(n, x, d, dtype=dt) for x in (hk * g, hk, hk))
    cache.decode(q, k, v)
    cache.lengths.copy_(_i32([0, 20])), cache.seen.copy_(_i32([0, 70]))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.decode(q, k, v)
    for _ in range(15):
        graph.replay()
    assert cache.lengths.tolist() == [15, 32] and cache.seen.tolist() == [15, 82]
    full = [x[1].clone() for x in (cache.k, cache.v, cache.mass, cache.positions)]
    for _ in range(3):
        graph.replay()
    assert cache.lengths.tolist() == [18, 32] and cache.seen.tolist() == [18, 82]
    assert all(torch.equal(a, b[1]) for a, b in zip(full, (cache.k, cache.v, cache.mass, cache.positions)))
    cache.evict()
    assert cache.lengths.tolist() == [18, 24] and sorted(cache.positions[1, 0, :24].tolist())[-6:] == list(range(76, 82))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_longest_chunk_is_looked_up(dtype):
    """Without `longest` a batch is treated as with it: what stays does not depend on how many sequences share a call."""
    sh, dt, n, hk, g, d = _sh(), DT[dtype], 6, 2, 2, 64
    sides = []
    for given in (True, False):
        rnd = _rnd(7)
        cache = sh.MassCache(n, hk * g, hk, d, 24, 6, 16, dtype=dtype)
        cache.lengths[4] = -1
        got = []
        for counts in ([9, 10, 0, 3, 5, 1], [10, 10, 10, 10, 0, 10], [10, 1, 0, 0, 0, 10], [9, 9, 9, 0, 0, 0], [41, 3, 0, 0, 0, 0], [4, 4, 4, 4, 4, 4]):
            starts = [1]
            for x in counts:
                starts.append(starts[-1] + x)
            q, k, v = (rnd(starts[-1] + 2, x, d, dtype=dt) for x in (hk * g, hk, hk))
            options = dict(longest=max(counts)) if given else {}
            got.append(cache.prefill(q, k, v, _i32(starts), **options))
        sides.append(got + [cache.lengths, cache.seen, cache.k, cache.v, cache.mass, cache.positions])
    for a, b in zip(*sides):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_a_cache_of_the_chunks_own_size_holds_anything_at_first(dtype):
    """New memory is filled with NaN (and the largest integers): nothing of the cache in which a long chunk is read counts before it is written."""
    sh, dt, n, hk, g, d = _sh(), DT[dtype], 4, 2, 3, 64
    sides = []
    for poisoned in (False, True):
        rnd = _rnd(11)
        cache = sh.MassCache(n, hk * g, hk, d, 24, 6, 16, dtype=dtype)
        got = []
        torch.use_deterministic_algorithms(poisoned, warn_only=True)      # (with it, torch fills what it allocates)
        try:
            for counts in ([70, 1, 0, 33], [2, 0, 0, 90], [200, 200, 200, 1]):
                starts = [0]
                for x in counts:
                    starts.append(starts[-1] + x)
                q, k, v = (rnd(starts[-1], x, d, dtype=dt) for x in (hk * g, hk, hk))
                got.append(cache.prefill(q, k, v, _i32(starts), longest=max(counts)))
        finally:
            torch.use_deterministic_algorithms(False)
        sides.append(got + [cache.lengths, cache.seen, cache.k, cache.v, cache.mass, cache.positions])
    for a, b in zip(*sides):
        assert a.isfinite().all() and torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,hk,g,slots,held", [(3, 2, 4, 300, [299, 100, 64]), (1, 1, 4, 12000, [11990]), (40, 8, 2, 500, [480] * 40), (5, 3, 1, 100, [99, 0, 50, 7, 98])])
def test_a_prior_that_is_not_finite(dtype, n, hk, g, slots, held):
    """It shows in its own elements.  All others, and the masses, are the same bits: the keys are not gone over again for it.  (One CTA or a cluster a
    unit, a unit dealt out and merged; weights added by a launch of their own, by the unit, from shared memory.)"""
    sh, rnd, dt, d = _sh(), _rnd(slots), DT[dtype], 64
    q, k, v = (rnd(n, x, d, dtype=dt) for x in (hk * g, hk, hk))
    state = [rnd(n, hk, slots, d, dtype=dt), rnd(n, hk, slots, d, dtype=dt), torch.ones(n, hk, slots, device="cuda"), torch.zeros(n, hk, slots, dtype=torch.int32, device="cuda")]
    for odt in (torch.float32, dt):
        prior, lse = rnd(n, hk * g, d, dtype=odt), torch.full((n, hk * g), 5.0, device="cuda")
        bad = prior.clone()
        bad[0, 1, 3], bad[0, 2, 63], bad[n - 1, 0, 0] = NAN, INF, -INF
        runs = []
        for p in (prior, bad):
            now = [x.clone() for x in state]
            runs.append([sh.mass_decode(q, k, v, _i32(held), *now, _i32(held), prior=(p, lse))] + now)
        odd = ~bad.isfinite()
        assert torch.equal(runs[0][0][~odd], runs[1][0][~odd])
        assert _same(runs[1][0][odd], bad[odd].to(dt))
        for a, b in zip(runs[0][1:], runs[1][1:]):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("log", [NAN, INF, -INF])
def test_a_prior_whose_log_is_not_finite(dtype, log):
    """NaN and infinity take their row with them, and the masses of its key head; minus infinity is a prior that has seen nothing."""
    sh, rnd, dt, n, hk, g, d, slots = _sh(), _rnd(8), DT[dtype], 2, 2, 2, 128, 400
    q, k, v = (rnd(n, x, d, dtype=dt) for x in (hk * g, hk, hk))
    state = [rnd(n, hk, slots, d, dtype=dt), rnd(n, hk, slots, d, dtype=dt), torch.ones(n, hk, slots, device="cuda"), torch.zeros(n, hk, slots, dtype=torch.int32, device="cuda")]
    held, prior, lse = [399, 20], rnd(n, hk * g, d, dtype=torch.float32), torch.full((n, hk * g), 4.0, device="cuda")
    odd = lse.clone()
    odd[0, 1] = log
    if log == -INF:
        prior[0, 1] = NAN
    runs = []
    for x in (None, lse, odd):
        now = [t.clone() for t in state]
        runs.append([sh.mass_decode(q, k, v, _i32(held), *now, _i32(held), prior=None if x is None else (prior, x))] + now)
    (alone, _, _, _, _), (clean, _, _, mass, _), (out, _, _, got, _) = runs
    others = torch.ones(n, hk * g, dtype=torch.bool, device="cuda")
    others[0, 1] = False
    assert torch.equal(out[others], clean[others])
    assert torch.equal(got[1], mass[1]) and torch.equal(got[0, 1], mass[0, 1])
    if log == -INF:
        assert torch.equal(out[0, 1], alone[0, 1])
    else:
        assert out[0, 1].isnan().all() and got[0, 0, :400].isnan().all()


@pytest.mark.parametrize("dtype,tokens,held", [("bf16", 1024, 1000), ("f16", 64, 3000)])
def test_rows_that_a_prior_spoils_are_not_computed_again(dtype, tokens, held):
    """A log that is NaN makes its row NaN, whatever the keys are: going over them again, a row by a warp (30 to 100 times the whole call's time
    here), could change nothing.  (One CTA an item; items dealt out and merged.)"""
    sh, rnd, dt, hk, g, d = _sh(), _rnd(tokens), DT[dtype], 8, 4, 128
    q, k, v = (rnd(tokens, x, d, dtype=dt) for x in (hk * g, hk, hk))
    slots = held + tokens
    state = [rnd(1, hk, slots, d, dtype=dt), rnd(1, hk, slots, d, dtype=dt), torch.ones(1, hk, slots, device="cuda"), torch.zeros(1, hk, slots, dtype=torch.int32, device="cuda")]
    prior, lse = rnd(tokens, hk * g, d, dtype=torch.float32), torch.full((tokens, hk * g), 3.0, device="cuda")
    odd = lse.clone()
    odd[:, 5] = NAN
    outs, times = [], []
    for x in (lse, odd):
        call = lambda: sh.mass_prefill(q, k, v, _i32([0, tokens]), _i32([held]), *state, _i32([held]), prior=(prior, x), out=out)
        out, us = torch.empty_like(q), []
        for _ in range(6):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record(), call(), b.record()
            torch.cuda.synchronize()
            us.append(a.elapsed_time(b) * 1000)
        outs.append(out), times.append(min(us))
    others = [h for h in range(hk * g) if h != 5]
    assert torch.equal(outs[0][:, others], outs[1][:, others]) and outs[1][:, 5].isnan().all()
    assert times[1] < 4 * times[0] + 100, times


def test_captured_chunks_without_longest():
    """Under capture nothing can be looked up: all tokens are the bound.  Replays read starts and lengths as they are then."""
    sh, rnd, dt, n, hk, g, d = _sh(), _rnd(3), torch.float16, 3, 2, 2, 64
    cache = sh.MassCache(n, hk * g, hk, d, 40, 6, 16, dtype="f16")
    q, k, v = (rnd(12, x, d, dtype=dt) for x in (hk * g, hk, hk))
    starts = _i32([0, 4, 8, 12])
    cache.prefill(q, k, v, starts)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = cache.prefill(q, k, v, starts)
    want = [4, 4, 4]
    for at in ([0, 12, 12, 12], [1, 3, 9, 11], [0, 0, 5, 12]):
        starts.copy_(_i32(at))
        old = [x.clone() for x in (cache.k, cache.v, cache.mass, cache.positions)]
        graph.replay()
        for i in range(n):
            a, b = at[i], at[i + 1]
            if a < b:
                _check_sequence(old, (cache.k, cache.v, cache.mass, cache.positions), i, want[i], b - a, q[a:b], k[a:b], v[a:b], out[a:b], want[i], g, dt, PROMPT)
            want[i] += b - a
        assert cache.lengths.tolist() == want and cache.seen.tolist() == want
