"""Calls of the shared contexts and of the cache with accumulated weights that lie at the edge of what they take."""
import pytest
import torch

from test_gpu_mass import DT, INF, NAN, STEP, _check_sequence, _i32, _rnd, _sh

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
