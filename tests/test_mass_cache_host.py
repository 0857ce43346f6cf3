"""What the cache object does on the host: whom it counts, when it evicts and which calls it makes.  (The kernels are replaced by their rules of
who takes part; no device call is made.)"""
import pytest
import torch


@pytest.fixture
def made(monkeypatch):
    """The binding, with a list of the calls that a MassCache on the host has made."""
    from paper_2305_17118_b200 import binding as sh
    calls = []

    def prefill(q, k, v, starts, lengths, k_cache, *rest, out=None, **options):
        calls.append(("prefill", k_cache.shape[2], lengths.tolist()))
        return torch.zeros_like(q) if out is None else out

    def decode(q, k, v, lengths, k_cache, *rest, out=None, **options):
        calls.append(("decode", k_cache.shape[2], lengths.tolist()))
        return torch.zeros_like(q) if out is None else out

    def evict(k_cache, v_cache, mass, positions, lengths, *, keep, recent, into=None, left=None):
        calls.append(("evict", k_cache.shape[2], lengths.tolist()))
        now = lengths.clamp(max=keep)
        return now if left is None else left.copy_(now)

    for name, fake in (("mass_prefill", prefill), ("mass_decode", decode), ("mass_evict", evict)):
        monkeypatch.setattr(sh, name, fake)
    sh.calls = calls
    yield sh
    del sh.calls


def _cache(sh, sequences, budget, spare):
    return sh.MassCache(sequences, 4, 2, 64, budget, 2, spare, dtype="f16", device="cpu")


def _rows(tokens):
    t = lambda heads: torch.zeros(tokens, heads, 64, dtype=torch.float16)
    return t(4), t(2), t(2)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32)


def test_a_chunk_without_room_is_not_counted(made):
    cache = _cache(made, 4, 24, 8)
    cache.lengths.copy_(_i32([0, 30, -1, 5]))
    cache.seen.copy_(_i32([0, 90, 0, 7]))
    cache.prefill(*_rows(40), _i32([0, 33, 35, 38, 40]), longest=20)      # 33 rows into 32 slots; two into 30 held; an idle one; two
    assert made.calls == [("prefill", 32, [0, 30, -1, 5])]
    assert cache.lengths.tolist() == [0, 32, -1, 7] and cache.seen.tolist() == [0, 92, 0, 9]


def test_a_chunk_that_a_cache_of_its_own_has_no_room_for_is_not_counted(made):
    cache = _cache(made, 3, 24, 8)
    cache.lengths.copy_(_i32([30, 2, 3]))
    cache.seen.copy_(_i32([30, 2, 3]))
    cache.prefill(*_rows(120), _i32([0, 34, 100, 120]), longest=33)       # 24 + 33 slots
    assert [c[:2] for c in made.calls] == [("evict", 32), ("prefill", 57), ("evict", 57)]
    assert made.calls[2][2] == [24, 2, 23]
    assert cache.lengths.tolist() == [24, 2, 23] and cache.seen.tolist() == [30, 2, 23]


def test_starts_that_leave_the_tensor_count_as_the_kernels_take_them(made):
    cache = _cache(made, 3, 24, 8)
    cache.prefill(*_rows(10), _i32([-5, 4, 2, 50]), longest=8)
    assert cache.lengths.tolist() == [4, 0, 8] and cache.seen.tolist() == [4, 0, 8]


def test_a_token_without_room_is_not_counted(made):
    cache = _cache(made, 4, 24, 8)
    cache.lengths.copy_(_i32([32, 31, -1, 0]))
    cache.seen.copy_(_i32([50, 60, 0, 0]))
    for lengths, seen in (([32, 32, -1, 1], [50, 61, 0, 1]), ([32, 32, -1, 2], [50, 61, 0, 2])):
        cache.decode(*_rows(4))
        assert cache.lengths.tolist() == lengths and cache.seen.tolist() == seen


def test_the_longest_chunk_is_looked_up(made):
    """How many sequences share a call does not matter for when it evicts."""
    cache = _cache(made, 8, 100, 64)
    cache.lengths[5] = -1
    starts = _i32([3, 13, 13, 23, 33, 42, 92, 102, 105])                  # ten rows at most (fifty are an idle sequence's), some of nobody
    for _ in range(16):
        cache.prefill(*_rows(110), starts)
    assert [c[:2] for c in made.calls] == [("prefill", 164)] * 16
    cache.prefill(*_rows(110), starts)
    assert [c[:2] for c in made.calls[16:]] == [("evict", 164), ("prefill", 164)]


def test_a_call_without_rows_of_any_sequence_does_nothing(made):
    cache = _cache(made, 2, 10, 4)
    assert cache.prefill(*_rows(7), _i32([3, 3, 3])).shape == (7, 4, 64)
    assert made.calls == [] and cache.lengths.tolist() == [0, 0] and cache.seen.tolist() == [0, 0]


@pytest.mark.parametrize("starts", [[0, 7], [0, 3, 5, 7], [7]])
def test_prefill_refuses_starts_of_another_batch(made, starts):
    cache = _cache(made, 2, 10, 4)
    for longest in (None, 5):
        with pytest.raises(ValueError):
            cache.prefill(*_rows(7), _i32(starts), longest=longest)
    with pytest.raises(ValueError):
        cache.prefill(*_rows(7), torch.tensor([0, 3, 7]))                 # (not int32)
    assert made.calls == []
