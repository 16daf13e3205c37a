"""The example's cache of keys and values: what has no room is refused, and nothing else is touched."""
import pytest
import torch

from paper_2604_16855_amd.attention_layer import Cache

S, ROOM, HK, D = 3, 10, 2, 8


def _cu(counts):
    return torch.tensor([0] + list(counts)).cumsum(0).to(torch.int32)


def _tokens(counts, first):
    """Keys that name their sequence and place, values their negatives."""
    k = torch.tensor([100.0 * s + f + i for s, (n, f) in enumerate(zip(counts, first)) for i in range(n)])
    K = k[:, None, None].expand(-1, HK, D).contiguous()
    return K, -K


def _holds(cache, used):
    """Sequence s holds its first used[s] tokens in order."""
    assert cache.used.tolist() == used
    assert cache.cu.tolist() == [ROOM * s for s in range(S + 1)] and cache.K.shape == cache.V.shape == (S * ROOM, HK, D)
    for s, n in enumerate(used):
        want, _ = _tokens([0] * s + [n], [0] * (s + 1))
        assert torch.equal(cache.K[s * ROOM:s * ROOM + n], want) and torch.equal(cache.V[s * ROOM:s * ROOM + n], -want)


def _filled(counts):
    cache = Cache(S, ROOM, HK, D, torch.float32, "cpu")
    cache.append(*_tokens(counts, [0] * S), _cu(counts))
    return cache


def test_prompts_then_tokens_up_to_the_room():
    cache, used = _filled([7, 0, 3]), [7, 0, 3]
    _holds(cache, used)
    for counts in ([1, 1, 1], [0, 4, 2], [1, 0, 0], [1, 5, 4]):
        cache.append(*_tokens(counts, used), _cu(counts))
        used = [a + b for a, b in zip(used, counts)]
        _holds(cache, used)
    assert used == [10, 10, 10]


@pytest.mark.parametrize("have,counts", [([10, 2, 0], [1, 1, 1]), ([4, 10, 5], [0, 1, 0]), ([1, 2, 9], [3, 0, 2]),
                                         ([1, 1, 1], [0, 0, 20])])
def test_a_sequence_without_room_is_refused(have, counts):
    """In front, in the middle and at the end of the cache, before anything is written."""
    cache = _filled(have)
    K, V = cache.K.clone(), cache.V.clone()
    with pytest.raises(ValueError, match="room"):
        cache.append(*_tokens(counts, have), _cu(counts))
    _holds(cache, have)
    assert torch.equal(cache.K.nan_to_num(), K.nan_to_num()) and torch.equal(cache.V.nan_to_num(), V.nan_to_num())
    less = [min(n, ROOM - h) for n, h in zip(counts, have)]  # (what has room still joins)
    cache.append(*_tokens(less, have), _cu(less))
    _holds(cache, [h + n for h, n in zip(have, less)])


def test_many_steps_of_one_token():
    """However the steps are counted on the host, the last that fits is taken and the next one refused."""
    cache = _filled([2, 2, 2])
    for i in range(2, ROOM):
        cache.append(*_tokens([1] * S, [i] * S), _cu([1] * S))
        _holds(cache, [i + 1] * S)
    with pytest.raises(ValueError, match="room"):
        cache.append(*_tokens([1] * S, [ROOM] * S), _cu([1] * S))
    _holds(cache, [ROOM] * S)


def test_offsets_that_do_not_fit_the_tokens_are_refused():
    cache = _filled([2, 2, 2])
    K, V = _tokens([3, 3, 3], [2, 2, 2])
    for cu in (_cu([3, 3]), _cu([3, 3, 3, 0])):
        with pytest.raises(ValueError):
            cache.append(K, V, cu)
    with pytest.raises(ValueError):
        cache.append(K, V[:8], _cu([3, 3, 3]))
    _holds(cache, [2, 2, 2])


def test_without_the_hosts_look_nothing_is_written_outside_a_sequence():
    """A replayed graph does not ask the host: tokens without room, or outside the offsets, go nowhere."""
    cache = _filled([9, 5, 10])
    K, V = _tokens([3, 1, 2], [9, 5, 10])
    cache._write(K, V, _cu([3, 1, 2]))
    cache.used.copy_(torch.tensor([10, 6, 10], dtype=torch.int32))
    _holds(cache, [10, 6, 10])
    before = cache.K.clone()
    cache._write(K, V, torch.tensor([2, 2, 2, 2], dtype=torch.int32))
    assert torch.equal(cache.K.nan_to_num(), before.nan_to_num())
