"""The bookkeeping of the example's paged cache, on the CPU: what the attention is told that sequences have in common is what their tables share."""
import importlib.util
import os

import pytest

spec = importlib.util.spec_from_file_location("decoder_attention", os.path.join(os.path.dirname(__file__), "..", "examples", "decoder_attention.py"))
example = importlib.util.module_from_spec(spec)
spec.loader.exec_module(example)
PAGE = 16


def make(sequences, max_kv=200):
    return example.PagedCache(sequences, max_kv, 1, 16, 8, PAGE, device="cpu")


def shared_by(cache):
    """{sequence: (first sequence of its group, keys in common)} as ptq_paged_attention_shared reads groups, of sequences that hold something."""
    cu, shared = cache.groups_device.tolist(), cache.shared_device.tolist()
    assert len(cu) == len(shared) + 1 and all(a <= b for a, b in zip(cu, cu[1:])) and cu[0] >= 0 and cu[-1] <= len(cache.lens)
    return {s: (a, n) for a, b, n in zip(cu, cu[1:], shared) for s in range(a, b) if n > 0 and b - a > 1 and cache.lens[s] > 0}


def check(cache, want):
    """Sequences in `want` go on behind what they share, and no other."""
    got = shared_by(cache)
    for s, (first, n) in got.items():
        assert cache.lens[first] >= n and cache.lens[s] >= n
        assert cache.table[s, :n // PAGE].tolist() == cache.table[first, :n // PAGE].tolist(), (s, first)
    assert sorted(got) == sorted(want)


def forked(length=64):
    cache = make(8)
    cache.extend([length, 0, 0, 0, 0, 2 * length, 0, 0])
    cache.fork([[0, 1, 2, 3, 4], [5, 6, 7]])
    cache.extend([1] * 8)
    return cache


def test_forks_share_what_they_have_in_common():
    check(forked(), range(8))


@pytest.mark.parametrize("prompt", [1, 5, 64, 150])
@pytest.mark.parametrize("gone,alone", [(0, [0]), (2, [2, 3, 4]), (3, [3, 4]), (4, [4]), (1, [0, 1]), (6, [5, 6, 7])])
def test_a_slot_taken_by_another_sequence(gone, alone, prompt):
    """Of a family cut in two the longer part goes on behind the prefix (of two as long the first), the others by themselves; a part of one is by itself."""
    cache = forked()
    groups = cache.groups_device
    cache.release(gone)
    check(cache, [s for s in range(8) if s != gone])          # (an empty slot in between is no matter)
    new = [0] * 8
    new[gone] = prompt
    cache.extend(new)
    check(cache, [s for s in range(8) if s not in alone])
    assert cache.groups_device is groups                      # in place: a graph that was captured goes on reading it
    cache.extend([1] * 8)
    check(cache, [s for s in range(8) if s not in alone])
    cache.compact()
    check(cache, [s for s in range(8) if s not in alone])


def test_all_of_a_family_gone_and_its_slots_taken():
    cache = forked()
    for s in range(5):
        cache.release(s)
    check(cache, [5, 6, 7])
    cache.extend([80, 70, 0, 0, 90, 0, 0, 0])
    check(cache, [5, 6, 7])
    cache.release(0)
    cache.release(1)
    cache.release(4)
    cache.extend([64, 0, 0, 0, 0, 0, 0, 0])
    cache.fork([[0, 1, 2]])                                    # (from now on this is what is shared)
    check(cache, [0, 1, 2])


def test_pages_are_freed_once():
    cache = forked()
    for s in (0, 2, 4, 1, 3):
        cache.release(s)
    cache.extend([30, 0, 100, 0, 0, 0, 0, 0])
    used = [p for p, n in enumerate(cache.users) if n]
    assert sorted(used + cache.free) == list(range(len(cache.users)))
    for s in (5, 6, 7, 0, 2):
        cache.release(s)
    assert not any(cache.users) and sorted(cache.free) == list(range(len(cache.users)))


def test_a_graph_of_before_a_second_fork_goes_on_reading_what_is_so():
    """It has the tensors' addresses: they stay what they are, or stay there and say that nothing is shared."""
    cache = forked()
    cache.extend([15] * 8)                                     # (whole pages: nothing is copied on a device)
    groups, shared = cache.groups_device, cache.shared_device
    at = groups.data_ptr(), shared.data_ptr()
    for s in (1, 2, 3, 4, 6, 7):
        cache.release(s)
    cache.fork([[0, 1, 2], [5, 6]])                            # as many families: in place
    assert cache.groups_device is groups and cache.shared_device is shared
    check(cache, [0, 1, 2, 5, 6])
    for s in (1, 2, 6):
        cache.release(s)
    cache.fork([[5, 6, 7]])
    check(cache, [5, 6, 7])
    assert cache.groups_device is not groups and shared.tolist() == [0] * 4
    del groups, shared
    taken = [cache._put([7] * n) for n in (4, 5) for _ in range(50)]
    assert not {t.data_ptr() for t in taken} & set(at)         # nobody else has got their memory
