"""GPU parity of a round's layout (rows, pages, positions, slots) with the same laid out token by token."""

import numpy as np
import pytest
import torch

from _batch import PAGE, i32, lay_out
from paper_2608_20397_amd import nexus as N

pytestmark = pytest.mark.gpu


def run(cached, fresh, n_free, max_tokens, stride, seed=0, capacity=None):
    rng = np.random.default_rng(seed)
    held = [max(0, -(-min(c, PAGE * stride) // PAGE)) for c in cached]
    order = rng.permutation(sum(held) + max(n_free, 0) + 5)
    maps = np.full((len(cached), stride), -7)
    at = 0
    for b, h in enumerate(held):
        maps[b, :h] = order[at:at + h]
        at += h
    free = order[at:][:capacity]
    dmaps = i32(maps)
    args = (i32(cached), i32(fresh), i32(free), i32([n_free]))
    rows = N.batch_pages(dmaps, *args, max_tokens)
    torch.cuda.synchronize()
    want = lay_out(cached, fresh, free, n_free, maps, max_tokens)
    for name, got, ref in zip(("maps", "q_start", "seq_len", "pos", "slot", "n_left"),
                              (dmaps, rows.q_start, rows.seq_len, rows.pos, rows.slot, rows.n_left), want):
        assert np.array_equal(got.cpu().numpy().reshape(-1), np.reshape(ref, -1)), name
    assert torch.equal(args[2].cpu(), torch.tensor(free, dtype=torch.int32))     # the list itself stays


@pytest.mark.parametrize("cached,fresh,n_free,max_tokens,stride", [
    ([0], [1], 1, 1, 1), ([0], [1], 0, 1, 1), ([15], [1], 0, 4, 1), ([16], [1], 3, 4, 2), ([0], [0], 3, 4, 2),
    ([5, 0, 16, 31], [1, 40, 0, 2], 10, 50, 4), ([5, 0, 16, 31], [1, 40, 0, 2], 3, 50, 4),
    ([5, 0, 16, 31], [1, 40, 0, 2], 2, 50, 4),                  # not enough for the second, the last refused with it
    ([0, 5, 0], [40, 1, 0], 2, 50, 4),                          # one that needs no page goes on
    ([-1, 3, 3], [4, -2, 4], 9, 20, 4),                         # lengths that are none
    ([60, 60], [4, 5], 9, 20, 4),                               # as long as a map row, and longer
    ([0, 0, 0], [10, 10, 10], 9, 25, 2),                        # rows past max_tokens
    ([0, 0, 0], [10, 100, 1], 9, 25, 8),                        # ... and what comes after them
    ([0, 0], [2 ** 31 - 1, 3], 9, 25, 8), ([2 ** 31 - 1, 1], [2 ** 31 - 1, 3], 9, 25, 8),
    ([0], [30], -4, 40, 4), ([0, 16], [17, 17], 100, 40, 4),
])
def test_small(cached, fresh, n_free, max_tokens, stride):
    run(cached, fresh, n_free, max_tokens, stride)


def test_free_count_above_the_list_is_clamped():
    run([0, 3], [33, 20], 50, 60, 4, capacity=4)


@pytest.mark.parametrize("n,top,n_free,seed", [(63, 5, 500, 1), (64, 40, 60, 2), (1024, 3, 5000, 3), (1025, 9, 300, 4),
                                               (4097, 2, 5000, 5), (8192, 2, 9000, 6), (300, 700, 20000, 7)])
def test_many(n, top, n_free, seed):
    rng = np.random.default_rng(seed)
    cached = rng.integers(0, 60, n).tolist()
    fresh = rng.integers(0, top + 1, n).tolist()
    for b in rng.integers(0, n, 3):
        cached[b] = -5
    run(cached, fresh, n_free, sum(fresh) + 77, (60 + top + 15) // 16, seed)
    run(cached, fresh, n_free, max(1, sum(fresh) // 2), (60 + top + 15) // 16, seed)


def test_a_page_that_is_none_gives_no_slot():
    """Numbers whose slots would pass 32 bits and come round to the cache, in the map and in the list."""
    maps = i32([[1 << 28, 3], [-1, 2], [1, (1 << 27) - 1]])
    rows = N.batch_pages(maps, i32([3, 2, 17]), i32([15, 1, 1]), i32([(1 << 27) + 4]), i32([1]), 17)
    pos, slot = rows.pos.tolist(), rows.slot.tolist()
    assert pos == list(range(3, 18)) + [2, 17]
    assert slot == [-1] * 16 + [((1 << 27) - 1) * 16 + 1] and rows.n_left.item() == 0


def test_refusals():
    m, c, f = i32(np.zeros((2, 4))), i32([1, 1]), i32([1, 1])
    free, n = i32(range(9)), i32([9])
    for call in (lambda: N.batch_pages(m, c, f[:1], free, n, 4), lambda: N.batch_pages(m[:1], c, f, free, n, 4),
                 lambda: N.batch_pages(m, c.long(), f, free, n, 4), lambda: N.batch_pages(m, c, f, free, n, 0),
                 lambda: N.batch_pages(m, c, f, free, i32([1, 2]), 4),
                 lambda: N.batch_pages(m, c, f, free, n, 4, out=N.BatchRows(i32([0, 0, 0]), c, i32([0] * 4),
                                                                           i32([0] * 4), i32([0]))),
                 lambda: N.batch_pages(m, c, f, free, n, 4, out=N.BatchRows(i32([0, 0, 0]), i32([0, 0]), i32([0] * 4),
                                                                           i32([0] * 4), n))):
        with pytest.raises(N.NexusError) as e:
            call()
        assert e.value.status == N.EINVAL


@pytest.mark.parametrize("cached,fresh,n_free,max_tokens,stride", [
    ([0], [40], 9, 32, 4), ([0], [33], 9, 32, 4), ([0], [100], 9, 50, 8), ([7], [26], 9, 25, 4),
    ([0, 0], [0, 40], 9, 32, 4), ([3, 0, 0], [-2, 40, 1], 9, 32, 4), ([-1, 0], [0, 33], 9, 32, 4),
    ([0, 5], [100, 1], 9, 50, 8), ([0, 5, 16], [100, 0, 0], 9, 50, 8), ([0, 5], [50, 1], 9, 50, 8),
    ([0, 0, 0], [0, 51, 3], 9, 50, 8), ([100], [51], 0, 50, 16),
])
def test_a_sequence_longer_than_the_launch(cached, fresh, n_free, max_tokens, stride):
    """More rows than the whole launch has, with none before them: refused, its map and the free list left as they are,
    and all that comes after it and has rows."""
    run(cached, fresh, n_free, max_tokens, stride)


@pytest.mark.parametrize("n_free", [0, 5])
def test_a_free_list_without_entries(n_free):
    """Every page is given out: sequences that need none go on, those that do are refused."""
    run([5, 15, 16, 3], [3, 1, 2, 1], n_free, 20, 4, capacity=0)
