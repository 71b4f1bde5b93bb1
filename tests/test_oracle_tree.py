"""CPU pins of the oracle of drafted tokens: against hand-worked cases, against the causal oracle where a tree is a chain, and the law that verification keeps: the
next tokens are distributed as the target has it, whatever was drafted."""
import itertools

import numpy as np
import pytest

from oracle import paged as op
from oracle import tree as ot


def test_fit_by_hand():
    table = np.array([[7, 3, -1], [5, -1, -1], [8, 6, -1]])
    held, free = [2, 1, 2], [1, 2, 4, -1, -1]
    # 16 to a page: sequence 0 keeps its pages, 1 grows into a second and third, 2 is over
    got = ot.fit([20, 16, 0], [3, 20, 0], 16, table, held, free, 3, 25)
    assert got[0] == [0, 3, 23, 23] and got[1] == [23, 36, 0]
    assert got[2][:3] == [3 * 16 + 4, 3 * 16 + 5, 3 * 16 + 6] and got[3][:4] == [20, 21, 22, 16]
    # (8 comes off the stack first: the last page that went back was the first of sequence 2)
    assert held == [2, 3, 0] and table[1].tolist() == [5, 8, 6] and got[4] == 3 and free[:3] == [1, 2, 4]
    assert got[2][3] == 8 * 16 and got[2][19] == 6 * 16 and got[2][23:] == [-1, -1] and got[3][23:] == [0, 0]
    # ... and more than there is
    got = ot.fit([23, 36, 0], [0, 0, 100], 16, table, held, free, 3, 100)
    assert held == [2, 3, 3] and got[4] == 0 and got[2][48:] == [-1] * 52            # (a row of three entries)
    held2 = [0]
    t2 = np.full((1, 4), 9)
    got = ot.fit([0], [50], 16, t2, held2, [3, 1], 2, 50)
    assert held2 == [2] and t2.tolist() == [[1, 3, -1, -1]] and got[4] == -2 and got[2][31] == 3 * 16 + 15 and got[2][32] == -1


def test_a_chain_is_causal():
    g = np.random.default_rng(1)
    k, v, q = g.normal(size=(5, 4, 2, 8)), g.normal(size=(5, 4, 2, 8)), g.normal(size=(9, 4, 8))
    table, starts, lengths = np.array([[2, 0, 4, -1], [1, 3, -1, -1]]), [0, 6, 9], [11, 3]
    seen, depths = zip(*[ot.ancestors([i - 1 for i in range(n)]) for n in (6, 3)])
    mask = ot.masks([s for x in seen for s in x], 1)
    for window in (0, 4):
        w = [ot.ancestors([i - 1 for i in range(n)], window)[0] for n in (6, 3)]
        mask = ot.masks([s for x in w for s in x], 1)
        got = ot.attend(q, k, v, table, starts, lengths, mask, [d for x in depths for d in x], window)
        want = op.attend(q, k, v, table, starts, lengths, None, True, window)
        assert np.allclose(got[0], want[0], atol=1e-14) and np.allclose(got[1], want[1], atol=1e-14)


def test_masks_by_hand():
    seen, depths = ot.ancestors([-1, 0, 0, 1, 3, 9, 5])
    assert seen == [[0], [1, 0], [2, 0], [3, 1, 0], [4, 3, 1, 0], [5], [6, 5]] and depths == [0, 1, 1, 2, 3, 0, 1]
    assert ot.ancestors([-1, 0, 0, 1, 3, 9, 5], 2)[0][4] == [4, 3]
    assert ot.masks([[0, 63], [64, 130], []], 2).view(np.uint64).tolist() == [[(1 << 63) | 1, 0], [0, 1], [0, 0]]


@pytest.mark.parametrize("drafted", [True, False])
def test_the_next_token_is_the_targets(drafted):
    """One node, its children drawn from q (or fixed): the token behind the root (the child that stands, or the next token) has the law p.  The random numbers run over
    a fine grid of midpoints; with two children and three random numbers a cell is 1 / 16 wide, and the law is met to the share of cells that borders cut."""
    p, q = np.array([0.5, 0.2, 0.3]), np.array([0.25, 0.5, 0.25])
    n = 16
    grid = (np.arange(n) + 0.5) / n
    law = np.zeros(3)
    for x, y in itertools.product(range(3), range(3)) if drafted else [(1, 0)]:
        weight = (q[x] * q[y] if drafted else 1.0) / n ** 3
        target, draft = np.tile(p, (3, 1)), np.tile(q, (3, 1)) if drafted else None
        for u0, u1, r in itertools.product(grid, grid, grid):
            path, _, following = ot.verify(target, draft, [0, x, y], [-1, 0, 0], [0, 3], [0, u0, u1], [r], 2)
            law[[x, y][path[0][1] - 1] if path[0][1] > 0 else following[0]] += weight
    assert np.abs(law - p).max() < 2 / n, law


def test_compact_reads_before_it_writes():
    cache = np.arange(12).reshape(3, 4, 1) * 10
    table = np.array([[2, 0]])
    before = cache.copy()
    ot.compact(cache, table, np.array([6]), np.array([[0, 2, 3, 4]]), np.array([4]))         # past 2: positions 4, 5, 6 to 3, 4, 5
    at = lambda c, p: c[table[0, p // 4], p % 4, 0]  # noqa: E731
    assert [at(cache, p) for p in range(8)] == [at(before, p) for p in (0, 1, 2, 4, 5, 6, 6, 7)]
    assert (cache[1] == before[1]).all()
