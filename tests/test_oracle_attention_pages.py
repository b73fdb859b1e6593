"""Pins of the attention and page oracles on the CPU: against a softmax
written out with exact fractions of weights, closed forms and invariants."""
import math

import numpy as np
import pytest

from oracle.attention import attend, attend_row, visible
from oracle.pages import BOUNDS, OK, Pages


def test_visible_sets():
    assert visible(-1, 0, 0) == []
    assert visible(0, 0, 0) == [0]
    assert visible(4, 0, 3) == [0, 1, 2, 3, 4]
    assert visible(9, 3, 0) == [7, 8, 9]
    assert visible(9, 3, 2) == [0, 1, 7, 8, 9]
    assert visible(3, 3, 2) == [0, 1, 2, 3]
    assert visible(5, 1, 100) == [0, 1, 2, 3, 4, 5]


@pytest.mark.parametrize("planes", [1, 2])
def test_attend_row_by_hand(planes):
    """Weights 1 : 2 : 4 from scores 0, ln 2, ln 4, over pages 2 and 0."""
    pool = np.zeros((3, planes, 2, 1, 2))
    for j, (page, slot) in enumerate([(2, 0), (2, 1), (0, 0)]):
        pool[page, 0, slot, 0] = [j * math.log(2), 10.0 * j]
        if planes == 2:
            pool[page, 1, slot, 0] = [j * math.log(2), 10.0 * j]
    out, lse, spread, size = attend_row(pool, [2, 0], 2, np.array([1.0, 0.0]), 0, 1.0, 2)
    np.testing.assert_allclose(out, [(2 * math.log(2) + 8 * math.log(2)) / 7, (20 + 80) / 7])
    assert lse == pytest.approx(math.log(7)) and size == pytest.approx(math.log(4))
    # page 2 outside the pool: the third token alone is left
    out, lse, _, _ = attend_row(pool, [9, 0], 2, np.array([1.0, 0.0]), 0, 1.0, 2)
    np.testing.assert_allclose(out, [2 * math.log(2), 20.0])
    out, lse, _, _ = attend_row(pool, [-1, 3], 2, np.array([1.0, 0.0]), 0, 1.0, 2)
    assert (out == 0).all() and lse == -np.inf


def test_attend_positions():
    """The last new token of a request sits at its last position."""
    rng = np.random.default_rng(0)
    pool = rng.standard_normal((4, 2, 4, 2, 3))
    q = rng.standard_normal((5, 4, 3))
    got = attend(pool, [[0, 1], [2, 3]], [6, 2], [0, 2, 5], q, 2, 0.5, 3)
    assert sorted({t for t, _ in got}) == [0, 1, 2, 3, 4]
    want = attend_row(pool, [0, 1], 4, q[0, 3], 1, 0.5, 3)
    np.testing.assert_array_equal(got[0, 3][0], want[0])
    assert got[2, 0][1] == -np.inf                   # three new tokens in a request of two


def _state(seed, rows=6, stride=5, pages=40, P=4):
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, stride * P + 1, rows)
    tables = np.full((rows, stride), -1)
    perm = iter(rng.permutation(pages))
    for r, n in enumerate(lens):
        for j in range(-(-int(n) // P)):
            tables[r, j] = next(perm)
    s = Pages([0] * pages, tables, lens, P)
    assert s.count()[0] == OK
    return s


def _consistent(s):
    refs = list(s.refs)
    t = Pages(refs, s.tables, s.lens, s.P)
    assert t.count()[0] == OK and t.refs == refs


@pytest.mark.parametrize("seed", range(5))
def test_pages_stay_consistent(seed):
    s = _state(seed)
    s.free([1, 3])
    _consistent(s)
    st, pairs, want, bad = s.fork([0, 0], [1, 3])
    assert st == OK and len(pairs) == want
    _consistent(s)
    assert s.lens[1] == s.lens[0] and list(s.tables[1, :s.lens[0] // 4]) == list(s.tables[0, :s.lens[0] // 4])
    s.free([0], [max(0, s.lens[0] - 1)])
    if s.lens[1] < 20:
        st, pairs, _, _ = s.grow([1], [s.lens[1] + 1])
        assert st == OK and not pairs                # its partial page was its own already
    _consistent(s)
    s.free([2])
    live = sum(1 for c in s.refs if c)
    st, pairs, u, _ = s.compact()
    assert st == OK and u == live and all(c > 0 for c in s.refs[:u]) and not any(s.refs[u:])
    _consistent(s)
    assert s.compact()[1] == []


def test_pages_refusals():
    s = _state(1)
    s.lens[0] = 7
    before = (list(s.refs), s.tables.copy(), list(s.lens))
    assert s.fork([0, 0], [1, 1])[0] == BOUNDS and s.grow([0], [21])[0] == BOUNDS and s.grow([0], [6])[0] == BOUNDS
    assert before[0] == s.refs and (before[1] == s.tables).all() and before[2] == s.lens


def test_grow_copies_shared_partial_page():
    s = Pages([0] * 6, [[3, -1], [-1, -1]], [3, 0], 4)
    s.count()
    s.fork([0], [1])
    s.free([1], [0])
    s.tables[1, 0], s.lens[1] = 3, 2                 # a row that was cut inside a shared page
    s.count()
    assert s.refs[3] == 2
    assert s.grow([0, 1], [5, 3]) == (OK, [(3, 0), (3, 2)], 3, 0)
    assert s.refs == [1, 1, 1, 0, 0, 0] and s.tables.tolist() == [[0, 1], [2, -1]]
