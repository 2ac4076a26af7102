"""Pins of oracle/draft.py (CPU only)."""
import numpy as np
import pytest

import oracle
from oracle import draft as OD
from oracle import shared as OS


@pytest.mark.parametrize("pol", [[-1, 0, 0, -1, 0], [9, 4, 2, 5, 1], [7, 0, 0, 1, 0], [3, 1, 8, 2, 40]])
def test_a_chain_sees_what_single_steps_retain(pol):
    seg, T = np.array([3, 30, 2, 6]), 9
    parent = np.arange(-1, T - 1)
    for t in range(T):
        idx, n = oracle.retained((seg + [0, 0, 0, t])[None], np.array(pol))
        cached, nodes = OD.sees(seg, pol, parent, t)
        assert list(cached) + [seg.sum() - 1 + x for x in nodes] == list(idx[0, :n[0]])


def test_branches_do_not_see_each_other():
    parent = [-1, 0, 0, 1, 2, 4]
    seg, pol = np.array([2, 4, 0, 3]), [-1, 0, 0, -1, 0]
    assert [OD.sees(seg, pol, parent, t)[1] for t in range(6)] == [[0], [0, 1], [0, 2], [0, 1, 3], [0, 2, 4], [0, 2, 4, 5]]
    assert all(list(OD.sees(seg, pol, parent, t)[0]) == list(range(8)) for t in range(6))
    near = [-1, 0, 0, 2, 0]  # two outputs: a node and the one before it
    assert [OD.sees(seg, near, parent, t)[1] for t in range(6)] == [[0], [0, 1], [0, 2], [1, 3], [2, 4], [4, 5]]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [2, 50, 128])
def test_rotation(rot, interleaved):
    rng = np.random.default_rng(rot)
    freq = [int(x) for x in rng.integers(0, 2 ** 62, size=rot // 2)]
    x, y = rng.standard_normal((2, 128))
    turn = lambda z, p: OD.rotate(z, OD.turns(p, freq), rot, interleaved, 1.0)  # noqa: E731
    back = OD.rotate(turn(x, 77777), -OD.turns(77777, freq), rot, interleaved, 1.0)
    assert np.allclose(back, x, atol=1e-12) and np.array_equal(turn(x, 0), x)
    # products depend on the distance alone, however far
    assert np.isclose(turn(x, 10 ** 6 + 5) @ turn(y, 10 ** 6), turn(x, 5) @ turn(y, 0), atol=1e-9)
    assert np.array_equal(turn(x, 9)[rot:], x[rot:])


def test_reserve_keeps_the_pool_whole():
    rng = np.random.default_rng(3)
    for trial in range(60):
        B, cols, n_blocks, bs = 7, 12, 40, int(rng.choice([1, 4, 16]))
        held = rng.integers(0, 4, size=B)
        order = list(rng.permutation(n_blocks))
        table = np.full((B, cols), -1, dtype=np.int32)
        for b in range(B):
            for c in range(held[b]):
                table[b, c] = order.pop()
        st = dict(table=table, stack=order[:], ref=OS.recount(table, n_blocks), n_blocks=n_blocks)
        length = np.maximum(held * bs - rng.integers(0, bs + 1, size=B), 0)
        new = rng.integers(0, 6 * bs, size=B)
        per = int(new.max()) + 1 if trial % 2 else 0
        got = OD.reserve(st, length, new, bs, per, B * per + 1 if per else int(new.sum()) + 1, cols)
        named = st["table"][st["table"] >= 0]
        assert sorted(list(named) + st["stack"]) == list(range(n_blocks))
        assert np.array_equal(st["ref"], OS.recount(st["table"], n_blocks))
        kept = got["slot"][got["slot"] >= 0]
        assert len(set(kept)) == len(kept) == sum(int(x) for x in got["got"] if x > 0)


def test_accept():
    parent, token = [-1, 0, 0, 1, 2, 2], [5, 7, 8, 9, 1, 1]
    assert OD.accept(parent, token, [8, 0, 1, 0, 4, 3]) == ([0, 2, 4], 4)  # of equals the first
    assert OD.accept(parent, token, [7, 0, 1, 0, 4, 3]) == ([0, 1], 0)
    assert OD.accept(parent, token, [6, 0, 1, 0, 4, 3]) == ([0], 6)
    assert OD.accept(parent, [-1] + token[1:], [7] * 6) == ([], -1)
