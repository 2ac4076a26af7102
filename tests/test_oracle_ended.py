"""Pins of the oracle's rule for sequences that are not there (oracle/shared.py, step), CPU only."""
import copy

import numpy as np
import pytest

from oracle import shared as OS


@pytest.mark.parametrize("seed", range(4))
def test_step_as_if_the_absent_rows_were_not_in_the_batch(seed):
    rng = np.random.default_rng(seed)
    B, bs, steps = 9, 4, 20
    lo = np.arange(B) // 3 * 3
    seg = np.tile(np.array([[3, 12, 1, 5]], dtype=np.int32), (B, 1))
    seg[:, 3] += rng.integers(0, 9, 3)[np.arange(B) // 3].astype(np.int32)
    pol = np.tile(np.array([6, 2, 1, 5, 1], dtype=np.int32), (B, 1))
    length = seg.sum(axis=1) - 1
    max_blocks = int(-(-(length.max() + steps) // bs))
    n = B * max_blocks
    free = list(range(n))
    table = np.full((B, max_blocks), -1, dtype=np.int32)
    for b in range(B):
        for c in range(-(-int(length[b]) // bs)):
            table[b, c] = free.pop() if b == lo[b] else table[lo[b], c]
    st = {"table": table, "ref": OS.recount(table, n), "stack": free}
    live = np.ones(B, dtype=bool)
    for _ in range(steps):
        parent = np.where(rng.random(B) < 0.1, -1, lo + rng.integers(0, 3, B))
        OS.fork(st, parent)
        live = (parent >= 0) & live[parent]
        assert (st["table"][~live] == -1).all()
        alone = copy.deepcopy(st)
        alone["table"] = alone["table"][live]
        copied = OS.step(st, np.where(live[:, None], seg, 0), pol, bs)
        assert (copied[~live] == -2).all() and (copied[live] >= -1).all()
        assert np.array_equal(copied[live], OS.step(alone, seg[live], pol[live], bs))
        assert np.array_equal(st["table"][live], alone["table"]) and (st["table"][~live] == -1).all()
        assert np.array_equal(st["ref"], alone["ref"]) and st["stack"] == alone["stack"]
        assert np.array_equal(st["ref"], OS.recount(st["table"], n))
        seg[:, 3] += 1
