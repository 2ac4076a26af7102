"""Pins of the oracle of shared pages and shared prefixes (oracle/shared.py), CPU only."""
import copy

import numpy as np
import pytest

import oracle
from oracle import paged as OP
from oracle import shared as OS
from _shared import forked_state


def consistent(st):
    used = set(st["table"][st["table"] >= 0].ravel().tolist())
    assert np.array_equal(st["ref"], OS.recount(st["table"], len(st["ref"])))
    assert sorted(st["stack"] + list(used)) == list(range(len(st["ref"])))


@pytest.mark.parametrize("seed", range(6))
def test_fork(seed):
    rng = np.random.default_rng(seed)
    B = int(rng.integers(1, 9))
    st = forked_state(rng, B, int(rng.integers(1, 7)), 60)
    consistent(st)
    before = copy.deepcopy(st)
    OS.fork(st, np.arange(B))
    assert np.array_equal(st["table"], before["table"]) and st["stack"] == before["stack"]
    perm = rng.permutation(B)
    OS.fork(st, perm)
    OS.fork(st, np.argsort(perm))
    assert np.array_equal(st["table"], before["table"]) and st["stack"] == before["stack"]
    OS.fork(st, rng.integers(-1, B, B))
    consistent(st)
    OS.fork(st, np.full(B, -1))
    consistent(st)
    assert len(st["stack"]) == 60 and (st["table"] == -1).all()


def test_fork_pushes_by_first_entry():
    st = {"table": np.array([[4, 1, -1], [4, 2, 3]], dtype=np.int32), "stack": [0, 5]}
    st["ref"] = OS.recount(st["table"], 6)
    OS.fork(st, np.array([-1, -1]))
    assert st["stack"] == [0, 5, 4, 1, 2, 3]


def test_fork_keeps_what_the_caller_holds():
    st = {"table": np.array([[1, 2]], dtype=np.int32), "stack": [0]}
    st["ref"] = OS.recount(st["table"], 3) + np.array([0, 1, 0])
    OS.fork(st, np.array([-1]))
    assert st["stack"] == [0, 2] and st["ref"].tolist() == [0, 1, 0]


def test_step_without_sharing_is_the_paged_rule():
    rng = np.random.default_rng(5)
    B, bs, steps = 5, 4, 40
    seg = np.stack([rng.integers(0, 9, B), rng.integers(5, 40, B), rng.integers(0, 4, B), rng.integers(1, 9, B)], 1)
    pol = np.stack([rng.integers(2, 9, B), rng.integers(0, 5, B), rng.integers(0, 3, B), rng.integers(1, 9, B),
                    rng.integers(0, 3, B)], 1).astype(np.int32)
    n_blocks = int((-(-(seg.sum(1) + steps) // bs)).sum())
    width = int((-(-(seg.sum(1) + steps) // bs)).max())
    table, free = np.full((B, width), -1, dtype=np.int32), list(range(n_blocks))
    for b in range(B):
        for c in range(-(-(int(seg[b].sum()) - 1) // bs)):
            table[b, c] = free.pop()
    st = {"table": table.copy(), "ref": OS.recount(table, n_blocks), "stack": list(free)}
    for _ in range(steps):
        s32 = seg.astype(np.int32)
        for b in range(B):
            for blk in OP.freeable_blocks(s32[b], pol[b], bs):
                if table[b, blk] >= 0:
                    free.append(int(table[b, blk]))
                    table[b, blk] = -1
        for b in range(B):
            blk = (int(seg[b].sum()) - 1) // bs
            if table[b, blk] < 0:
                table[b, blk] = free.pop()
        assert (OS.step(st, s32, pol, bs) == -1).all()
        assert np.array_equal(st["table"], table) and st["stack"] == free
        consistent(st)
        seg[:, 3] += 1


def test_step_copies_for_all_but_the_one_furthest_ahead():
    st = {"table": np.array([[0], [0], [0], [0]], dtype=np.int32), "stack": [1, 2, 3, 4]}
    st["ref"] = OS.recount(st["table"], 5)
    seg = np.array([[0, 0, 0, 3], [0, 0, 0, 5], [0, 0, 0, 5], [0, 0, 0, 2]], dtype=np.int32)
    pol = np.tile(np.array([-1, 0, 0, -1, 0], dtype=np.int32), (4, 1))
    copied = OS.step(st, seg, pol, 8)
    assert copied.tolist() == [0, 0, -1, 0] and st["table"][:, 0].tolist() == [4, 3, 0, 2]
    assert st["ref"].tolist() == [1, 0, 1, 1, 1] and st["stack"] == [1]
    st["ref"][0] += 1  # a reference of the caller's own: nobody may write there
    assert OS.step(st, seg, pol, 8).tolist() == [-1, -1, 0, -1] and st["table"][2, 0] == 1


@pytest.mark.parametrize("seed", range(4))
def test_compact(seed):
    rng = np.random.default_rng(seed)
    st = forked_state(rng, 6, 5, 50)
    before = copy.deepcopy(st)
    new = OS.compact(st)
    consistent(st)
    n = int((before["ref"] > 0).sum())
    assert sorted(new[new >= 0].tolist()) == list(range(n))
    assert np.array_equal(new >= 0, before["ref"] > 0)
    keep = (before["ref"] > 0) & (np.arange(50) < n)
    assert np.array_equal(new[keep], np.flatnonzero(keep))
    assert st["stack"] == list(range(49, n - 1, -1))
    assert np.array_equal(OS.compact(st)[:n], np.arange(n))  # nothing is left to move


def test_attend_and_common():
    rng = np.random.default_rng(2)
    from paper_2606_01483_amd import workloads as W
    q, k, v = (W.f32_to_bf16_bits(rng.standard_normal(s)) for s in ((1, 1, 6, 128), (1, 1, 2, 9, 128), (1, 1, 2, 9, 128)))
    idx = np.array([[0, 3, 4, 8]], dtype=np.int32)
    want, want_lse = oracle.attend(q, k, v, idx, np.array([4]), scale=0.3)
    f = W.bf16_bits_to_f32
    rows = [f(x[0, 0])[:, idx[0]].transpose(1, 0, 2) for x in (k, v)]
    out, lse = OS.attend(f(q[0, 0]), *rows, 0.3)
    assert np.abs(out - want[0, 0]).max() < 1e-13 and np.abs(lse - want_lse[0, 0]).max() < 1e-13
    assert OS.common([[1, 2, 3], [1, 2, 4], [1, 2]]) == 2 and OS.common([[5, 6]]) == 2 and OS.common([[1], [2]]) == 0
