"""Shared pages and attention over shared prefixes -- TEST INFRASTRUCTURE (oracle side).

Only ``tests/`` may import this module; it imports nothing from the GPU package.  Plain definitions, run literally on
a dict ``st`` of ``table`` [B, max_blocks], ``ref`` [n_blocks] and ``stack`` (a list, top last):

  * ``fork``    -- rows become copies of their parents' rows; counts are recounted from the tables, and a block whose
                   entries are all gone is pushed when its first entry is met (row by row, column by column);
  * ``step``    -- one decode step: freeable blocks (oracle/paged.py's scan of later retained sets) are given up
                   sequence by sequence; then the writers, least far ahead first, each take a block, or copy one that
                   someone else still names; a sequence whose layout is all zeros is not there;
  * ``compact`` -- the blocks in use, those behind the last one that is to stay moved one by one into the first free;
  * ``attend``  -- Equation 1 over a list of pool rows, in fp64;
  * ``common``  -- the leading entries that several lists share.

Pins (``tests/test_oracle_shared.py``): counts always equal a recount of the table and every block is either named or
on the stack once; a fork of the identity changes nothing and a fork by a permutation is undone by its inverse; tables
that share nothing step exactly as ``oracle/paged.py``'s rule does; attention equals the oracle's over one cache.
"""
from __future__ import annotations

import numpy as np

from oracle import paged as OP


def recount(table, n_blocks: int) -> np.ndarray:
    return np.bincount(table[table >= 0].ravel(), minlength=n_blocks).astype(np.int32)


def fork(st: dict, parent) -> None:
    old = st["table"].copy()
    extra = st["ref"] - recount(old, len(st["ref"]))  # references that the caller holds itself
    for b, p in enumerate(parent):
        st["table"][b] = old[p] if p >= 0 else -1
    st["ref"] = recount(st["table"], len(st["ref"])) + extra
    for x in old.ravel():
        if x >= 0 and st["ref"][x] == 0 and x not in st["stack"]:
            st["stack"].append(int(x))


def step(st: dict, seg, pol, bs: int, freeable=None) -> np.ndarray:
    """Returns copied [B].  freeable(b): the sequence's blocks to give up (default: the oracle's scan)."""
    table, ref, stack, B = st["table"], st["ref"], st["stack"], len(seg)
    given = []
    here = [b for b in range(B) if np.any(seg[b])]
    for b in here:
        for blk in (freeable(b) if freeable else OP.freeable_blocks(seg[b], pol[b], bs)):
            if blk < table.shape[1] and table[b, blk] >= 0:
                given.append(int(table[b, blk]))
                ref[table[b, blk]] -= 1
                table[b, blk] = -1
    for x in given:
        if ref[x] == 0 and x not in stack:
            stack.append(x)
    pos = seg.sum(axis=1) - 1
    copied = np.full(B, -2, dtype=np.int32)
    copied[here] = -1
    wants = np.zeros(B, dtype=bool)
    named = ref.copy()
    for b in sorted(here, key=lambda b: (pos[b], b)):
        x = table[b, pos[b] // bs]
        if x < 0:
            wants[b] = True
        elif named[x] > 1:
            wants[b], copied[b] = True, x
            named[x] -= 1
    for b in range(B):
        if wants[b]:
            got = stack.pop()
            if copied[b] >= 0:
                ref[copied[b]] -= 1
            ref[got] = 1
            table[b, pos[b] // bs] = got
    return copied


def compact(st: dict) -> np.ndarray:
    """Returns the new number of every block (-1: free)."""
    ref = st["ref"]
    n, new = len(ref), np.full(len(ref), -1, dtype=np.int32)
    live = [x for x in range(n) if ref[x] > 0]
    free = [x for x in range(len(live)) if ref[x] <= 0]
    for x in live:
        new[x] = x if x < len(live) else free.pop(0)
    st["table"] = np.where(st["table"] >= 0, new[st["table"]], -1).astype(np.int32)
    moved = np.zeros_like(ref)
    moved[new[live]] = ref[live]
    st["ref"] = moved
    st["stack"] = list(range(n - 1, len(live) - 1, -1))
    return new


def common(lists) -> int:
    n = 0
    while all(len(x) > n for x in lists) and len({int(x[n]) for x in lists}) == 1:
        n += 1
    return n


def attend(q, k, v, scale: float):
    """One sequence, one layer: q [Hq, D], k and v [rows, Hkv, D] of its list, fp64.  Returns (out, lse)."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    g = q.shape[0] // k.shape[1]
    out, lse = np.zeros_like(q), np.zeros(q.shape[0])
    for h in range(q.shape[0]):
        s = scale * (k[:, h // g] @ q[h])
        m = s.max()
        w = np.exp(s - m)
        out[h] = (w / w.sum()) @ v[:, h // g]
        lse[h] = m + np.log(w.sum())
    return out, lse
