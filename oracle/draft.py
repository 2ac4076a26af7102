"""Requests into a paged pool, rotary positions and trees of drafted tokens -- TEST INFRASTRUCTURE (oracle side).

Only ``tests/`` may import this module; it imports nothing from the GPU package.  Plain definitions, run literally:

  * ``reserve``  -- sequence by sequence, block by block, off the end of a list;
  * ``turns``    -- a position times a table entry, a fraction of 2^64, in Python's integers;
  * ``rotate``   -- complex multiplication of a head's pairs, fp64;
  * ``sees``     -- what a node attends to: the retained set (oracle.retained) of its own step, whose outputs from the
                    root on are its path's nodes;
  * ``attend``   -- Equation 1 over that, in fp64;
  * ``accept``   -- the walk from the root.

Pins (``tests/test_oracle_draft.py``): a chain sees what single steps retain; rotations by p and -p undo each other, and
products of rotated vectors depend on the distance alone; a pool is neither leaked nor named twice by ``reserve``.
"""
from __future__ import annotations

import math

import numpy as np

import oracle


def reserve(st: dict, length, new, bs: int, per_seq: int, n_tokens: int, max_blocks: int) -> dict:
    """st: table [B, max_blocks], stack (a list, top last), ref (array or None), n_blocks; changed.  Returns the maps
    and the sequences refused, with the reason."""
    B = len(length)
    slot, pos, seq = (np.full(n_tokens, -1, dtype=np.int32) for _ in range(3))
    start, got, why = np.zeros(B + 1, dtype=np.int32), np.zeros(B, dtype=np.int32), {}
    at, short = 0, False
    for b in range(B):
        n = int(new[b]) if length[b] >= 0 else 0
        n = max(n, 0)
        if per_seq:
            at = b * per_seq
        start[b] = min(at, 2 ** 31 - 1)
        cols = range(int(length[b]) // bs, (int(length[b]) + n - 1) // bs + 1) if n else []
        need = [c for c in cols if st["table"][b, c] < 0] if cols and cols[-1] < max_blocks else []
        if length[b] < 0 or new[b] < 0:
            why[b] = "count"
        elif cols and cols[-1] >= max_blocks:
            why[b] = "block"
        elif per_seq and n > per_seq:
            why[b] = "overflow"
        elif any(st["table"][b, c] >= st["n_blocks"] for c in cols):
            why[b] = "block"
        elif st["ref"] is not None and any(st["table"][b, c] >= 0 and st["ref"][st["table"][b, c]] > 1 for c in cols):
            why[b] = "block"
        elif at + n > n_tokens:
            why[b] = "overflow"
        elif need and (short or len(need) > len(st["stack"])):
            why[b] = "pool"
            short = True
        else:
            for c in need:
                x = st["stack"].pop()
                st["table"][b, c] = x
                if st["ref"] is not None:
                    st["ref"][x] = 1
        got[b] = -1 if b in why else n
        for i in range(min(n if not per_seq else min(n, per_seq), max(n_tokens - at, 0))):
            p = int(length[b]) + i
            pos[at + i], seq[at + i] = min(p, 2 ** 31 - 1), b
            if b not in why:
                slot[at + i] = st["table"][b, p // bs] * bs + p % bs
        at += n
    start[B] = B * per_seq if per_seq else min(at, 2 ** 31 - 1)
    return dict(slot=slot, pos=pos, seq=seq, start=start, got=got, why=why)


def turns(p: int, freq) -> np.ndarray:
    """The fraction of a turn of every pair at position p, correctly rounded."""
    return np.array([(int(p) * int(f) % 2 ** 64) / 2.0 ** 64 for f in freq])


def rotate(x, fractions, rot: int, interleaved: bool, gain: float) -> np.ndarray:
    """x [..., D] turned, fp64."""
    y = np.array(x, dtype=np.float64)
    i = np.arange(rot // 2)
    re, im = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    z = (y[..., re] + 1j * y[..., im]) * (gain * np.exp(2j * math.pi * np.asarray(fractions)))
    y[..., re], y[..., im] = z.real, z.imag
    return y


def path(parent, t: int) -> list:
    """Nodes from the root to t."""
    up = [int(t)]
    while parent[up[-1]] >= 0:
        up.append(int(parent[up[-1]]))
    return up[::-1]


def sees(seg, pol, parent, t: int):
    """(cached positions, nodes) that node t attends to."""
    way = path(parent, t)
    step = np.array(seg, dtype=np.int32)
    step[3] += len(way) - 1
    root = int(np.sum(seg)) - 1  # the root's position
    idx, n = oracle.retained(step[None], np.asarray(pol, dtype=np.int32))
    idx = idx[0, :n[0]]
    return idx[idx < root], [way[i] for i in idx[idx >= root] - root]


def attend(q, k, v, scale: float):
    """One node and layer: q [Hq, D], k and v [rows, Hkv, D], fp64.  Returns (out, lse)."""
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


def accept(parent, token, said):
    """(path, last): one sequence's accepted nodes and the token after them."""
    if parent[0] != -1 or token[0] < 0:
        return [], -1
    way = [0]
    while True:
        kids = [t for t in range(len(parent)) if parent[t] == way[-1] and token[t] >= 0 and token[t] == said[way[-1]]]
        if not kids:
            return way, int(said[way[-1]])
        way.append(kids[0])
