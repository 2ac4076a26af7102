"""Helpers of the tests of shared pages and shared prefixes: forked states on the host and the error bounds of the
attention."""
import numpy as np

from oracle import shared as OS

U = 2.0 ** -24  # half a step of fp32, relative


def forked_state(rng, B, max_blocks, n_blocks, shared_columns=True):
    """A random consistent state: a forest of rows, each sharing a leading part with an earlier one or with none."""
    table = np.full((B, max_blocks), -1, dtype=np.int32)
    free = list(rng.permutation(n_blocks))
    for b in range(B):
        n = int(rng.integers(0, max_blocks + 1))
        if b and shared_columns and rng.random() < 0.8:
            o = int(rng.integers(0, b))
            keep = int(rng.integers(0, max_blocks + 1))
            table[b, :keep] = table[o, :keep]
            n = max(n, keep)
        for c in range(n):
            if table[b, c] < 0 and free and rng.random() < 0.9:  # holes: blocks that left the windows
                table[b, c] = free.pop()
    return {"table": table, "ref": OS.recount(table, n_blocks), "stack": [int(x) for x in free]}


def attn_bounds(q, k, v, scale, out, lse):
    """How far the fp32 computation may be from the 64-bit one for one sequence and layer (q [Hq, D], k and v
    [n, Hkv, D], out and lse the exact results): absolute bounds for out [Hq, 1] and lse [Hq].

    A logit is a sum of D products, exact in fp32 each (bf16 x bf16), added in any order: at most (D + 2) U times
    the sum of their sizes, the scale's rounding and the subtraction of the maximum included; in exp2's argument
    another rounding of its size (at most twice the largest logit, 2 U).  A weight carries the exponent's error,
    exp2's own (2 U) and the split into two bf16 parts (2^-17 and 2^-18: 2^-16 with the second part's rounding).
    Sums over n weights add n U, the join of partial results 16 U; numerator and denominator count both."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    g, n, D = q.shape[0] // k.shape[1], k.shape[0], q.shape[1]
    out_b, lse_b = np.zeros((q.shape[0], 1)), np.zeros(q.shape[0])
    for h in range(q.shape[0]):
        size = abs(scale) * (np.abs(k[:, h // g]) @ np.abs(q[h]))
        top = float(size.max())
        logit = (D + 2) * U * top + 4 * U * top
        weight = logit + 2 * U + n * U + 16 * U
        out_b[h] = (2 * weight + 2.0 ** -16) * np.abs(v[:, h // g]).max() + 4 * U * np.abs(out[h]).max()
        lse_b[h] = weight + 4 * U * max(1.0, abs(float(lse[h])), top)
    return out_b, lse_b
