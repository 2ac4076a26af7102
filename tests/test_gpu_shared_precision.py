"""fp32 outputs of the attention over shared prefixes keep their weights to fp32's own precision: weights that two bf16
parts miss by 2^-18 of their size and more, in lists whose other errors are far smaller.

Each list has one position of logit 0 and value 0, one of logit -t and value 1, and any number of logit -2^15, whose
weight is 0 exactly: the output is w / (1 + w), w = exp(-t / 4).  The logits are exact (a query of one 1).  With U = 2^-24:
the exponent's argument is off by 3 U of its size (the scale in log2 units, its constant, the product; times ln 2 and
t / 4 <= 1/4: under 1 U of w), exp2 by 2 U, the sum of three products by 2 U, the sum 1 + w by 1 U and w's own 3 U, the
reciprocal and the product by 1 U each: 11 U.  A join of partial results multiplies by exp2 of a difference of maxima,
0 or so far down that nothing is left, and adds zeros: up to 4 U more where the two positions lie in different parts (the
maximum of a part is -t / 4 in log2 units, off by 1 U, its weight exp2 of that, 2 U, and a product).  16 U in all."""
import numpy as np
import pytest
import torch

from paper_2606_01483_amd import murmur as M
from test_gpu_shared_attn import CUT, Case

U, SCALE = 2.0 ** -24, 0.25
BOUND = 16 * U


def to_bf16(x):
    bits = np.asarray(x, dtype=np.float32).view(np.uint32)
    return ((bits + 0x7fff + (bits >> 16 & 1)) & 0xffff0000).astype(np.uint32).view(np.float32)


def parts(w, n):
    """The sum of n bf16 parts of fp32 weights, each the rounding of what the ones before leave."""
    left, got = np.asarray(w, dtype=np.float32), np.zeros(np.shape(w))
    for _ in range(n):
        p = to_bf16(left)
        got, left = got + p, left - p
    return got


def logits(n):
    """The n multiples of 1/256 up to 1 whose weights two parts miss by most."""
    t = np.arange(1, 257) / 256
    w = np.exp(-SCALE * t)
    off = np.abs(parts(w, 2) / w - 1)
    return np.sort(t[np.argsort(-off)[:n]])


def test_two_parts_are_too_few():
    """On the host: with these weights two parts miss the bound by far, three keep well inside it."""
    w = np.exp(-SCALE * logits(8))
    assert (np.abs(parts(w, 2) / w - 1) > 2.5 * BOUND).all()
    assert (np.abs(parts(w, 3) / w - 1) < BOUND / 8).all()


# (positions a group shares, the rests; which of the list's positions is the one of logit 0, which the one of logit -t)
LISTS = {
    "both in the rest": ([(0, [2, 2, 2])], 0, 1),
    "both shared": ([(2, [0, 0, 0])], 1, 0),
    "one each": ([(1, [1, 1])], 0, 1),
    "the larger in the rest": ([(1, [1, 1])], 1, 0),
    "far apart": ([(700, [33, 40, 65])], 3, 720),
    "both shared, long": ([(700, [33, 1])], 40, 690),
}


@pytest.mark.gpu
@pytest.mark.parametrize("extra_keep", [0, CUT])
@pytest.mark.parametrize("hq,hkv", [(8, 2), (16, 1)])
@pytest.mark.parametrize("name", sorted(LISTS))
def test_weights_of_fp32_outputs(name, hq, hkv, extra_keep):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    print(f"\n[case] precision, {name}, {hq}/{hkv}, +{extra_keep}", flush=True)
    groups, top, low = LISTS[name]
    c = Case(51, groups, hq=hq, hkv=hkv, scale=SCALE, extra_keep=extra_keep)
    for t in logits(8):
        c.q.zero_()
        c.q[..., 0] = 1
        for x in c.lists:
            c.k[:, x], c.v[:, x] = 0, 5
            c.k[:, x, :, 0] = -2.0 ** 15
        for x in c.lists:
            c.k[:, [x[top]], :, 0], c.v[:, x[top]] = 0, 0
            c.k[:, [x[low]], :, 0], c.v[:, x[low]] = -float(t), 1
        c.make_plan()
        c.attend()
        torch.cuda.synchronize()
        w = np.exp(-SCALE * t)
        assert np.abs(c.out.cpu().numpy() * (1 + w) / w - 1).max() <= BOUND, t
        assert np.abs(c.lse.cpu().numpy() - np.log1p(w)).max() <= BOUND, t
    assert M.murmur_device_error() == 0
