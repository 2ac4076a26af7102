"""Every instance of the kernels of murmur_decode_attn_tree: the shapes of a workgroup, lists whole and cut, both joins, both
types of outputs; several rounds of passes; trees whose rows fill a row set, a part of it or one tile, so that its wavefronts
are ways by rows and groups by passes in every proportion.  And the third part of the weights of fp32 outputs, in each."""
import numpy as np
import pytest
import torch

from paper_2606_01483_amd import murmur as M
from _draft import OFF, TreeCase, random_tree
from _tree_forms import FORMS
from test_gpu_shared_precision import BOUND, SCALE, logits

pytestmark = pytest.mark.gpu
ALL = [OFF, 0, 0, OFF, 0]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    M.lib()
    yield
    torch.cuda.synchronize()
    assert M.murmur_device_error() == 0


def planned(case, keep):
    """The schedule of lists of up to `keep`."""
    assert case.keep <= keep
    case.keep, case.ws_bytes = keep, M.murmur_decode_attn_tree_workspace(case.NL, case.B, case.hq, case.hkv, case.T, keep)
    case.ws = torch.full((max(case.ws_bytes, 256) // 4,), float("nan"), dtype=torch.float32, device="cuda")
    return case


@pytest.mark.parametrize("f32", [True, False])
@pytest.mark.parametrize("name", sorted(FORMS))
def test_forms(name, f32):
    print(f"\n[case] {name}, f32 {f32}", flush=True)
    (NL, B, hq, hkv, T, keep), _ = FORMS[name]
    rng = np.random.default_rng(keep + B)
    seg, pol, parent = [], [], []
    for b in range(B):
        n = keep if b == 0 else int(rng.integers(max(keep // 4, T + 100), keep + 1))  # cached positions and nodes
        out = int(rng.integers(1, 90))
        pre = int(rng.integers(0, 9))
        seg.append([pre, n - T - pre - out + 1, 0, out])
        pol.append(ALL if b % 2 == 0 else [int(rng.integers(keep // 8, keep // 2)), int(rng.integers(0, 40)), int(rng.integers(0, 70)),
                                           int(rng.integers(1, 60)), int(rng.integers(0, 9))])
        parent.append(random_tree(rng, T, wide=int(rng.integers(1, 5)), gone=[0, T // 2, T - 2, 0, T - 1, T // 4][b % 6]))
    planned(TreeCase(B, seg, pol, np.stack(parent), NL=NL, hq=hq, hkv=hkv, f32=f32), keep).run().check(60)


@pytest.mark.parametrize("name", sorted(FORMS))
def test_weights_of_fp32_outputs(name):
    """As test_gpu_shared_precision.py: one cached position of logit 0 and value 0, one of logit -t and value 1, every other
    one and the nodes so far down that they weigh nothing; each output is w / (1 + w) within the bound derived there.  The
    two in one pass, in passes apart either way round, and at the two ends of the list (a maximum that lags counts the same:
    its weights are up to exp(t / 4), exact where w is not)."""
    print(f"\n[case] precision, {name}", flush=True)
    (NL, B, hq, hkv, T, keep), _ = FORMS[name]
    rng = np.random.default_rng(B)
    case = planned(TreeCase(B, [[0, keep - T - 4, 0, 5]] * B, ALL, random_tree(rng, T), NL=NL, hq=hq, hkv=hkv, scale=SCALE), keep)
    last = keep - T - 1
    for top, low in ((35, 40), (40, 37), (1, last), (last, 2), (last // 2, last // 2 + 33)):
        rows = [torch.tensor([case.row(b, p)[0] for b in range(B)], device="cuda") for p in (top, low)]
        for t in logits(4):
            case.q.zero_()
            case.q[..., 0] = 1
            for k, v in ((case.k, case.v), (case.k_tree, case.v_tree)):
                k.zero_()
                v.fill_(5)
                k[..., 0] = -2.0 ** 15
            case.k[:, rows[0], :, 0], case.v[:, rows[0]] = 0, 0
            case.k[:, rows[1], :, 0], case.v[:, rows[1]] = -float(t), 1
            case.run()
            w = np.exp(-SCALE * t)
            assert np.abs(case.out.cpu().numpy() * (1 + w) / w - 1).max() <= BOUND, (top, low, t)
            assert np.abs(case.lse.cpu().numpy() - np.log1p(w)).max() <= BOUND, (top, low, t)


@pytest.mark.parametrize("total,pol,good", [(2 ** 31 - 65, [20, 3, 1, 9, 0], True), (2 ** 31 - 64, [20, 3, 1, 9, 0], False),
                                            (2 ** 31 - 65, ALL, False), (2 ** 31 - 1, ALL, False)])
def test_the_longest_layouts(total, pol, good):
    """Positions to the deepest node's, and the ranks of a list to the end of its last pass, are 32-bit numbers: what is longer
    is an error, and nothing of it is read."""
    print(f"\n[case] layout of {total}, policy {pol}", flush=True)
    T, block = 40, 1 << 16
    case = TreeCase(1, [[2, 100, 0, 30]], [20, 3, 1, 9, 0], random_tree(np.random.default_rng(40), T), hq=4, hkv=1, block=block)
    case.k.nan_to_num_(nan=0.25)
    case.v.nan_to_num_(nan=-0.5)
    # every column of a table to 2^31 names one block
    case.cols, case.table = 1 << 15, case.table.expand(1, 1 << 15).contiguous()
    case.seg[0] = torch.tensor([0, 50, 0, total - 50], dtype=torch.int32)
    case.pol.copy_(torch.tensor(pol, dtype=torch.int32))
    case.run()
    assert M.murmur_device_error() == (0 if good else M.MURMUR_DEVERR_POLICY)
    assert bool(torch.isfinite(case.out).all()) == good and bool(torch.isnan(case.out).all()) != good
    if good:  # as many blocks fewer: the same rows, since the window is all that is kept of the outputs
        case.seg_np, case.table_np = case.seg.cpu().numpy() - [0, 0, 0, 32766 * block], case.table.cpu().numpy()
        case.check(12)
