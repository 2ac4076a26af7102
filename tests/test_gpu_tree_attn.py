"""Attention of trees of drafted tokens (murmur_decode_attn_tree) against Equation 1 in fp64, node by node, within bounds
derived from the inputs (tests/_shared.py)."""
import numpy as np
import pytest
import torch

from oracle import draft as OD
from paper_2606_01483_amd import murmur as M
from _draft import D, OFF, TreeCase, bf16, i32, random_tree

pytestmark = pytest.mark.gpu


def announce(msg):
    print(f"\n[case] {msg}", flush=True)


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    M.lib()
    yield
    torch.cuda.synchronize()
    assert M.murmur_device_error() == 0


ALL = [OFF, 0, 0, OFF, 0]


@pytest.mark.parametrize("T,hq,hkv", [(1, 4, 4), (1, 28, 4), (2, 28, 4), (3, 28, 4), (5, 28, 4), (9, 28, 4), (18, 28, 4),
                                      (19, 28, 4), (37, 28, 4), (64, 28, 4), (64, 16, 1), (64, 2, 2), (33, 6, 2), (7, 15, 1)])
@pytest.mark.parametrize("f32", [True, False])
def test_sizes(T, hq, hkv, f32):
    """Row counts around the workgroups' row sets, every type."""
    announce(f"T {T} heads {hq}/{hkv} f32 {f32}")
    rng = np.random.default_rng(T * 100 + hq)
    parent = np.stack([random_tree(rng, T), random_tree(rng, T, wide=1)])
    TreeCase(T, [[3, 150, 4, 20], [0, 40, 0, 1]], ALL, parent, hq=hq, hkv=hkv, f32=f32).run().check(40)


@pytest.mark.parametrize("length", [1, 2, 3, 31, 32, 33, 63, 64, 65, 127, 129, 255, 257, 1000, 4099])
@pytest.mark.parametrize("block", [0, 1, 16])
def test_lengths(length, block):
    """Cached positions from none on, odd ones, blocks that end inside a pass."""
    announce(f"length {length} block {block}")
    rng = np.random.default_rng(length)
    seg = [[0, 0, 0, length], [length // 2, length // 4, length // 8, length - length // 2 - length // 4 - length // 8 + 1]]
    TreeCase(length, seg, ALL, np.stack([random_tree(rng, 6) for _ in seg]), block=block).run().check(12)


POLICIES = [ALL, [40, 3, 0, OFF, 0], [40, 30, 5, 16, 0], [7, 0, 3, 3, 2], [1, 0, 0, 1, 0], [1, 0, 0, 1, 90], [39, 12, 60, 5, 4],
            [64, 8, 200, 9, 6], [5000, 0, 0, 5000, 0], [33, 1, 1, 2, 1], [32, 25, 16, 12, 11], [2, 2 ** 31 - 1, 7, 2 ** 31 - 1, 2 ** 31 - 1],
            [11, 0, 2 ** 31 - 1, 4, 0]]


@pytest.mark.parametrize("pol", POLICIES)
@pytest.mark.parametrize("block", [0, 8])
def test_windows(pol, block):
    """Windows that move between the nodes of a tree, that are shorter than a path, that sinks touch or cover; the nodes of
    a chain and of a bush; sequences before, in and behind the delay."""
    announce(f"policy {pol} block {block}")
    rng = np.random.default_rng(5)
    seg = [[5, 100, 3, j] for j in (1, 2, 11, 28, 70)] + [[0, 33, 0, 30], [9, 0, 1, 12]]
    parent = np.stack([random_tree(rng, 23, wide=1 + i % 4, gone=i % 3) for i in range(len(seg))])
    TreeCase(7, seg, pol, parent, block=block).run().check(60)


def test_one_tree_for_all_and_policies_per_sequence_and_layer():
    announce("shared tree, policies per sequence and layer")
    rng = np.random.default_rng(1)
    pol = [[[30 + 10 * i, 5 * b, i, 8 + i, b] if (i + b) % 3 else ALL for b in range(4)] for i in range(3)]
    TreeCase(1, [[4, 90, 2, 9 + 7 * b] for b in range(4)], pol, random_tree(rng, 12), NL=3, layout="head").run().check(80)
    TreeCase(2, [[4, 90, 2, 9 + 7 * b] for b in range(4)], pol[1], random_tree(rng, 12), block=0, layout="head").run().check(40)


def test_sequences_and_nodes_that_are_not_there():
    announce("absent sequences and nodes")
    rng = np.random.default_rng(2)
    parent = np.stack([random_tree(rng, 20, gone=g) for g in (0, 20, 3, 19, 0)])
    parent[2, 5] = -2  # a leaf inside the tree
    parent[2, 6:17] = np.where(parent[2, 6:17] == 5, 4, parent[2, 6:17])
    TreeCase(3, [[5, 60, 0, 9], [5, 60, 0, 9], [5, 600, 0, 9], [0, 0, 0, 1], [0, 0, 0, 0]], [50, 4, 2, 6, 1], parent).run().check()


def test_many_splits_and_whole_lists():
    """The same batch with lists cut into splits and (in layers that fill the chip) whole; a schedule made for shorter or
    longer lists than there are."""
    announce("splits")
    rng = np.random.default_rng(4)
    parent = random_tree(rng, 16, wide=5)
    seg, pol = [[30, 2000, 9, 700], [30, 900, 0, 5]], [900, 64, 8, 300, 4]
    one = TreeCase(9, seg, pol, parent, hq=8, hkv=1)
    one.run().check(24)
    first = one.out.clone()
    for keep in (1, 100, one.keep * 20):
        n = M.murmur_decode_attn_tree_workspace(1, 2, 8, 1, 16, keep)
        one.ws, one.ws_bytes = torch.full((max(n, 256) // 4,), float("nan"), device="cuda"), n
        one.out.fill_(7.5)
        one.run(keep=keep).check(10)
    assert torch.allclose(first, one.out, atol=1e-5)
    TreeCase(10, seg, pol, parent, NL=90, hq=8, hkv=2).run().check(20)


@pytest.mark.parametrize("scale,lift", [(0.0, 1.0), (-0.3, 1.0), (1.0, 1.0), (D ** -0.5, 60.0), (2.0 ** -20, 2.0 ** 12)])
def test_scales(scale, lift):
    announce(f"scale {scale} lift {lift}")
    rng = np.random.default_rng(11)
    TreeCase(11, [[3, 70, 0, 40]], [50, 10, 0, 20, 2], random_tree(rng, 21)[None], scale=scale, lift=lift).run().check()


def test_a_chain_equals_single_steps():
    """What the nodes of a chain get is what murmur_decode_step gives token after token."""
    announce("chain against murmur_decode_step")
    T, hq, hkv = 12, 28, 4
    pol = [60, 9, 4, 7, 3]
    case = TreeCase(12, [[6, 200, 5, 14], [2, 90, 0, 3]], pol, np.arange(-1, T - 1, dtype=np.int32), block=0)
    case.run().check()
    rows = case.rows + T
    k, v = (torch.full((1, 2, rows, hkv, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for x, c, t in ((k, case.k, case.k_tree), (v, case.v, case.v_tree)):
        x[:, :, :case.rows] = c
        for b in range(2):
            at = int(case.seg_np[b].sum()) - 1
            x[0, b, at:at + T] = t[0, b]
    kv = M.make_kv(k, v, 1, rows, (k.stride(0), k.stride(1), k.stride(3), k.stride(2)))
    n = M.murmur_decode_attn_workspace(1, 2, hq, hkv, 400, 0)
    ws = torch.zeros(max(n, 256) // 4, dtype=torch.int32, device="cuda")
    for t in range(T):
        seg = i32(case.seg_np + [0, 0, 0, t])
        out, lse = torch.empty((1, 2, hq, D), device="cuda"), torch.empty((1, 2, hq), device="cuda")
        M.murmur_decode_step(seg, case.pol, 0, case.q[:, :, t].contiguous(), kv, None, None, None, 400, 2, hq, hkv, D, case.scale,
                             0, out, M.MURMUR_DTYPE_F32, lse, ws, n)
        # both within the bounds of the same exact values: 2 x 2^-16 of the values, and the sums' rounding
        assert torch.allclose(out, case.out[:, :, t], atol=2 * 2.0 ** -16 * 6), t
        assert torch.allclose(lse, case.lse[:, :, t], atol=2e-5), t


@pytest.mark.parametrize("what", ["k", "v"])
@pytest.mark.parametrize("value", [float("inf"), float("nan"), float("-inf")])
@pytest.mark.parametrize("T", [5, 40])
def test_what_a_node_does_not_see_does_not_touch_it(what, value, T):
    """An infinity or a NaN in a node's row, or in a cached row that windows have left, reaches those that attend to it
    and no other node."""
    announce(f"{what} {value} T {T}")
    rng = np.random.default_rng(13)
    case = TreeCase(13, [[4, 80, 2, 20]], [30, 3, 0, 9, 1], random_tree(rng, T, wide=2)[None])
    node = T // 2
    (case.k_tree if what == "k" else case.v_tree)[0, 0, node, :, 5] = value
    oldest = min(p for p in case.kept[0][0] if p >= 4)  # speech that only the root's window holds
    (case.k if what == "k" else case.v)[0, case.row(0, oldest)[0], :, 9] = value
    case.run()
    out = case.out.cpu().numpy()[0, 0]
    touched = []
    for t in range(T):
        cached, nodes = OD.sees(case.seg_np[0], case.pol_np, case.tree(0), t)
        touched.append(node in nodes or oldest in cached)
        if not touched[-1]:
            want, _, k, v, q = case.exact(0, 0, t)
            assert np.isfinite(out[t]).all() and np.abs(out[t] - want).max() < 1e-3, t
        elif what == "v":  # only the element that it is in
            want = np.array([5] * (node in nodes) + [9] * (oldest in cached))
            assert not np.isfinite(out[t][:, want]).any() and np.isfinite(np.delete(out[t], want, axis=1)).all(), t
        elif value != value:
            assert np.isnan(out[t]).all(), t
    assert any(touched) and not all(touched)


def test_rows_of_minus_infinity():
    """Logits of minus infinity weigh nothing; a node that has no others is NaN, as the formula says."""
    announce("minus infinity")
    rng = np.random.default_rng(14)
    case = TreeCase(14, [[0, 0, 0, 200]], ALL, random_tree(rng, 9)[None], hq=4, hkv=4)
    case.q[..., 0] = 1.0
    rows = torch.tensor([case.row(0, p)[0] for p in range(150)], device="cuda")
    case.k[0, rows, :, 0] = float("-inf")
    case.run()
    assert torch.isfinite(case.out).all() and torch.isfinite(case.lse).all()
    case.k[..., 0], case.k_tree[..., 0] = float("-inf"), float("-inf")
    case.run()
    assert torch.isnan(case.out).all() and (case.lse == float("-inf")).all()


@pytest.mark.parametrize("rows", [3_500_000, 6_000_000])
def test_far_rows(rows):
    """Pools of more than 2^31 and 2^32 bytes a plane."""
    announce(f"far rows {rows}")
    hkv, T = 4, 3
    rng = np.random.default_rng(15)
    case = TreeCase(15, [[2, 60, 0, 5]], [30, 2, 0, OFF, 0], random_tree(rng, T)[None], block=16)
    k = torch.empty((1, rows, hkv, D), dtype=torch.bfloat16, device="cuda")
    v = torch.empty((1, rows, hkv, D), dtype=torch.bfloat16, device="cuda")
    old = case.table_np.copy()
    case.table_np = np.where(old >= 0, rows // 16 - 1 - old, -1).astype(np.int32)
    for c in np.flatnonzero(old[0] >= 0):
        a, b = int(old[0, c]) * 16, int(case.table_np[0, c]) * 16
        k[0, b:b + 16], v[0, b:b + 16] = case.k[0, a:a + 16], case.v[0, a:a + 16]
    case.k, case.v, case.table, case.rows = k, v, i32(case.table_np), rows
    case.kv = M.make_kv(k, v, 1, rows, (rows * hkv * D, 0, D, hkv * D))
    case.run().check()


def nan_rows(case):
    return [bool(torch.isnan(case.out[:, b]).any()) for b in range(case.B)]


def test_device_errors():
    """Layouts, trees, positions and blocks that only the device sees are its errors, NaN for their sequence alone."""
    announce("device errors")
    rng = np.random.default_rng(16)
    T = 6
    seg = [[4, 60, 0, 8]] * 4
    good = random_tree(rng, T)
    for bad in ([0, 0, 1, 1, 2, 2], [-1, -1, 0, 0, 0, 0], [-1, 1, 0, 0, 0, 0], [-1, 0, 5, 0, 0, 0], [-1, 0, -2, 2, 0, 0],
                [-2, 0, 0, 0, 0, 0], [-1, 0, -3, 0, 0, 0], [-1, 0, 0, 2 ** 31 - 1, 0, 0]):
        case = TreeCase(16, seg, ALL, np.stack([good] * 4))
        case.parent[2] = torch.tensor(bad, dtype=torch.int32)
        case.run()
        assert M.murmur_device_error() == M.MURMUR_DEVERR_TREE, bad
        there = torch.tensor([x != -2 for x in bad])
        assert torch.isnan(case.out[0, 2].cpu()[there]).all() and (case.out[0, 2].cpu()[~there] == 7.5).all(), bad
        assert nan_rows(case) == [False, False, True, False]
    for field, pol in (([4, -1, 0, 8], None), ([4, 60, 0, 0], None), ([2 ** 31 - 1, 1, 0, 8], None), (None, [0, 0, 0, OFF, 0])):
        case = TreeCase(17, seg, [ALL] * 4, np.stack([good] * 4))
        if field:
            case.seg[1] = torch.tensor(field, dtype=torch.int32)
        else:
            case.pol[1] = torch.tensor(pol, dtype=torch.int32)
        case.run()
        assert M.murmur_device_error() == M.MURMUR_DEVERR_POLICY, (field, pol)
        assert nan_rows(case) == [False, True, False, False] and torch.isnan(case.lse[:, 1]).all()
    case = TreeCase(18, seg, ALL, np.stack([good] * 4))
    case.table[3, 2] = -1
    case.run()
    assert M.murmur_device_error() == M.MURMUR_DEVERR_BLOCK and nan_rows(case) == [False, False, False, True]
    case = TreeCase(18, seg, ALL, np.stack([good] * 4))
    case.seg[0, 3] = 2000  # past the table
    case.run()
    assert M.murmur_device_error() == M.MURMUR_DEVERR_BLOCK and nan_rows(case) == [True, False, False, False]
    case = TreeCase(19, seg, ALL, np.stack([good] * 4))
    case.table[1, 0] = 2 ** 30
    case.run()
    assert M.murmur_device_error() == M.MURMUR_DEVERR_POSITION and nan_rows(case) == [False, True, False, False]
    case = TreeCase(20, seg, ALL, np.stack([good] * 4), block=0)
    case.seg[2, 3] = 2000
    case.run()
    assert M.murmur_device_error() == M.MURMUR_DEVERR_POSITION and nan_rows(case) == [False, False, True, False]


def test_graph_and_streams():
    """Captured and replayed, with eager work of another batch between; two streams with a workspace each."""
    announce("graph")
    rng = np.random.default_rng(21)
    a = TreeCase(21, [[5, 300, 0, 90]] * 3, [200, 30, 0, 40, 0], random_tree(rng, 9))
    b = TreeCase(22, [[5, 500, 0, 9]] * 2, ALL, random_tree(rng, 30), block=0)
    a.run().check(10)
    b.run().check(10)
    want_a, want_b = a.out.clone(), b.out.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        a.call(stream=side)
    for _ in range(4):
        a.out.fill_(7.5)
        a.ws.fill_(float("nan"))
        b.out.fill_(7.5)
        torch.cuda.synchronize()
        g.replay()
        b.call()
        torch.cuda.synchronize()
        assert torch.equal(a.out, want_a) and torch.equal(b.out, want_b)
    # another sequence length and tree in the same buffers, as the captured call finds them
    a.seg[1, 3] = 40
    a.seg_np[1, 3] = 40
    a.parent.copy_(i32(random_tree(np.random.default_rng(5), 9, wide=1)))
    a.parent_np = a.parent.cpu().numpy()
    a.k.nan_to_num_(nan=0.25)
    a.v.nan_to_num_(nan=-0.5)
    a.table_np[:] = np.where(a.table_np < 0, 0, a.table_np)
    a.table.copy_(i32(a.table_np))
    g.replay()
    torch.cuda.synchronize()
    a.check()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for s in (s1, s2):
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        a.call(stream=s1)
        b.call(stream=s2)
    torch.cuda.synchronize()
    a.check(10)
    assert torch.equal(b.out, want_b)


@pytest.mark.parametrize("seed", range(12))
def test_random(seed):
    rng = np.random.default_rng(1000 + seed)
    B, T, NL = int(rng.integers(1, 6)), int(rng.integers(1, 65)), int(rng.integers(1, 4))
    hkv = int(rng.choice([1, 2, 4]))
    hq = hkv * int(rng.integers(1, 17))
    seg = [[int(rng.integers(0, 50)), int(rng.integers(0, 900)), int(rng.integers(0, 9)), int(rng.integers(1, 400))] for _ in range(B)]
    pol = [[int(rng.choice([OFF, rng.integers(1, 300)])), int(rng.integers(0, 100)), int(rng.integers(0, 40)),
            int(rng.choice([OFF, rng.integers(1, 100)])), int(rng.integers(0, 12))] for _ in range(B)]
    parent = np.stack([random_tree(rng, T, wide=int(rng.integers(1, 9)), gone=int(rng.integers(0, T))) for _ in range(B)])
    announce(f"seed {seed}: B {B} T {T} NL {NL} heads {hq}/{hkv}")
    TreeCase(seed, seg, pol, parent, NL=NL, hq=hq, hkv=hkv, block=int(rng.choice([0, 1, 8, 64])), f32=bool(rng.random() < 0.5),
             layout=str(rng.choice(["flash", "head"])), extra_keep=int(rng.choice([0, 0, 5000]))).run().check(30)
