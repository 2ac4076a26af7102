"""Sequences that are not there: hypotheses that ended, rows of a padded batch.  A murmur_seg of zeros takes nothing,
writes nothing and has no list (count -1); the plan passes over it, also where it is the first of its group."""
import copy

import numpy as np
import pytest
import torch

import oracle
from oracle import shared as OS
from paper_2606_01483_amd import murmur as M
from paper_2606_01483_amd import workloads as W
from paper_2606_01483_amd.decode import BeamBatch
from _shared import attn_bounds
from test_gpu_shared_attn import CUT, Case, bf16
from test_gpu_shared_pages import Device, grown_pool

pytestmark = pytest.mark.gpu
D = 128


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


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def leave(c, gone):
    """Takes sequences out of a Case; what the others of each group share is a property of their lists."""
    for b in gone:
        c.count[b] = -1
        c.idx[b] = -1
    here = [[c.lists[b] for b in range(lo, hi) if b not in gone] for lo, hi in zip(c.starts[:-1], c.starts[1:])]
    return [OS.common(x) if x else 0 for x in here]


def untouched(c, gone):
    return bool((c.out[:, gone] == 55).all()) and bool((c.lse[:, gone] == 55).all())


@pytest.mark.parametrize("extra_keep", [0, CUT])
@pytest.mark.parametrize("hq,hkv", [(28, 4), (3, 3)])
@pytest.mark.parametrize("gone", [[1], [0], [0, 1, 4], [0, 1, 2, 3], [5, 6], [0, 3, 4, 5, 8], list(range(9))], ids=str)
@pytest.mark.parametrize("common", [40, 1500])  # lists that the planner compares itself, and that another launch does
def test_absent_sequences_cost_their_group_nothing(common, gone, hq, hkv, extra_keep):
    announce(f"absent {gone}, common {common}, {hq}/{hkv}, +{extra_keep}")
    c = Case(31, [(common, [10, 0, 5, 70]), (20, [3, 2]), (33, [1, 0, 40])], NL=2, hq=hq, hkv=hkv, extra_keep=extra_keep)
    shared = leave(c, gone)
    c.make_plan()
    c.attend()
    c.check([b for b in range(c.B) if b not in gone])
    assert untouched(c, gone)
    assert c.shared.cpu().tolist() == shared
    assert M.murmur_device_error() == 0


@pytest.mark.parametrize("extra_keep", [0, CUT])
def test_absent_sequences_beside_bad_counts(extra_keep):
    """The other counts outside [1, max_keep] are errors as before, the first list that is there among them."""
    announce("absent and bad counts")
    c = Case(32, [(50, [10, 0, 5, 9]), (40, [3, 2, 8])], extra_keep=extra_keep)
    leave(c, [0, 4])
    c.count[2] = c.keep + 1
    c.count[5] = 0
    c.make_plan()
    c.attend()
    torch.cuda.synchronize()
    assert M.murmur_device_error() == M.MURMUR_DEVERR_COUNT
    assert torch.isnan(c.out[:, [2, 5]]).all() and untouched(c, [0, 4])
    c.check([1, 3, 6])
    assert c.shared.cpu().tolist() == [50, 0]


@pytest.mark.parametrize("extra_keep", [0, CUT])
def test_given_shares_and_range_tables(extra_keep):
    """The caller's shares are read from the first sequence that is there; from range tables, a total of -1."""
    announce("absent, given shares and range tables")
    rng = np.random.default_rng(33)
    NL, B, hq, hkv, prompt, L = 2, 6, 8, 2, 75, 400
    seg = np.stack([np.full(B, prompt), rng.integers(60, 200, B), np.full(B, 3), rng.integers(1, 90, B)], 1).astype(np.int32)
    pol = np.tile(np.array([50, 9, 4, 20, 2], dtype=np.int32), (B, 1))
    idx, cnt = oracle.retained(seg, pol)
    keep = idx.shape[1] + extra_keep
    q, k, v = bf16(rng, NL, B, hq, D), bf16(rng, NL, B, hkv, L, D), bf16(rng, NL, B, hkv, L, D)
    gone, first = [0, 1, 4], {0: 2, 1: 3}  # groups of 3: the first ones that are there
    whole = []
    for x in (k, v):
        for g in range(2):
            x[:, 3 * g:3 * g + 3, :, :prompt] = x[:, 3 * g:3 * g + 1, :, :prompt]
        whole.append(x.float().cpu().numpy().transpose(0, 1, 3, 2, 4).copy())
        x[:, [b for b in range(B) if b != first[b // 3]], :, :prompt] = float("nan")
        x[:, gone] = float("nan")
    d_idx, d_cnt, ranges = i32(np.zeros((B, keep))), i32(np.zeros(B)), i32(np.zeros((B, 6, 2)))
    M.murmur_evict_compact(i32(seg), i32(pol), 1, B, d_idx, keep, d_cnt, ranges)
    d_cnt[gone], d_idx[gone], ranges[gone] = -1, -1, 0
    ranges[gone, 0, 1] = -1
    group, shared = i32([0, 3, 6]), i32([prompt, prompt - 5])
    ws_bytes, plan_bytes = M.murmur_decode_attn_shared_workspace(NL, B, hq, hkv, keep, 2)
    ws, plan = (torch.zeros(n // 4, dtype=torch.int32, device="cuda") for n in (ws_bytes, plan_bytes))
    kv = M.kv_from_tensors(k, v)
    k[:, 5, :, prompt - 5:prompt], v[:, 5, :, prompt - 5:prompt] = (
        torch.from_numpy(x[:, 5, prompt - 5:prompt].transpose(0, 2, 1, 3).copy()).to(k) for x in whole)
    for table in (ranges, None):
        out, lse = torch.full((NL, B, hq, D), 55.0, device="cuda"), torch.full((NL, B, hq), 55.0, device="cuda")
        M.murmur_shared_plan(d_idx, table, d_cnt, keep, B, group, 2, shared, False, NL, hq, hkv, plan, plan_bytes)
        M.murmur_decode_attn_shared(q, kv, d_idx, table, keep, B, 2, hq, hkv, D, 0.11, out, M.MURMUR_DTYPE_F32, lse,
                                    plan, plan_bytes, ws, ws_bytes)
        torch.cuda.synchronize()
        assert M.murmur_device_error() == 0
        assert (out[:, gone] == 55).all() and (lse[:, gone] == 55).all()
        for b in (2, 3, 5):
            at = idx[b, :cnt[b]]
            for layer in range(NL):
                args = q[layer, b].float().cpu().numpy(), whole[0][layer, b][at], whole[1][layer, b][at], 0.11
                want, want_lse = OS.attend(*args)
                far, far_lse = attn_bounds(*args, want, want_lse)
                assert (np.abs(out[layer, b].cpu().numpy() - want) <= far).all(), (b, layer)
                assert (np.abs(lse[layer, b].cpu().numpy() - want_lse) <= far_lse).all(), (b, layer)


def test_no_list_of_an_absent_sequence():
    """murmur_evict_compact_paged: count -1, no entry, no error; murmur_evict_compact reports such a layout as before."""
    announce("lists of absent sequences")
    seg = np.array([[3, 9, 1, 4], [0, 0, 0, 0], [3, 9, 1, 6], [0, 0, 0, 0]], dtype=np.int32)
    pol = np.tile(np.array([-1, 0, 0, -1, 0], dtype=np.int32), (4, 1))
    table = i32(np.arange(4 * 5).reshape(4, 5))
    table[1] = -1
    idx, cnt, rng = i32(np.full((4, 24), 7)), i32(np.full(4, 7)), i32(np.full((4, 6, 2), 7))
    M.murmur_evict_compact_paged(i32(seg), i32(pol), 1, 4, table, 5, 4, idx, 24, cnt, rng)
    torch.cuda.synchronize()
    assert M.murmur_device_error() == 0
    assert cnt.cpu().tolist() == [17, -1, 19, -1]
    assert (idx[[1, 3]] == -1).all() and (idx[0, :17] >= 0).all()
    assert rng[[1, 3]].sum(dim=(1, 2)).cpu().tolist() == [-1, -1] and rng[1, 0].cpu().tolist() == [0, -1]
    M.murmur_evict_compact(i32(seg), i32(pol), 1, 4, idx, 24, cnt, rng)
    torch.cuda.synchronize()
    assert M.murmur_device_error() == M.MURMUR_DEVERR_POLICY
    assert cnt.cpu().tolist() == [17, 0, 19, 0] and (rng[[1, 3]] == 0).all()


@pytest.mark.parametrize("B,bs", [(24, 4), (300, 8), (1030, 4)])
def test_step_of_absent_sequences(B, bs):
    """Hypotheses end and come back as copies of others over 12 steps: table, counts, stack and the rows written."""
    announce(f"steps with absent sequences: {B}, block {bs}")
    rng = np.random.default_rng(B)
    NL, Hkv, steps = 1, 2, 12
    lo = np.arange(B) // 3 * 3
    seg = np.tile(np.array([[3, 12, 1, 5]], dtype=np.int32), (B, 1))
    seg[:, 3] += rng.integers(0, 9, (B + 2) // 3)[np.arange(B) // 3].astype(np.int32)
    pol = np.tile(np.array([6, 2, 1, 5, 1], dtype=np.int32), (B, 1))
    length = seg.sum(axis=1) - 1
    max_blocks = int(-(-(length.max() + steps) // bs))
    n_blocks = B * max_blocks
    free = [int(x) for x in rng.permutation(n_blocks)]
    table = np.full((B, max_blocks), -1, dtype=np.int32)
    for b in range(B):
        for c in range(-(-int(length[b]) // bs)):
            table[b, c] = free.pop() if b == lo[b] else table[lo[b], c]
    st = {"table": table, "ref": OS.recount(table, n_blocks), "stack": free}
    d = Device(st)
    k, v, kv = grown_pool(rng, NL, n_blocks * bs, Hkv)
    host = [x.cpu().numpy().copy() for x in (k, v)]
    live = np.ones(B, dtype=bool)
    for s in range(steps):
        parent = np.minimum(lo + rng.integers(0, 3, B), B - 1)
        parent = np.where(rng.random(B) < 0.15, -1, parent)
        if s == 2:
            parent[:3] = -1  # a whole group
        d.fork(i32(parent))
        OS.fork(st, parent)
        live = (parent >= 0) & live[parent]
        now = np.where(live[:, None], seg, 0).astype(np.int32)
        new = [rng.integers(0, 1 << 15, (NL, B, Hkv, 128)).astype(np.int16) for _ in range(2)]
        d.step(i32(now), i32(pol), bs, s == 0, kv, Hkv, *(torch.from_numpy(x).cuda() for x in new))
        before = copy.deepcopy(st["table"])
        copied = OS.step(st, now, pol, bs)
        d.check(st, f"step {s}")
        assert np.array_equal(d.copied.cpu().numpy(), copied), f"step {s}"
        assert (copied[~live] == -2).all() and (before[~live] == -1).all() and (st["table"][~live] == -1).all()
        old = [x.copy() for x in host]
        for b in np.flatnonzero(live):
            p = int(seg[b].sum()) - 1
            x = int(st["table"][b, p // bs])
            for h, o, n in zip(host, old, new):
                if copied[b] >= 0:
                    h[:, x * bs:x * bs + p % bs] = o[:, copied[b] * bs:copied[b] * bs + p % bs]
                h[:, x * bs + p % bs] = n[:, b]
        for x, h in zip((k, v), host):
            assert np.array_equal(x.cpu().numpy(), h), f"step {s}"
        seg[:, 3] += 1
    assert M.murmur_device_error() == 0


def beams(rng, steps, width, bs):
    seg0 = np.array([[16, 60, 4, 10], [30, 50, 0, 25], [5, 20, 0, 3]], dtype=np.int32)
    pol = np.array([[32, 20, 4, 24, 2], [-1, 0, 0, -1, 0], [8, 3, 1, 9, 1]], dtype=np.int32)
    wl = W.build("beams_ended", 719, 2, seg0, pol, steps, planted=False, hq=8, hkv=2)
    last = int((-(-wl.seg(steps - 1).sum(axis=1) // bs)).sum())
    return wl, pol, BeamBatch(wl, width, bs, last * width)


@pytest.mark.parametrize("stream", [False, True])
def test_beams_that_end(stream):
    """A beam decode of 40 steps in which hypotheses end, the first of a group and all of one among them, and come back
    as copies of others: the survivors' outputs, what they share, the pool and the error word."""
    announce(f"beams that end, stream of its own: {stream}")
    rng = np.random.default_rng(34)
    steps, width, bs = 40, 4, 4
    wl, pol, bb = beams(rng, steps, width, bs)
    B = 3 * width
    side = torch.cuda.Stream() if stream else None
    L = int(wl.seg(steps - 1).sum(axis=1).max())
    caches = []
    for x in (wl.k, wl.v):
        y = np.zeros((2, B, 2, L, D), dtype=np.uint16)
        n = min(L, x.shape[3])
        y[:, :, :, :n] = np.repeat(x[:, :, :, :n], width, axis=1)
        caches.append(y)
    policy = np.repeat(pol, width, axis=0)
    live, partly = np.ones(B, dtype=bool), 0
    f = W.bf16_bits_to_f32
    for s in range(steps):
        parent = np.arange(B) // width * width + rng.integers(0, width, B)
        parent = np.where(rng.random(B) < 0.5, np.arange(B), parent)
        parent = np.where(rng.random(B) < 0.04, -1, parent)
        if s == 3:
            parent[0] = -1  # the first of its group
        if s in (4, 5):
            parent[:width] = np.arange(width)
        if s == 20:
            parent[2 * width:] = -1  # a chunk is done
        live = (parent >= 0) & live[parent]
        seg = np.repeat(wl.seg(s), width, axis=0)
        q, kn, vn = (W.f32_to_bf16_bits(rng.standard_normal(sh)) for sh in ((2, B, 8, D), (2, B, 2, D), (2, B, 2, D)))
        up = [torch.from_numpy(x).view(torch.bfloat16).cuda() for x in (q, kn, vn)]
        given = i32(parent)
        bb.out.fill_(55)
        torch.cuda.synchronize()
        bb.step(s, given, *up, stream=side.cuda_stream if stream and s % 2 else side)
        if s % 9 == 8:
            bb.compact(stream=side)
        torch.cuda.synchronize()
        assert M.murmur_device_error() == 0, f"step {s}"
        caches = [x[:, np.maximum(parent, 0)].copy() for x in caches]
        for x, new in zip(caches, (kn, vn)):
            for b in range(B):
                x[:, b, :, int(seg[b].sum()) - 1] = new[:, b]
        idx, cnt = oracle.retained(seg, policy)
        assert np.array_equal(bb.count.cpu().numpy(), np.where(live, cnt, -1)), f"step {s}"
        lists = bb.idx.cpu().numpy()
        shares = []
        for g in range(3):
            here = [lists[b, :cnt[b]] for b in range(g * width, g * width + width) if live[b]]
            shares.append(OS.common(here) if here else 0)
        assert bb.shared.cpu().tolist() == shares, f"step {s}"
        if s == 3:
            assert shares[0] > 50 and not live[0]
        want, want_lse = oracle.attend(q, *caches, idx, cnt, scale=wl.scale, n_threads=16)
        out, lse = bb.out.cpu().numpy(), bb.lse.cpu().numpy()
        assert (out[:, ~live] == 55).all()
        for layer in range(2):
            for b in np.flatnonzero(live):
                at = idx[b, :cnt[b]]
                far, far_lse = attn_bounds(f(q[layer, b]), f(caches[0][layer, b])[:, at].transpose(1, 0, 2),
                                           f(caches[1][layer, b])[:, at].transpose(1, 0, 2), wl.scale, want[layer, b],
                                           want_lse[layer, b])
                assert (np.abs(out[layer, b] - want[layer, b]) <= far).all(), (s, layer, b)
                assert (np.abs(lse[layer, b] - want_lse[layer, b]) <= far_lse).all(), (s, layer, b)
        table = bb.bt.cpu().numpy()
        assert (table[~live] == -1).all()
        used = set(table.ravel().tolist()) - {-1}
        free = bb.stack[:int(bb.top.item())].cpu().numpy().tolist()
        assert sorted(list(used) + free) == list(range(bb.n_blocks)), f"step {s}"
        partly += 0 < live.sum() < B
    assert partly == 33 and not live.any() and len(free) == bb.n_blocks  # the last ones end at step 33


def test_beams_that_end_and_bad_parents():
    """A parent outside [-1, B) leaves its row as it is, ended or not, and is reported."""
    announce("beams with bad parents")
    wl, _, bb = beams(np.random.default_rng(35), 4, 3, 8)
    ins = [[bf16(np.random.default_rng(s), 2, 9, h, D) for h in (8, 2, 2)] for s in range(4)]
    bb.step(0, i32([0, 1, -1, 3, 4, 5, 6, 7, 8]), *ins[0])
    bb.step(1, None, *ins[1])
    torch.cuda.synchronize()
    assert M.murmur_device_error() == 0
    bb.step(2, i32([0, 9, 9, -2, 4, 5, 1 << 30, 7, -(1 << 31)]), *ins[2])
    torch.cuda.synchronize()
    assert M.murmur_device_error() == M.MURMUR_DEVERR_PARENT
    assert (bb.count < 0).cpu().tolist() == [False, False, True] + [False] * 6
    bb.step(3, i32([0, 1, 0, 3, 4, 5, 6, 7, 8]), *ins[3])
    torch.cuda.synchronize()
    assert M.murmur_device_error() == 0 and (bb.count > 0).all()


def test_beams_that_end_captured():
    """Six steps with endings in one graph, replayed three times from the starting state, the eager run's bits."""
    announce("beams that end, captured")
    rng = np.random.default_rng(36)
    wl, _, bb = beams(rng, 6, 4, 8)
    parents = [np.arange(12) // 4 * 4 + rng.integers(0, 4, 12) for _ in range(6)]
    parents[1][[0, 5]] = -1
    parents[3][8:] = -1
    parents = [i32(p) for p in parents]
    ins = [[bf16(rng, 2, 12, h, D) for h in (8, 2, 2)] for _ in range(6)]
    start = bb.state()

    def run():
        for s in range(6):
            bb.step(s, parents[s], *ins[s])

    run()
    torch.cuda.synchronize()
    want = (bb.count.clone(), bb.out.clone(), bb.lse.clone(), bb.shared.clone()) + bb.state()
    assert (want[0][8:] == -1).all() and (want[0][:8] > 0).any()
    bb.restore(start)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        bb.restore(start)
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip((bb.count, bb.out, bb.lse, bb.shared) + bb.state(), want):
            assert torch.equal(got, w)
        bb.restore(start)
        run()
        torch.cuda.synchronize()
        for got, w in zip((bb.count, bb.out, bb.lse, bb.shared) + bb.state(), want):
            assert torch.equal(got, w)
    assert M.murmur_device_error() == 0
