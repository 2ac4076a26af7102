"""Shared pages on the GPU (murmur_paged_fork, murmur_paged_step_shared, murmur_paged_compact) against the literal rules
of oracle/shared.py: tables, counts, stacks and copied rows exactly."""
import copy

import numpy as np
import pytest
import torch

from oracle import paged as OP
from oracle import shared as OS
from paper_2606_01483_amd import murmur as M
from _shared import forked_state

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


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


class Device:
    """The same state on the device."""

    def __init__(self, st):
        self.B, self.max_blocks = st["table"].shape
        self.n = len(st["ref"])
        self.table, self.ref = i32(st["table"]), i32(st["ref"])
        self.stack, self.top = i32(st["stack"] + [0] * (self.n - len(st["stack"]))), i32([len(st["stack"])])
        self.bytes = M.murmur_paged_workspace(self.B, self.max_blocks, self.n)
        self.ws = torch.zeros(self.bytes // 4, dtype=torch.int32, device="cuda")
        self.copied, self.map = i32(np.full(self.B, -7)), i32(np.full(self.n, -7))

    def args(self):
        return self.table, self.max_blocks

    def rest(self):
        return self.ref, self.n, self.stack, self.top, self.n

    def fork(self, parent):
        M.murmur_paged_fork(parent, self.B, *self.args(), *self.rest(), self.ws, self.bytes)

    def step(self, seg, pol, bs, full, pool=None, Hkv=0, k=None, v=None):
        M.murmur_paged_step_shared(seg, pol, 1, self.B, *self.args(), bs, *self.rest(), full, self.copied, pool, Hkv, k, v)

    def compact(self, bs, pool=None, Hkv=0):
        M.murmur_paged_compact(self.B, *self.args(), bs, *self.rest(), self.map, pool, Hkv, self.ws, self.bytes)

    def check(self, st, what=""):
        torch.cuda.synchronize()
        top = int(self.top.item())
        assert np.array_equal(self.table.cpu().numpy(), st["table"]), what
        assert np.array_equal(self.ref.cpu().numpy(), st["ref"]), what
        assert self.stack[:top].cpu().numpy().tolist() == st["stack"], what


@pytest.mark.parametrize("B,max_blocks", [(1, 1), (2, 3), (5, 7), (97, 40), (33, 513), (600, 11), (1025, 3), (3, 2100)])
def test_fork(B, max_blocks):
    """Rounds of random parents, endings, permutations and the identity on one workspace."""
    announce(f"fork {B} x {max_blocks}")
    rng = np.random.default_rng(B * 7919 + max_blocks)
    st = forked_state(rng, B, max_blocks, B * max_blocks // 2 + 5)
    d = Device(st)
    rounds = [np.arange(B), rng.permutation(B), rng.integers(0, B, B), rng.integers(-1, B, B),
              np.where(rng.random(B) < 0.5, np.arange(B), rng.integers(0, B, B)), np.full(B, B - 1), np.full(B, -1)]
    for i, parent in enumerate(rounds):
        d.fork(i32(parent))
        OS.fork(st, parent)
        d.check(st, f"round {i}")
    assert M.murmur_device_error() == 0


def test_fork_keeps_blocks_that_the_caller_holds():
    announce("fork with references of the caller")
    rng = np.random.default_rng(3)
    st = forked_state(rng, 9, 12, 100)
    st["ref"][st["table"][0][st["table"][0] >= 0]] += 1
    d = Device(st)
    for parent in (np.full(9, 4), np.full(9, -1)):
        d.fork(i32(parent))
        OS.fork(st, parent)
        d.check(st)


def test_fork_reports_bad_parents_and_blocks():
    announce("fork with bad parents and blocks")
    rng = np.random.default_rng(4)
    st = forked_state(rng, 6, 5, 40)
    d = Device(st)
    d.fork(i32([0, 6, -2, 1 << 30, 0, -(1 << 31)]))
    OS.fork(st, [0, 1, 2, 3, 0, 5])
    d.check(st)
    assert M.murmur_device_error() == M.MURMUR_DEVERR_PARENT
    d.table[1, 2] = 40  # past the pool: copied along, counted nowhere
    d.fork(i32([1, 1, 2, 3, 4, 5]))
    torch.cuda.synchronize()
    assert M.murmur_device_error() == M.MURMUR_DEVERR_BLOCK
    assert int(d.table[0, 2]) == 40


def test_fork_with_a_stack_that_does_not_agree():
    """A full stack: what is freed is reported and dropped, nothing is written past it."""
    announce("fork with a full stack")
    st = forked_state(np.random.default_rng(5), 3, 4, 12)
    d = Device(st)
    guard = torch.full((64,), 99, dtype=torch.int32, device="cuda")
    d.stack = torch.cat([torch.zeros(12, dtype=torch.int32, device="cuda"), guard])
    d.top.fill_(12)
    d.fork(i32([-1, -1, -1]))
    torch.cuda.synchronize()
    assert M.murmur_device_error() == M.MURMUR_DEVERR_POOL
    assert int(d.top.item()) == 12 and torch.equal(d.stack[12:], guard)


def grown_pool(rng, NL, rows, Hkv, layout="flash"):
    """A pool of random bf16 bits, as tensors [NL, rows, Hkv, 128] over either storage order, and its murmur_kv."""
    shape = (NL, rows, Hkv, 128) if layout == "flash" else (NL, Hkv, rows, 128)
    k, v = (torch.from_numpy(rng.integers(0, 1 << 15, shape).astype(np.int16)).cuda() for _ in range(2))
    if layout == "flash":
        kv = M.make_kv(k, v, NL, rows, (rows * Hkv * 128, 0, 128, Hkv * 128))
        return k, v, kv
    kv = M.make_kv(k, v, NL, rows, (rows * Hkv * 128, 0, rows * 128, 128))
    return k.transpose(1, 2), v.transpose(1, 2), kv


@pytest.mark.parametrize("bs,B,layout", [(1, 3, "flash"), (4, 24, "flash"), (16, 9, "head"), (8, 300, "flash"),
                                         (64, 5, "head")])
def test_decode_with_forks(bs, B, layout):
    """Steps with a fork before each and a compaction now and then: bookkeeping as the rules say, and every row that
    a table names holds what its sequence wrote there, whoever wrote it."""
    announce(f"decode with forks: block {bs}, {B} sequences, {layout}")
    rng = np.random.default_rng(bs * 131 + B)
    NL, Hkv, steps = 2, 3, 14 if B > 100 else 40
    seg = np.tile(np.array([[5, 30, 2, 1]], dtype=np.int32), (B, 1))
    seg[:, 1] = rng.integers(10, 40, (B + 2) // 3)[np.arange(B) // 3]
    pol = np.tile(np.array([[12, 4, 3, 9, 2]], dtype=np.int32), (B, 1))
    pol[B // 2:] = [-1, 0, 0, -1, 0]
    lo = np.arange(B) // 3 * 3  # groups of three, of one length
    pol, width = pol[lo], np.minimum(lo + 3, B) - lo
    length = seg.sum(axis=1) - 1
    max_blocks = int(-(-(length.max() + steps) // bs))
    n_blocks = int(sum(-(-(length + steps + bs) // bs))) + 8
    free = [int(x) for x in rng.permutation(n_blocks)]
    table = np.full((B, max_blocks), -1, dtype=np.int32)
    for b in range(B):
        for c in range(-(-int(length[b]) // bs)):
            table[b, c] = free.pop() if b == lo[b] else table[lo[b], c]
    st = {"table": table, "ref": OS.recount(table, n_blocks), "stack": free}
    d = Device(st)
    k, v, kv = grown_pool(rng, NL, n_blocks * bs, Hkv, layout)
    host = [x.cpu().numpy().copy() for x in (k, v)]
    rows_of = lambda b, n: np.array([st["table"][b, p // bs] * bs + p % bs for p in range(n)])  # noqa: E731
    # what every sequence wrote, by position; rows of blocks that it has given up are not compared
    truth = [{p: (host[0][:, r], host[1][:, r]) for p, r in enumerate(rows_of(b, int(length[b])))} for b in range(B)]
    pol_d = i32(pol)
    for s in range(steps):
        parent = lo + (rng.random(B) * width).astype(np.int64)
        parent = np.where(rng.random(B) < 0.4, np.arange(B), parent)
        d.fork(i32(parent))
        OS.fork(st, parent)
        d.check(st, f"fork {s}")
        truth = [dict(truth[p]) for p in parent]
        new = [rng.integers(0, 1 << 15, (NL, B, Hkv, 128)).astype(np.int16) for _ in range(2)]
        d.step(i32(seg), pol_d, bs, s == 0, kv, Hkv, *(torch.from_numpy(x).cuda() for x in new))
        copied = OS.step(st, seg, pol, bs)
        d.check(st, f"step {s}")
        assert np.array_equal(d.copied.cpu().numpy(), copied), f"step {s}"
        for b in range(B):
            truth[b][int(seg[b].sum()) - 1] = (new[0][:, b], new[1][:, b])
        if s % 5 == 4:
            d.compact(bs, kv, Hkv)
            new_number = OS.compact(st)
            d.check(st, f"compact {s}")
            assert np.array_equal(d.map.cpu().numpy(), new_number), f"compact {s}"
        got = [x.cpu().numpy() for x in (k, v)]
        for b in range(B):
            for p, want in truth[b].items():
                x = st["table"][b, p // bs]
                if x >= 0:
                    assert np.array_equal(got[0][:, x * bs + p % bs], want[0]), (s, b, p)
                    assert np.array_equal(got[1][:, x * bs + p % bs], want[1]), (s, b, p)
        seg[:, 3] += 1
    assert M.murmur_device_error() == 0


def test_step_copies_for_all_but_the_one_furthest_ahead():
    """Sharers of one block at different positions; and a reference of the caller's, which nobody may overwrite."""
    announce("sharers at different positions")
    st = {"table": np.array([[0], [0], [0], [0]], dtype=np.int32), "stack": [1, 2, 3, 4]}
    st["ref"] = OS.recount(st["table"], 5)
    seg = np.array([[0, 0, 0, 3], [0, 0, 0, 5], [0, 0, 0, 5], [0, 0, 0, 2]], dtype=np.int32)
    pol = np.tile(np.array([-1, 0, 0, -1, 0], dtype=np.int32), (4, 1))
    d = Device(st)
    d.step(i32(seg), i32(pol), 8, True)
    assert OS.step(st, seg, pol, 8).tolist() == [0, 0, -1, 0]
    d.check(st)
    assert d.copied.cpu().tolist() == [0, 0, -1, 0]
    d.ref[0] += 1
    st["ref"][0] += 1
    d.step(i32(seg), i32(pol), 8, True)
    assert OS.step(st, seg, pol, 8).tolist() == [-1, -1, 0, -1]
    d.check(st)


def test_step_many_sequences_of_one_block():
    """600 sequences (three rounds of the workgroup) that all name the same blocks, in descending order of position."""
    announce("600 sharers")
    B, bs = 600, 1024
    st = {"table": np.zeros((B, 1), dtype=np.int32), "stack": list(range(B, 0, -1))}
    st["ref"] = OS.recount(st["table"], B + 1)
    seg = np.zeros((B, 4), dtype=np.int32)
    seg[:, 3] = 700 - np.arange(B)
    seg[300, 3] = 700  # a tie for the lead
    pol = np.tile(np.array([-1, 0, 0, -1, 0], dtype=np.int32), (B, 1))
    d = Device(st)
    d.step(i32(seg), i32(pol), bs, True)
    copied = OS.step(st, seg, pol, bs)
    d.check(st)
    assert np.array_equal(d.copied.cpu().numpy(), copied) and copied[300] == -1 and copied[0] == 0


@pytest.mark.parametrize("B", [1024, 1025, 2300])
def test_step_of_more_sequences_than_the_workgroup_has_threads(B):
    announce(f"steps of {B} sequences")
    rng = np.random.default_rng(B)
    bs, steps = 4, 6
    lo = np.arange(B) // 3 * 3
    seg = np.tile(np.array([[3, 9, 1, 8]], dtype=np.int32), (B, 1))
    seg[:, 3] += rng.integers(0, 12, (B + 2) // 3)[np.arange(B) // 3].astype(np.int32)
    pol = np.tile(np.array([[4, 2, 1, 5, 1]], dtype=np.int32), (B, 1))
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
    for s in range(steps):
        parent = np.minimum(lo + rng.integers(0, 3, B), B - 1)
        d.fork(i32(parent))
        OS.fork(st, parent)
        d.step(i32(seg), i32(pol), bs, s == 0)
        copied = OS.step(st, seg, pol, bs)
        d.check(st, f"step {s}")
        assert np.array_equal(d.copied.cpu().numpy(), copied), f"step {s}"
        seg[:, 3] += 1


def test_2500_sharers_of_one_block():
    announce("2500 sharers")
    B, bs = 2500, 4096
    st = {"table": np.zeros((B, 1), dtype=np.int32), "stack": list(range(B, 0, -1))}
    st["ref"] = OS.recount(st["table"], B + 1)
    seg = np.zeros((B, 4), dtype=np.int32)
    seg[:, 3] = 1 + np.random.default_rng(5).integers(0, 900, B)
    pol = np.tile(np.array([-1, 0, 0, -1, 0], dtype=np.int32), (B, 1))
    d = Device(st)
    d.step(i32(seg), i32(pol), bs, True)
    copied = OS.step(st, seg, pol, bs)
    d.check(st)
    assert np.array_equal(d.copied.cpu().numpy(), copied) and (copied == -1).sum() == 1


def test_step_on_unshared_rows_is_paged_step():
    announce("unshared rows against murmur_paged_step")
    rng = np.random.default_rng(9)
    B, bs, steps = 300, 4, 12
    seg = np.stack([rng.integers(0, 9, B), rng.integers(5, 40, B), rng.integers(0, 4, B), rng.integers(1, 9, B)], 1).astype(np.int32)
    pol = np.stack([rng.integers(2, 9, B), rng.integers(0, 5, B), rng.integers(0, 3, B), rng.integers(1, 9, B),
                    rng.integers(0, 3, B)], 1).astype(np.int32)
    n = int((-(-(seg.sum(1) + steps) // bs)).sum())
    table = np.full((B, int((-(-(seg.sum(1) + steps) // bs)).max())), -1, dtype=np.int32)
    free = list(range(n))
    for b in range(B):
        for c in range(-(-(int(seg[b].sum()) - 1) // bs)):
            table[b, c] = free.pop()
    st = {"table": table, "ref": OS.recount(table, n), "stack": free}
    d = Device(st)
    table2, stack2, top2 = d.table.clone(), d.stack.clone(), d.top.clone()
    for s in range(steps):
        d.step(i32(seg), i32(pol), bs, s == 0)
        M.murmur_paged_step(i32(seg), i32(pol), 1, B, table2, d.max_blocks, bs, stack2, top2, n, s == 0)
        torch.cuda.synchronize()
        assert torch.equal(d.table, table2) and torch.equal(d.top, top2)
        assert torch.equal(d.stack[:int(top2.item())], stack2[:int(top2.item())])
        seg[:, 3] += 1
    assert M.murmur_device_error() == 0


def test_step_errors():
    """An invalid sequence is left as is and nothing is written for it, a pool without blocks costs the sequence its
    entry, a token past the table is reported; the other sequences go on."""
    announce("step errors")
    st = {"table": np.array([[0, -1], [0, -1], [0, -1], [1, 2]], dtype=np.int32), "stack": [3]}
    st["ref"] = OS.recount(st["table"], 4)
    d = Device(st)
    k, v, kv = grown_pool(np.random.default_rng(1), 1, 16, 1)
    before = k.clone()
    seg = np.array([[0, 0, 0, 2], [0, 0, 0, -5], [0, 0, 0, 2], [0, 0, 0, 9]], dtype=np.int32)
    pol = np.tile(np.array([-1, 0, 0, -1, 0], dtype=np.int32), (4, 1))
    new = torch.full((1, 4, 1, 128), 77, dtype=torch.int16, device="cuda")
    d.step(i32(seg), i32(pol), 4, True, kv, 1, new, new)
    torch.cuda.synchronize()
    assert M.murmur_device_error() == M.MURMUR_DEVERR_POLICY | M.MURMUR_DEVERR_BLOCK | M.MURMUR_DEVERR_POOL
    # sequences 0 and 2 may not write into block 0, which sequence 1 names too: one block for two copies
    assert d.table.cpu().tolist() == [[3, -1], [0, -1], [-1, -1], [1, 2]]
    assert d.ref.cpu().tolist() == [1, 1, 1, 1] and int(d.top.item()) == 0
    assert d.copied.cpu().tolist() == [0, -2, -2, -1]
    want = before.clone()
    want[:, 12] = before[:, 0]
    want[:, 13] = 77
    assert torch.equal(k, want)


@pytest.mark.parametrize("n_blocks,used", [(1, 0), (1, 1), (7, 3), (1024, 500), (2500, 2499), (5000, 1200)])
def test_compact(n_blocks, used):
    announce(f"compact {used} of {n_blocks}")
    rng = np.random.default_rng(n_blocks + used)
    blocks = rng.permutation(n_blocks)
    B, width = 7, -(-max(used, 1) // 7) + 1
    table = np.full((B, width), -1, dtype=np.int32)
    table.ravel()[rng.permutation(B * width)[:used]] = blocks[:used]
    table[3] = np.where(rng.random(width) < 0.5, table[2], -1) if used > 50 else table[3]
    st = {"table": table, "ref": OS.recount(table, n_blocks)}
    st["stack"] = [int(x) for x in np.flatnonzero(st["ref"] == 0)]
    before = copy.deepcopy(st)
    d = Device(st)
    k, v, kv = grown_pool(rng, 2, n_blocks * 2, 1)
    old = k.clone(), v.clone()
    d.compact(2, kv, 1)
    new = OS.compact(st)
    d.check(st)
    assert np.array_equal(d.map.cpu().numpy(), new)
    live = np.flatnonzero(before["ref"] > 0)
    for x, y in zip((k, v), old):
        x, y = x.view(2, n_blocks, -1), y.view(2, n_blocks, -1)
        assert torch.equal(x[:, torch.from_numpy(new[live]).long().cuda()], y[:, torch.from_numpy(live).cuda()])
    d.compact(2)  # nothing to move, and no pool
    d.check(st)
    assert M.murmur_device_error() == 0


def test_compact_reports_names_of_free_blocks():
    announce("compact with names of free blocks")
    st = {"table": np.array([[5, 2, -1, 9]], dtype=np.int32), "ref": np.array([0, 0, 0, 0, 0, 1], dtype=np.int32),
          "stack": [0, 1, 2, 3, 4]}
    d = Device(st)
    d.compact(1)
    torch.cuda.synchronize()
    assert M.murmur_device_error() == M.MURMUR_DEVERR_BLOCK
    assert d.table.cpu().tolist() == [[0, -1, -1, 9]] and d.ref.cpu().tolist() == [1, 0, 0, 0, 0, 0]
    assert int(d.top.item()) == 5 and d.stack[:5].cpu().tolist() == [5, 4, 3, 2, 1]


def test_captured_and_on_another_stream():
    """A fork, a step and a compaction captured into one graph and replayed three times from the same state, with
    eager calls on the same workspace in between."""
    announce("captured pages")
    rng = np.random.default_rng(21)
    B, bs = 12, 4
    seg = np.tile(np.array([[3, 20, 0, 4]], dtype=np.int32), (B, 1))
    pol = np.tile(np.array([[8, 2, 1, 3, 1]], dtype=np.int32), (B, 1))
    free = list(range(150))
    table = np.full((B, 8), -1, dtype=np.int32)
    for b in range(B):
        for c in range(7):
            table[b, c] = free.pop() if b % 4 == 0 else table[b - b % 4, c]
    st = {"table": table, "ref": OS.recount(table, 150), "stack": free}
    d, k_v = Device(st), grown_pool(rng, 2, 600, 2)
    k, v, kv = k_v
    parent, seg_d, pol_d = i32(np.arange(B) // 4 * 4 + rng.integers(0, 4, B)), i32(seg), i32(pol)
    new = torch.full((2, B, 2, 128), 7, dtype=torch.int16, device="cuda")
    state = [d.table, d.ref, d.stack, d.top, k, v, d.copied, d.map]
    start = [x.clone() for x in state]

    def work():
        d.fork(parent)
        d.step(seg_d, pol_d, bs, True, kv, 2, new, new)
        d.compact(bs, kv, 2)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        work()
    torch.cuda.synchronize()
    want = [x.clone() for x in state]
    for x, y in zip(state, start):
        x.copy_(y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for _ in range(3):
        for x, y in zip(state, start):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(state, want):
            assert torch.equal(x, y)
        for x, y in zip(state, start):
            x.copy_(y)
        work()
        torch.cuda.synchronize()
        for x, y in zip(state, want):
            assert torch.equal(x, y)
    assert M.murmur_device_error() == 0
