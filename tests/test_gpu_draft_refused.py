"""Rounds of decode.TreeBatch in which murmur_paged_reserve refuses sequences: a pool that runs out and recovers, a table
that ends, prompts that find no room, rows of sequences that are not there.  A sequence that is refused sits the round out
(nothing accepted, the same root again) and goes on as if the round had not been."""
import numpy as np
import pytest
import torch

import test_gpu_draft_rounds as rounds
from oracle import draft as OD
from paper_2606_01483_amd import murmur as M
from paper_2606_01483_amd.decode import TreeBatch
from _draft import OFF, i32, random_tree
from test_gpu_draft_rounds import SEG, Run, announce, follows

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


def empty(batch):
    """Takes every free block out of the pool; returns them."""
    held = batch.stack[:int(batch.top)].clone()
    batch.top.zero_()
    return held


def refill(batch, held):
    free = torch.cat([held, batch.stack[:int(batch.top)]])
    batch.stack[:len(free)] = free
    batch.top.fill_(len(free))


def said_of(token):
    return np.where(token >= 0, follows(token), -1)


def check_took(run, parent, token, said, got):
    """Counts, paths, next roots and layouts; returns the nodes that each live sequence took."""
    batch, taken = run.batch, {}
    for b in range(len(run.seg)):
        live, refused = b in run.live, b in run.live and got[b] < 0
        path, last = OD.accept(parent[b], token[b], said[b]) if live and not refused else ([], token[b, 0] if refused else -1)
        assert int(batch.count[b]) == len(path) and int(batch.last[b]) == last, (b, got[b])
        assert batch.path[b].tolist() == path + [-1] * (run.T - len(path))
        if live:
            run.tokens[b] += [int(token[b, t]) for t in path[1:]] + [int(last)] * (len(path) > 0)
            taken[b] = len(path)
            assert int(batch.seg[b].sum()) == len(run.tokens[b]), (b, got[b])
        else:
            assert int(batch.seg[b].abs().sum()) == 0
    return taken


def one_round(run):
    """A round against the oracle; what was refused, and the nodes that each live sequence took."""
    parent, depth, token = run.draft()
    run.batch.attend(i32(parent), i32(depth), *run.decoder(np.maximum(token, 0)))
    torch.cuda.synchronize()
    errors, got = M.murmur_device_error(), run.batch.got.tolist()
    short = [b for b in run.live if got[b] < 0]
    assert errors == (M.MURMUR_DEVERR_POOL if short else 0)
    run.check_outputs(parent, token)  # the cache of a refused sequence is whole, and so are its nodes
    run.batch.accept(i32(parent), i32(token), i32(said_of(token)))
    torch.cuda.synchronize()
    M.murmur_device_error()  # no block for the next root: its next reserve says so
    return short, check_took(run, parent, token, said_of(token), got)


@pytest.mark.parametrize("pol", [ALL, [30, 5, 3, 9, 2]])
def test_a_pool_that_runs_out_and_recovers(pol):
    announce(f"a pool that runs out, policy {pol}")
    run = Run(5, SEG, pol, T=9)
    refused, out_of = 0, None
    for turn in range(11):
        if turn in (2, 7):
            out_of = empty(run.batch)
        short, taken = one_round(run)
        assert out_of is not None or not short
        refused += len(short)
        if turn in (5, 8):
            refill(run.batch, out_of)
            out_of = None
        if out_of is None:
            run.check_cache()
    assert refused > 2 and min(taken.values()) > 0


def test_in_a_graph():
    """Refusals are the device's to find: the rounds of a captured graph sit them out too."""
    announce("refused rounds in a graph")
    seg, T = [s for s in SEG if any(s)], 7
    eager, graph = Run(6, seg, ALL, T=T), Run(6, seg, ALL, T=T)
    B = len(seg)
    parent, depth, token, said = (i32(np.full((B, T), -2)) for _ in range(4))
    q, k, v = (x.clone() for x in graph.decoder(np.zeros(B * T)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        graph.batch.attend(parent, depth, q, k, v, side)
        graph.batch.accept(parent, token, said, side)
    torch.cuda.synchronize()
    refused = 0
    for turn in range(7):
        if turn == 2:
            out_of = empty(eager.batch)
            empty(graph.batch)
        p, d, t = eager.draft()
        s, x = said_of(t), eager.decoder(np.maximum(t, 0))
        eager.batch.attend(i32(p), i32(d), *x)
        eager.batch.accept(i32(p), i32(t), i32(s))
        for to, value in ((parent, i32(p)), (depth, i32(d)), (token, i32(t)), (said, i32(s)), (q, x[0]), (k, x[1]), (v, x[2])):
            to.copy_(value)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        got = eager.batch.got.tolist()
        refused += sum(x < 0 for x in got)
        check_took(eager, p, t, s, got)
        check_took(graph, p, t, s, got)
        for name in ("out", "lse", "got", "seg", "bt", "ref", "top", "path", "count", "last", "k", "v"):
            assert torch.equal(getattr(eager.batch, name), getattr(graph.batch, name)), (turn, name)
        if turn == 4:
            for x in (eager, graph):
                refill(x.batch, out_of)
    assert M.murmur_device_error() == M.MURMUR_DEVERR_POOL and refused > 0
    eager.check_cache()


def bush(T, deep):
    """A chain of `deep` nodes behind the root, the rest children of the root."""
    parent = np.zeros(T, dtype=np.int32)
    parent[0] = -1
    parent[1:deep + 1] = np.arange(deep)
    depth = np.ones(T, dtype=np.int32)
    depth[:deep + 1] = np.arange(deep + 1)
    return parent, depth


@pytest.mark.parametrize("deep", [0, 1, 4])
def test_a_round_asks_for_its_deepest_path(deep):
    """Blocks are taken for the deepest path's positions, not for every node; the last positions of a table are used."""
    announce(f"deepest path {deep}")
    seg, T, block = [[0, 60, 2, 1], [3, 0, 0, 1]], 16, 4
    run = Run(7, seg, ALL, T=T, block=block)
    if deep == 0:
        parent, depth = np.full((2, T), -2, dtype=np.int32), np.full((2, T), -1, dtype=np.int32)
        parent[:, 0], depth[:, 0] = -1, 0
    else:
        parent, depth = (np.stack([x, x]) for x in bush(T, deep))
    for turn in range(3):
        token = np.full((2, T), 1)
        token[:, 0] = [x[-1] for x in run.tokens]
        for t in range(1, deep + 1):
            token[:, t] = follows(token[:, t - 1])
        before = [len(x) for x in run.tokens]
        run.batch.attend(i32(parent), i32(depth), *run.decoder(np.maximum(token, 0)))
        torch.cuda.synchronize()
        assert run.batch.got.tolist() == [deep + 1] * 2 and M.murmur_device_error() == 0
        table = run.batch.bt.cpu().numpy()
        for b in range(2):
            assert (table[b] >= 0).sum() == -(-(before[b] + deep) // block)
        run.check_outputs(parent, token)
        run.batch.accept(i32(parent), i32(token), i32(said_of(token)))
        torch.cuda.synchronize()
        assert M.murmur_device_error() == 0
        assert min(check_took(run, parent, token, said_of(token), [T, T]).values()) == deep + 1
        run.check_cache()


def test_the_end_of_the_table(monkeypatch):
    """A path that ends in the table's last position is served; a longer one is refused, and a shorter one goes on."""
    announce("end of the table")
    T, limit = 8, 48
    monkeypatch.setattr(rounds, "TreeBatch", lambda *a, max_len, **kw: TreeBatch(*a, max_len=limit, **kw))
    run = Run(8, [[4, 36, 2, 1]], ALL, T=T)  # the root at 42; 42 .. 47 are left
    for deep, served in ((7, False), (3, True), (4, False), (1, True)):  # the root then at 46 and 48
        parent, depth = (x[None] for x in bush(T, deep))
        token = np.full((1, T), 1)
        token[0, 0] = run.tokens[0][-1]
        for t in range(1, deep + 1):
            token[:, t] = follows(token[:, t - 1])
        run.batch.attend(i32(parent), i32(depth), *run.decoder(token))
        torch.cuda.synchronize()
        assert M.murmur_device_error() == (0 if served else M.MURMUR_DEVERR_BLOCK)
        got = run.batch.got.tolist()
        assert got == [deep + 1 if served else -1]
        run.check_outputs(parent, token)
        run.batch.accept(i32(parent), i32(token), i32(said_of(token)))
        torch.cuda.synchronize()
        assert M.murmur_device_error() == (M.MURMUR_DEVERR_BLOCK if run.batch.seg.sum() > limit else 0)  # no row for the next root
        assert check_took(run, parent, token, said_of(token), got)[0] == (deep + 1 if served else 0)
    assert len(run.tokens[0]) == limit + 1


def test_prompts_without_room():
    """A prompt that is refused is not there in the rounds that follow; the others are as if it had never been."""
    announce("a refused prompt")
    run = Run(9, SEG, ALL, T=6, n_blocks=20)  # nine for the first; the third needs twelve
    torch.cuda.synchronize()
    # the fourth needs seven, so it is refused with the third
    assert M.murmur_device_error() == M.MURMUR_DEVERR_POOL and run.batch.got.tolist() == [67, 0, -1, -1]
    assert run.batch.seg.tolist() == [SEG[0], [0] * 4, [0] * 4, [0] * 4]
    run.live = [0]
    for turn in range(4):
        short, taken = one_round(run)
        assert not short and taken[0] > 0
        run.check_cache()


def test_a_row_of_zeros_stays_one():
    """Trees and tokens of a sequence that is not there are not looked at."""
    announce("trees of absent sequences")
    run = Run(10, SEG, ALL, T=6)
    rng = np.random.default_rng(10)
    for turn in range(3):
        parent, depth, token = run.draft()
        parent[1], depth[1], token[1] = random_tree(rng, 6, wide=1), np.arange(6), follows(5)
        for t in range(6):
            token[1, t] = follows(token[1, t - 1]) if t else 5
        run.batch.attend(i32(parent), i32(depth), *run.decoder(np.maximum(token, 0)))
        run.batch.accept(i32(parent), i32(token), i32(said_of(token)))
        torch.cuda.synchronize()
        assert M.murmur_device_error() == 0
        check_took(run, parent, token, said_of(token), run.batch.got.tolist())
        run.check_cache()
