"""Speculative decoding as a user runs it (decode.TreeBatch): prompts into the pool, trees of drafts, accepted paths,
blocks behind the windows back to the pool -- against the same tokens decoded one by one."""
import numpy as np
import pytest
import torch

from oracle import draft as OD
from paper_2606_01483_amd import murmur as M
from paper_2606_01483_amd.decode import TreeBatch
from _draft import D, OFF, i32, random_tree
from _shared import attn_bounds

pytestmark = pytest.mark.gpu
VOCAB = 97


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


def follows(token):
    """The decoder's choice after a token."""
    return (31 * token + 7) % VOCAB


class Decoder:
    """Projections by token: q, k, v [NL, VOCAB, heads, D], before any rotation."""

    def __init__(self, rng, NL, hq, hkv):
        self.x = {n: torch.from_numpy(rng.standard_normal((NL, VOCAB, h, D), dtype=np.float32)).to(torch.bfloat16).cuda()
                  for n, h in (("q", hq), ("k", hkv), ("v", hkv))}

    def __call__(self, tokens):
        tokens = torch.as_tensor(np.asarray(tokens, dtype=np.int64).reshape(-1)).cuda()
        return [self.x[n][:, tokens].contiguous() for n in "qkv"]


class Run:
    def __init__(self, seed, seg, pol, T, NL=2, hq=8, hkv=2, block=8, n_blocks=200, rot=128):
        self.rng = rng = np.random.default_rng(seed)
        self.seg, self.pol, self.T, self.NL, self.hq, self.hkv = np.array(seg), np.array(pol), T, NL, hq, hkv
        self.decoder = Decoder(rng, NL, hq, hkv)
        self.freq, _ = M.murmur_rope_freqs_host(rot, 1e4)
        self.freq_dev = torch.from_numpy(self.freq.view(np.int64)).cuda()
        self.rot = rot
        self.batch = TreeBatch(self.seg, self.pol, T, M.make_rope(rot, False, self.freq_dev), NL, hq, hkv, block, n_blocks,
                               max_len=700, max_keep=300, scale=D ** -0.5)
        # every token of every sequence: the prompt at random, then what the decoder says
        self.tokens = [list(rng.integers(0, VOCAB, size=max(int(s.sum()), 0))) for s in self.seg]
        self.live = [b for b in range(len(self.seg)) if self.seg[b].any()]
        prompt = [x for b in self.live for x in self.tokens[b][:-1]]
        self.q_out = torch.zeros((NL, len(prompt), hq, D), dtype=torch.bfloat16, device="cuda")
        self.batch.prefill(*self.decoder(prompt), self.q_out)

    def draft(self):
        """(parent, depth, tokens): trees that hold the true continuation for some way, among others."""
        rng, T, B = self.rng, self.T, len(self.seg)
        parent, depth, token = np.full((B, T), -2), np.full((B, T), -1), np.full((B, T), -1)
        for b in self.live:
            parent[b] = random_tree(rng, T, wide=int(rng.integers(1, 4)), gone=int(rng.integers(0, T)))
            for t in range(T):
                if parent[b, t] == -1:
                    depth[b, t], token[b, t] = 0, self.tokens[b][-1]
                elif parent[b, t] >= 0:
                    depth[b, t] = depth[b, parent[b, t]] + 1
                    token[b, t] = follows(token[b, parent[b, t]]) if rng.random() < 0.7 else rng.integers(0, VOCAB)
        return parent, depth, token

    def check_outputs(self, parent, token):
        """Every node against its path decoded alone, from the cache as it stands."""
        batch = self.batch
        table, out, lse = batch.bt.cpu().numpy(), batch.out.double().cpu().numpy(), batch.lse.cpu().numpy()
        for b in self.live:
            seg = self.seg[b].copy()
            seg[3] += len(self.tokens[b]) - seg.sum()
            for t in range(self.T):
                if parent[b, t] < -1:
                    continue
                cached, nodes = OD.sees(seg, self.pol if self.pol.ndim == 1 else self.pol[b], parent[b], t)
                rows = torch.tensor([int(table[b, p // batch.bs]) * batch.bs + p % batch.bs for p in cached], dtype=torch.long, device="cuda")
                at = torch.tensor(nodes, dtype=torch.long, device="cuda")
                for layer in range(self.NL):
                    k = torch.cat([batch.k[layer, rows], batch.k_tree[layer, b, at]]).double().cpu().numpy()
                    v = torch.cat([batch.v[layer, rows], batch.v_tree[layer, b, at]]).double().cpu().numpy()
                    q = batch.q[layer, b, t].double().cpu().numpy()
                    want, want_lse = OD.attend(q, k, v, batch.scale)
                    o_b, l_b = attn_bounds(q, k, v, batch.scale, want, want_lse)
                    assert (np.abs(out[layer, b, t] - want) <= o_b).all() and (np.abs(lse[layer, b, t] - want_lse) <= l_b).all()
                    # the query is the token's, turned to the node's position
                    place = seg.sum() - 1 + len(OD.path(parent[b], t)) - 1
                    self.check_turned(q, self.decoder.x["q"][layer, token[b, t]], place)

    def check_turned(self, got, x, place):
        x = x.double().cpu().numpy()
        want = OD.rotate(x, OD.turns(place, self.freq), self.rot, False, 1.0)
        size = np.abs(want).max() + np.abs(x).max()
        assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 32 * 2.0 ** -24 * size).all()

    def check_cache(self):
        """Retained rows are the tokens' keys and values, turned to their places; freed blocks are the pool's again, and
        every block is named once or free."""
        batch = self.batch
        table, stack = batch.bt.cpu().numpy(), batch.stack.cpu().numpy()[:int(batch.top)]
        named = table[table >= 0]
        assert sorted([*named, *stack]) == list(range(batch.n_blocks))
        for b in self.live:
            seg = self.seg[b].copy()
            seg[3] += len(self.tokens[b]) - seg.sum()
            assert batch.seg[b].tolist() == seg.tolist()
            cached, _ = OD.sees(seg, self.pol if self.pol.ndim == 1 else self.pol[b], [-1], 0)
            for p in self.rng.choice(cached, min(6, len(cached)), replace=False):
                row = int(table[b, p // batch.bs]) * batch.bs + p % batch.bs
                assert row >= 0
                self.check_turned(batch.k[0, row].double().cpu().numpy(), self.decoder.x["k"][0, self.tokens[b][p]], int(p))
                assert torch.equal(batch.v[:, row], self.decoder.x["v"][:, self.tokens[b][p]])

    def took(self, parent, token, said):
        lengths = []
        for b in range(len(self.seg)):
            path, last = OD.accept(parent[b], token[b], said[b]) if b in self.live else ([], -1)
            assert self.batch.path[b].tolist() == path + [-1] * (self.T - len(path))
            assert int(self.batch.last[b]) == last
            if b in self.live:
                self.tokens[b] += [int(token[b, t]) for t in path[1:]] + [last]
                lengths.append(len(path))
        return lengths


SEG = [[5, 60, 2, 1], [0, 0, 0, 0], [1, 90, 0, 1], [17, 33, 4, 1]]


@pytest.mark.parametrize("pol", [[OFF, 0, 0, OFF, 0], [30, 5, 3, 9, 2], [[20, 3, 0, 6, 1], [1, 0, 0, 1, 0], [40, 9, 8, OFF, 0], [OFF, 0, 0, 12, 4]]])
def test_rounds(pol):
    announce(f"rounds, policy {pol}")
    run = Run(1, SEG, pol, T=9)
    accepted = []
    for turn in range(9):
        parent, depth, token = run.draft()
        said = np.where(token >= 0, follows(token), -1)
        run.batch.attend(i32(parent), i32(depth), *run.decoder(np.maximum(token, 0)))
        torch.cuda.synchronize()
        assert M.murmur_device_error() == 0
        run.check_outputs(parent, token)
        run.batch.accept(i32(parent), i32(token), i32(said))
        torch.cuda.synchronize()
        assert M.murmur_device_error() == 0
        accepted += run.took(parent, token, said)
        run.check_cache()
    assert max(accepted) > 2 and min(accepted) == 1


def test_rounds_in_one_graph():
    """A captured round replayed on other trees and tokens, with eager work of another batch between, against the same
    rounds in eager calls."""
    announce("rounds in a graph")
    seg = [s for s in SEG if any(s)]
    pol = [25, 4, 2, 7, 1]
    eager, graph, other = Run(2, seg, pol, T=7), Run(2, seg, pol, T=7), Run(3, seg, pol, T=5)
    B, T = len(seg), 7
    parent, depth, token, said = (i32(np.full((B, T), -2)) for _ in range(4))
    q, k, v = (x.clone() for x in graph.decoder(np.zeros(B * T)))
    keep = graph.batch.seg.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        graph.batch.attend(parent, depth, q, k, v, side)
        graph.batch.accept(parent, token, said, side)
    torch.cuda.synchronize()
    assert torch.equal(graph.batch.seg, keep)
    for turn in range(7):
        p, d, t = eager.draft()
        s = np.where(t >= 0, follows(t), -1)
        x = eager.decoder(np.maximum(t, 0))
        eager.batch.attend(i32(p), i32(d), *x)
        eager.batch.accept(i32(p), i32(t), i32(s))
        for to, value in ((parent, i32(p)), (depth, i32(d)), (token, i32(t)), (said, i32(s)), (q, x[0]), (k, x[1]), (v, x[2])):
            to.copy_(value)
        po, do, to_ = other.draft()
        other.batch.attend(i32(po), i32(do), *other.decoder(np.maximum(to_, 0)))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        eager.took(p, t, s)
        graph.took(p, t, s)
        graph.check_cache()
        for name in ("out", "lse", "seg", "bt", "ref", "top", "path", "count", "last", "k", "v"):
            assert torch.equal(getattr(eager.batch, name), getattr(graph.batch, name)), (turn, name)
    assert M.murmur_device_error() == 0
