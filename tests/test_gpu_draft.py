"""Requests into a paged pool, rotary positions and accepted paths on the GPU (murmur_paged_reserve, murmur_rope_append,
murmur_tree_accept) against oracle/draft.py."""
import numpy as np
import pytest
import torch

from oracle import draft as OD
from oracle import shared as OS
from paper_2606_01483_amd import murmur as M
from _draft import D, bf16, i32, random_tree

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


# ---- reserve --------------------------------------------------------------------------------------------------------

BITS = {"count": M.MURMUR_DEVERR_COUNT, "block": M.MURMUR_DEVERR_BLOCK, "overflow": M.MURMUR_DEVERR_OVERFLOW,
        "pool": M.MURMUR_DEVERR_POOL}


class Pool:
    def __init__(self, rng, B, bs, cols, held, spare, counted=True):
        self.B, self.bs, self.cols, self.n_blocks = B, bs, cols, int(np.sum(held)) + spare
        order = list(rng.permutation(self.n_blocks))
        table = np.full((B, cols), -1, dtype=np.int32)
        for b in range(B):
            for c in range(int(held[b])):
                table[b, c] = order.pop()
        self.st = dict(table=table, stack=[int(x) for x in order], ref=OS.recount(table, self.n_blocks) if counted else None,
                       n_blocks=self.n_blocks)
        self.upload()

    def upload(self):
        st = self.st
        self.table, self.top = i32(st["table"]), i32([len(st["stack"])])
        self.stack = i32(st["stack"] + [-9] * (self.n_blocks - len(st["stack"])))
        self.ref = i32(st["ref"]) if st["ref"] is not None else None

    def call(self, length, new, per=0, n_tokens=None, pos=True, seq=True, stream=None):
        B = self.B
        n = n_tokens if n_tokens is not None else (B * per if per else max(int(np.maximum(new, 0).sum()), 1))
        self.start, self.got = i32(np.full(B + 1, -7)), i32(np.full(B, -7))
        self.slot, self.pos, self.seq = (i32(np.full(n, -7)) for _ in range(3))
        nbytes = M.murmur_paged_reserve_workspace(B)
        ws = torch.full((nbytes // 4,), -123456, dtype=torch.int32, device="cuda")
        M.murmur_paged_reserve(i32(length), i32(new), B, self.table, self.cols, self.bs, self.ref, self.n_blocks, self.stack,
                               self.top, self.n_blocks, per, n, self.start, self.got, self.slot, self.pos if pos else None,
                               self.seq if seq else None, ws, nbytes, stream)
        torch.cuda.synchronize()
        return n

    def check(self, length, new, per=0, n_tokens=None, **kw):
        n = self.call(length, new, per, n_tokens, **kw)
        want = OD.reserve(self.st, length, new, self.bs, per, n, self.cols)
        for name in ("start", "got", "slot") + (("pos",) if kw.get("pos", True) else ()) + (("seq",) if kw.get("seq", True) else ()):
            assert np.array_equal(getattr(self, name).cpu().numpy(), want[name]), name
        assert np.array_equal(self.table.cpu().numpy(), self.st["table"])
        assert int(self.top) == len(self.st["stack"]) and self.stack.cpu().tolist()[:len(self.st["stack"])] == self.st["stack"]
        if self.st["ref"] is not None:
            assert np.array_equal(self.ref.cpu().numpy(), self.st["ref"])
        bits = 0
        for w in want["why"].values():
            bits |= BITS[w]
        assert M.murmur_device_error() == bits, want["why"]
        return want


@pytest.mark.parametrize("B", [1, 2, 15, 16, 17, 33, 300])
@pytest.mark.parametrize("bs", [1, 16, 64])
@pytest.mark.parametrize("padded", [False, True])
def test_reserve(B, bs, padded):
    """Several calls on one pool, as a decode makes them: lengths grow, drafts leave blocks behind, some get nothing."""
    announce(f"reserve B {B} bs {bs} padded {padded}")
    rng = np.random.default_rng(B * 100 + bs)
    cols = 40 if bs < 64 else 9
    pool = Pool(rng, B, bs, cols, rng.integers(0, 4, size=B), spare=B * cols, counted=bs != 16)
    length = np.zeros(B, dtype=np.int64)
    for turn in range(5):
        room = cols * bs - length
        new = np.where(rng.random(B) < 0.2, 0, np.minimum(rng.integers(0, 7 * max(bs, 3), size=B), room))
        per = int(new.max()) + turn if padded else 0
        pool.check(length, new, per=max(per, 1) if padded else 0, n_tokens=(B * max(per, 1) if padded else int(new.sum()) + 1) + turn,
                   pos=turn != 1, seq=turn != 2)
        length = length + rng.integers(0, new + 1)


def test_reserve_prompts():
    announce("reserve: long prompts")
    rng = np.random.default_rng(1)
    for bs, new in ((16, [2283, 1, 0, 9000, 17]), (1, [5000, 70000]), (1 << 16, [70000, 1, 131072])):
        cols = -(-max(new) // bs) + 1
        pool = Pool(rng, len(new), bs, cols, [0] * len(new), spare=sum(-(-n // bs) for n in new) + 3)
        pool.check([0] * len(new), new)
        pool.check(new, [3] * len(new))


def test_reserve_where_the_pool_is_too_small():
    announce("reserve: short pool")
    rng = np.random.default_rng(2)
    for spare in range(0, 14):
        pool = Pool(rng, 20, 4, 12, rng.integers(0, 3, size=20), spare=spare)
        length = (pool.st["table"] >= 0).sum(1) * 4
        new = rng.integers(0, 9, size=20)
        pool.check(length, new)
        pool.check(length, np.minimum(new, 2), per=8)


def test_reserve_refusals_on_the_device():
    announce("reserve: refusals")
    rng = np.random.default_rng(3)
    fresh = lambda: Pool(rng, 6, 16, 5, [2, 1, 0, 3, 1, 0], spare=20)  # noqa: E731
    length = [20, 16, 0, 40, 9, 0]
    fresh().check(length, [5, -1, 3, 4, 1, 2])
    fresh().check([20, -3, 0, 40, 9, 0], [5, 9, 3, 4, 1, 2])
    fresh().check(length, [5, 1, 81, 4, 1, 80])                       # past the table
    fresh().check(length, [5, 1, 2 ** 31 - 1, 4, 1, 2 ** 31 - 1], n_tokens=30)
    fresh().check([2 ** 31 - 1] * 6, [2 ** 31 - 1] * 6, n_tokens=30)
    fresh().check(length, [5, 9, 3, 4, 1, 2], per=4)                  # more than its places
    fresh().check(length, [5, 9, 3, 4, 1, 2], n_tokens=18)            # more than the map
    fresh().check(length, [5, 9, 3, 0, 0, 2], n_tokens=1)
    pool = fresh()
    pool.st["table"][3, 2] = pool.n_blocks                            # not a block of the pool
    pool.upload()
    pool.check(length, [5, 9, 3, 4, 1, 2])
    pool = fresh()
    pool.st["ref"][pool.st["table"][0, 1]] = 2                        # others name it too
    pool.upload()
    pool.check(length, [5, 9, 3, 4, 1, 2])
    pool.st["ref"][pool.st["table"][0, 0]] = 3                        # one that nothing goes into
    pool.upload()
    pool.check(np.array(length) + [5, 9, 3, 4, 1, 2], [0, 1, 1, 1, 1, 1])
    pool = fresh()
    pool.stack[int(pool.top) - 2] = 1 << 20                           # a stack that is not the pool's
    pool.call([20, 16, 0, 40, 9, 0], [0, 9, 3, 0, 0, 2])
    assert M.murmur_device_error() == M.MURMUR_DEVERR_POOL
    assert pool.got.tolist() == [0, 9, -1, 0, 0, 2] and int(pool.table[2, 0]) == -1
    assert (pool.slot[9:12] == -1).all() and (pool.slot[:9] >= 0).all() and (pool.slot[12:14] >= 0).all()


def test_reserve_in_a_graph():
    """A captured call reads lengths and pool as they are at the replay."""
    announce("reserve: graph")
    rng = np.random.default_rng(4)
    B, bs, cols, per = 9, 4, 30, 7
    pool = Pool(rng, B, bs, cols, [1] * B, spare=B * cols)
    length, new = i32(np.full(B, 3)), i32(np.zeros(B))
    nbytes = M.murmur_paged_reserve_workspace(B)
    ws = torch.zeros(nbytes // 4, dtype=torch.int32, device="cuda")
    start, got = i32(np.zeros(B + 1)), i32(np.zeros(B))
    slot, pos, seq = (i32(np.zeros(B * per)) for _ in range(3))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        M.murmur_paged_reserve(length, new, B, pool.table, cols, bs, pool.ref, pool.n_blocks, pool.stack, pool.top,
                               pool.n_blocks, per, B * per, start, got, slot, pos, seq, ws, nbytes, side)
    at = np.full(B, 3)
    for turn in range(6):
        n = rng.integers(0, per + 1, size=B)
        new.copy_(i32(n))
        length.copy_(i32(at))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        want = OD.reserve(pool.st, at, n, bs, per, B * per, cols)
        assert np.array_equal(slot.cpu().numpy(), want["slot"]) and np.array_equal(got.cpu().numpy(), want["got"])
        assert np.array_equal(pool.table.cpu().numpy(), pool.st["table"]) and int(pool.top) == len(pool.st["stack"])
        at = at + n


# ---- rope -----------------------------------------------------------------------------------------------------------

class Rope:
    def __init__(self, seed, n, hq=28, hkv=4, NL=1, rot=128, interleaved=False, f32=False, far=4000, gain=1.0, fused=True,
                 skew=0, own_caches=False):
        rng = self.rng = np.random.default_rng(seed)
        self.n, self.hq, self.hkv, self.NL, self.rot, self.interleaved, self.gain, self.own = n, hq, hkv, NL, rot, interleaved, gain, own_caches
        dt = torch.float32 if f32 else torch.bfloat16
        values = (hq + 2 * hkv) * D
        buf = torch.randn((NL * n * values + 64,), device="cuda", generator=torch.Generator("cuda").manual_seed(seed)).to(dt)
        x = buf[skew:skew + NL * n * values].view(NL, n, hq + 2 * hkv, D)
        self.q, self.k, self.v = x[:, :, :hq], x[:, :, hq:hq + hkv], x[:, :, hq + hkv:]
        if not fused:
            self.q, self.k, self.v = (y.contiguous() for y in (self.q, self.k, self.v))
        self.qkv = M.qkv_from_tensors(self.q, self.k, self.v)
        self.pos_np = rng.integers(0, far, size=n, endpoint=True)
        self.n_seqs = 3 if own_caches else 1
        self.rows = n + 9
        self.slot_np = rng.permutation(self.rows)[:n] if not own_caches else rng.permutation(self.rows * 3)[:n]
        self.seq_np = self.slot_np // self.rows if own_caches else np.zeros(n, dtype=np.int64)
        self.slot_np = self.slot_np % self.rows
        shape = (NL, self.n_seqs, self.rows, hkv, D)
        self.kc, self.vc = (torch.full(shape, 3.5, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        st = self.kc.stride()
        self.kv = M.make_kv(self.kc, self.vc, NL, self.rows, (st[0], st[1], st[3], st[2]))
        self.out = torch.full((NL, n, hq, D), 3.5, dtype=torch.bfloat16, device="cuda")
        if rot:
            self.freq, _ = M.murmur_rope_freqs_host(rot, 1e4)
        else:
            self.freq = np.zeros(1, dtype=np.uint64)
        self.freq_dev = torch.from_numpy(self.freq.view(np.int64)).cuda()

    def run(self, stream=None, out=None):
        rope = M.make_rope(self.rot, self.interleaved, self.freq_dev, self.gain)
        M.murmur_rope_append(rope, self.qkv, i32(self.pos_np), i32(self.slot_np), i32(self.seq_np) if self.own else None, self.n_seqs,
                             self.n, self.hq, self.hkv, D, self.out if out is None else out, self.kv, stream)
        torch.cuda.synchronize()
        return self

    def check(self, q=None):
        """A result is off by half a bf16 step (2^-8), and before that by the two products, their sum, the sine's and
        cosine's own error (below 4 of 2^-24: the angle's rounding pi / 4 of one, the series' two roundings and its rest)
        and the gain's, each relative to the pair's length: 8 x 2^-24 together."""
        q = self.q if q is None else q
        q, k, v = (x.double().cpu().numpy() for x in (q, self.k, self.v))
        out, kc, vc = (x.double().cpu().numpy() for x in (self.out, self.kc, self.vc))
        left = np.ones(kc.shape[:3], dtype=bool)
        i = np.arange(self.rot // 2)
        re, im = (2 * i, 2 * i + 1) if self.interleaved else (i, i + self.rot // 2)
        for t in range(self.n):
            if self.pos_np[t] < 0:
                assert (out[:, t] == 3.5).all(), t
                continue
            part = OD.turns(self.pos_np[t], self.freq[:self.rot // 2])

            def close(got, x, what):
                want = OD.rotate(x, part, self.rot, self.interleaved, self.gain)
                size = np.abs(want)
                size[..., re] = size[..., im] = abs(self.gain) * np.hypot(x[..., re], x[..., im])
                bound = 2.0 ** -8 * np.abs(want) + 8 * 2.0 ** -24 * 2 * size
                assert (np.abs(got - want) <= bound).all(), (what, t, float(np.max(np.abs(got - want) - bound)))

            close(out[:, t], q[:, t], "q")
            if 0 <= self.slot_np[t] < self.rows and 0 <= self.seq_np[t] < self.n_seqs:
                at = (slice(None), self.seq_np[t], self.slot_np[t])
                left[at] = False
                close(kc[at], k[:, t], "k")
                assert np.array_equal(vc[at], self.v[:, t].to(torch.bfloat16).double().cpu().numpy()), t
        assert (kc[left] == 3.5).all() and (vc[left] == 3.5).all()
        return self


@pytest.mark.parametrize("rot", [0, 2, 16, 50, 64, 96, 126, 128])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("f32", [False, True])
def test_rope(rot, interleaved, f32):
    announce(f"rope rot {rot} interleaved {interleaved} f32 {f32}")
    Rope(rot, 13, rot=rot, interleaved=interleaved, f32=f32, NL=2, gain=1.25).run().check()


@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 63, 64, 65, 257])
def test_rope_tokens(n):
    announce(f"rope {n} tokens")
    Rope(n, n, fused=bool(n % 2), own_caches=n % 3 == 0).run().check()


@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 4), (16, 1), (7, 7), (28, 4), (64, 8), (128, 16)])
def test_rope_heads(hq, hkv):
    announce(f"rope heads {hq}/{hkv}")
    Rope(hq, 6, hq=hq, hkv=hkv, NL=3).run().check()


@pytest.mark.parametrize("skew", [1, 2, 4, 8])
@pytest.mark.parametrize("f32", [False, True])
def test_rope_alignments(skew, f32):
    announce(f"rope skew {skew} f32 {f32}")
    Rope(skew, 9, skew=skew, f32=f32).run().check()
    Rope(skew, 9, skew=skew, f32=f32, rot=64, interleaved=True, hq=3, hkv=1).run().check()


def test_rope_far_positions():
    """Positions up to 2^31 - 1: the turn is an integer product, so nothing is lost."""
    announce("rope far positions")
    case = Rope(7, 40, far=2 ** 31 - 1)
    case.pos_np[:3] = [2 ** 31 - 1, 2 ** 30, 0]
    case.run().check()
    for kind in range(5):
        f, gain = M.murmur_rope_freqs_host(96, 5e5, kind, 8.0, 8192.0)
        case = Rope(8 + kind, 20, far=1 << 20, rot=96, gain=gain)
        case.freq, case.freq_dev = f, torch.from_numpy(f.view(np.int64)).cuda()
        case.run().check()


def test_rope_tokens_that_are_not_there_or_not_kept():
    announce("rope: absent tokens, slots out of range")
    case = Rope(9, 30)
    case.pos_np[::4] = -1
    case.slot_np[1::4] = -1
    case.q[:, ::4] = float("nan")
    case.run().check()
    assert M.murmur_device_error() == 0
    for slot, seq in ((case.rows, 0), (2 ** 31 - 1, 0), (0, 3), (0, -1), (5, 2 ** 31 - 1)):
        case = Rope(10, 12, own_caches=True)
        case.slot_np[7], case.seq_np[7] = slot, seq
        case.run().check()
        assert M.murmur_device_error() == M.MURMUR_DEVERR_POSITION


def test_rope_in_place():
    """q_out may be q itself."""
    announce("rope in place")
    for rot, interleaved in ((128, False), (50, False), (50, True), (16, True)):
        case = Rope(11, 21, fused=False, rot=rot, interleaved=interleaved)
        before = case.q.clone()
        case.out = case.q
        case.run().check(q=before)


@pytest.mark.parametrize("rot,skew", [(64, 0), (50, 0), (50, 1)])
def test_rope_values_that_are_not_finite(rot, skew):
    """An infinity or a NaN stays in its pair; V and the part that is not rotated pass as they are."""
    announce(f"rope not finite, rot {rot} skew {skew}")
    case = Rope(12, 3, rot=rot, skew=skew)
    case.q[0, 1, 2, 3], case.k[0, 1, 0, 100], case.v[0, 2, 1, 7] = float("nan"), float("inf"), float("-inf")
    case.run()
    out = case.out.cpu()
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[0, 1, 2, [3, 3 + rot // 2]] = True
    assert torch.equal(~torch.isfinite(out), bad)
    assert float(case.kc[0, 0, case.slot_np[1], 0, 100]) == float("inf") and int((~torch.isfinite(case.kc)).sum()) == 1
    assert float(case.vc[0, 0, case.slot_np[2], 1, 7]) == float("-inf") and int((~torch.isfinite(case.vc)).sum()) == 1


# ---- accept ---------------------------------------------------------------------------------------------------------

class Accept:
    def __init__(self, seed, parent, NL=1, hkv=4, agree=0.8, block_rows=None, own_caches=False):
        rng = self.rng = np.random.default_rng(seed)
        self.parent_np = np.array(parent, dtype=np.int32)
        B, T = self.B, self.T = len(self.parent_np), self.parent_np.shape[1]
        self.NL, self.hkv, self.own = NL, hkv, own_caches
        self.token_np = rng.integers(0, 40, size=(B, T)).astype(np.int32)  # few tokens: siblings that are alike
        self.said_np = np.full((B, T), 99, dtype=np.int32)
        for b in range(B):
            for t in range(T):
                kids = np.flatnonzero(self.parent_np[b] == t)
                if len(kids) and rng.random() < agree:
                    self.said_np[b, t] = self.token_np[b, rng.choice(kids)]
        self.rows = B * T + 5 if not own_caches else T + 5
        self.slot_np = (rng.permutation(self.rows)[:B * T].reshape(B, T) if not own_caches
                        else np.stack([rng.permutation(self.rows)[:T] for _ in range(B)])).astype(np.int32)
        self.k_tree, self.v_tree = bf16(rng, NL, B, T, hkv, D), bf16(rng, NL, B, T, hkv, D)
        shape = (NL, B if own_caches else 1, self.rows, hkv, D)
        self.kc, self.vc = (torch.full(shape, 3.5, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        st = self.kc.stride()
        self.kv = M.make_kv(self.kc, self.vc, NL, self.rows, (st[0], st[1] if own_caches else 0, st[3], st[2]))
        self.path, self.count, self.last = i32(np.full((B, T), -7)), i32(np.full(B, -7)), i32(np.full(B, -7))

    def run(self, shared_tree=False):
        parent = i32(self.parent_np[0] if shared_tree else self.parent_np)
        M.murmur_tree_accept(parent, int(not shared_tree), self.T, i32(self.token_np), i32(self.said_np), i32(self.slot_np), self.B,
                             self.k_tree, self.v_tree, self.kv, self.hkv, self.path, self.count, self.last)
        torch.cuda.synchronize()
        return self

    def check(self, absent=()):
        left = torch.ones(self.kc.shape[:3], dtype=torch.bool)
        lengths = []
        for b in range(self.B):
            path, last = ([], -1) if b in absent else OD.accept(self.parent_np[b], self.token_np[b], self.said_np[b])
            assert self.path[b].tolist() == path + [-1] * (self.T - len(path)), b
            assert int(self.count[b]) == len(path) and int(self.last[b]) == last, b
            lengths.append(len(path))
            for i, t in enumerate(path):
                row = int(self.slot_np[b, i])
                if not 0 <= row < self.rows:
                    continue
                at = (slice(None), b if self.own else 0, row)
                left[at] = False
                assert torch.equal(self.kc[at], self.k_tree[:, b, t]) and torch.equal(self.vc[at], self.v_tree[:, b, t]), (b, i)
        assert (self.kc.cpu()[left] == 3.5).all() and (self.vc.cpu()[left] == 3.5).all()
        return lengths


@pytest.mark.parametrize("T", [1, 2, 7, 33, 63, 64])
@pytest.mark.parametrize("own", [False, True])
def test_accept(T, own):
    announce(f"accept T {T} own {own}")
    rng = np.random.default_rng(T)
    parent = np.stack([random_tree(rng, T, wide=1 + i % 4, gone=min(i, T - 1) if i % 2 else 0) for i in range(9)])
    lengths = Accept(T, parent, NL=3, own_caches=own, agree=0.95).run().check()
    assert T == 1 or max(lengths) > 1
    case = Accept(T + 1, np.stack([parent[0]] * 4), hkv=1, own_caches=own)
    case.run(shared_tree=True).check()


def test_accept_a_whole_chain_and_nothing():
    announce("accept: whole chain, nothing")
    T = 64
    chain = np.arange(-1, T - 1, dtype=np.int32)
    assert Accept(1, np.stack([chain] * 3), NL=28, agree=1.0).run().check() == [T] * 3
    assert Accept(2, np.stack([chain] * 3), agree=0.0).run().check() == [1] * 3


def test_accept_what_is_not_there():
    announce("accept: absent sequences, tokens, slots")
    rng = np.random.default_rng(3)
    case = Accept(3, np.stack([random_tree(rng, 20) for _ in range(5)]), agree=1.0)
    case.token_np[1, 0] = -1
    case.parent_np[2] = -2
    case.token_np[3, 5:] = -4
    case.said_np[3, 4] = -4
    case.slot_np[4, 1:3] = -1
    case.run().check()
    assert M.murmur_device_error() == 0


def test_accept_device_errors():
    announce("accept: device errors")
    rng = np.random.default_rng(4)
    trees = np.stack([random_tree(rng, 6) for _ in range(3)])
    for bad in ([0, 0, 1, 1, 2, 2], [-1, -1, 0, 0, 0, 0], [-1, 1, 0, 0, 0, 0], [-1, 0, -2, 2, 0, 0], [-2, 0, 0, 0, 0, 0],
                [-1, 0, -3, 0, 0, 0], [-1, 0, 0, 2 ** 31 - 1, 0, 0]):
        case = Accept(5, trees)
        case.parent_np[1] = bad
        case.run().check(absent=[1])
        assert M.murmur_device_error() == M.MURMUR_DEVERR_TREE, bad
    case = Accept(6, trees, agree=1.0)
    case.slot_np[0, 0], case.slot_np[2, 1] = case.rows, 2 ** 31 - 1
    case.run().check()
    assert M.murmur_device_error() == M.MURMUR_DEVERR_POSITION
