"""Argument checks, sizes and the rotation's host table of the calls of murmur_draft.h (no GPU: every call here is
refused, or fails at its first HIP call, so the module is skipped where a GPU is visible)."""
import ctypes
import math
import os
import re
from decimal import Decimal, localcontext

import numpy as np
import pytest
import torch

from paper_2606_01483_amd import murmur as M

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="host-only checks run where no GPU is visible")

FAKE = 0x100000  # never dereferenced


def kv(**over):
    f = dict(k=FAKE, v=FAKE, n_layers=2, max_len=4096, stride_layer=4096 * 512, stride_b=0, stride_h=128, stride_pos=512)
    return M.murmur_kv(*{**f, **over}.values())


def rope(**over):
    f = dict(rot_dim=128, interleaved=0, gain=1.0, freq=FAKE)
    return M.murmur_rope(*{**f, **over}.values())


def qkv(**over):
    f = dict(q=FAKE, k=FAKE, v=FAKE, dtype=M.MURMUR_DTYPE_BF16, q_layer=0, q_token=4608, kv_layer=0, kv_token=4608)
    return M.murmur_qkv(*{**f, **over}.values())


WS = dict(ws_dev=FAKE, ws_bytes=1 << 30)
TREE = dict(parent_dev=FAKE, parent_per_seq=1, n_nodes=16)
CALLS = {
    "murmur_paged_reserve": dict(len_dev=FAKE, new_dev=FAKE, B=12, block_table_dev=FAKE, max_blocks=64, block_size=16,
                                 ref_dev=FAKE, n_blocks=256, free_stack_dev=FAKE, free_top_dev=FAKE, capacity=256, per_seq=8,
                                 n_tokens=96, start_dev=FAKE, got_dev=FAKE, slot_dev=FAKE, pos_dev=FAKE, seq_dev=FAKE, **WS,
                                 stream=0),
    "murmur_rope_append": dict(rope=rope(), qkv=qkv(), pos_dev=FAKE, slot_dev=FAKE, seq_dev=FAKE, n_seqs=1, n_tokens=96, Hq=28,
                               Hkv=4, D=128, q_out_dev=FAKE, kv=kv(), stream=0),
    "murmur_decode_attn_tree": dict(seg_dev=FAKE, pol_dev=FAKE, pol_per_seq=3, **TREE, q_dev=FAKE, kv=kv(), k_tree_dev=FAKE,
                                    v_tree_dev=FAKE, block_table_dev=FAKE, max_blocks=64, block_size=16, max_keep=900, B=12,
                                    Hq=28, Hkv=4, D=128, scale=1.0, out_dev=FAKE, out_dtype=M.MURMUR_DTYPE_BF16, lse_dev=None,
                                    **WS, stream=0),
    "murmur_tree_accept": dict(**TREE, token_dev=FAKE, next_dev=FAKE, slot_dev=FAKE, B=12, k_tree_dev=FAKE, v_tree_dev=FAKE,
                               kv=kv(), Hkv=4, path_dev=FAKE, count_dev=FAKE, last_dev=FAKE, stream=0),
}


def outcome(name, **over):
    try:
        getattr(M, name)(**{**CALLS[name], **over})
    except M.MurmurError as e:
        return e.code, M.murmur_last_error()
    except (TypeError, AttributeError, OverflowError, ctypes.ArgumentError):
        return "refused"
    return "returned"


@pytest.fixture(params=["converter", "ctypes"])
def route(request, monkeypatch):
    lib = M.lib()
    if request.param == "converter":
        if M._pycall is None:
            pytest.skip("built without the converter")
        assert all(lib.per_step[n][2] is not None for n in M._PER_STEP_DRAFT)
    else:
        monkeypatch.setattr(lib, "per_step", {n: (fn, at, None) for n, (fn, at, _) in lib.per_step.items()})


def test_exports_every_declared_function():
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "murmur_draft.h")).read()
    names = set(re.findall(r"^int (murmur_\w+)\(", header, re.M))
    assert names == set(CALLS) | {"murmur_paged_reserve_workspace", "murmur_rope_freqs_host", "murmur_decode_attn_tree_workspace"}
    for n in names:
        assert hasattr(ctypes.CDLL(M.LIB_PATH), n) and callable(getattr(M, n)), n


def test_every_call_is_here():
    assert sorted(CALLS) == sorted("murmur_" + n for n in M._PER_STEP_DRAFT)


def test_structures():
    assert ctypes.sizeof(M.murmur_rope) == 24 and ctypes.sizeof(M.murmur_qkv) == 64


@pytest.mark.parametrize("name", sorted(CALLS))
def test_the_call_arrives(route, name):
    assert outcome(name)[0] == M.MURMUR_EHIP
    for arg in ("ref_dev", "pos_dev", "seq_dev", "lse_dev"):
        if arg in CALLS[name] and (name, arg) != ("murmur_rope_append", "pos_dev"):
            assert outcome(name, **{arg: None})[0] == M.MURMUR_EHIP, arg
    for arg, x in (("kv", M.murmur_seg()), ("rope", M.murmur_kv()), ("qkv", M.murmur_rope()), ("B", "12"), ("n_tokens", 1.5)):
        if arg in CALLS[name]:
            assert outcome(name, **{arg: x}) == "refused", arg


INVALID = {
    "murmur_paged_reserve": dict(B=(0, -1, 65536), max_blocks=(0, 1 << 27), block_size=(0, 3, 1 << 21), n_blocks=(0, (1 << 30) + 1, 1 << 28),
                                 capacity=(255,), per_seq=(-1, 9), n_tokens=(0, 95)),
    "murmur_rope_append": dict(n_seqs=(0,), n_tokens=(0, -5), Hq=(0, 65536), Hkv=(0, 65536),
                               rope=(rope(rot_dim=-2), rope(rot_dim=3), rope(rot_dim=130), rope(interleaved=2), rope(gain=math.inf),
                                     rope(gain=math.nan), rope(freq=0), rope(freq=FAKE + 4)),
                               qkv=(qkv(q=0), qkv(k=0), qkv(v=0), qkv(dtype=7), qkv(q=FAKE + 1), qkv(dtype=2, k=FAKE + 2),
                                    qkv(q_token=-1), qkv(kv_layer=-8))),
    "murmur_decode_attn_tree": dict(pol_per_seq=(-1, 4), parent_per_seq=(2, -1), n_nodes=(0, -1), B=(0,), Hq=(0, 27), Hkv=(0, 5), max_keep=(0,),
                                    max_blocks=(0,), block_size=(0, 12), scale=(math.inf, math.nan), out_dtype=(0, 3),
                                    kv=(kv(stride_b=4096 * 512),)),
    "murmur_tree_accept": dict(parent_per_seq=(2,), n_nodes=(0,), B=(0, 65536), Hkv=(0, 65536)),
}
KV = (kv(k=0), kv(v=0), kv(n_layers=0), kv(max_len=0), kv(stride_pos=64), kv(stride_h=4), kv(stride_layer=-8), kv(k=FAKE + 8), kv(v=FAKE + 2))


@pytest.mark.parametrize("name", sorted(CALLS))
def test_invalid_arguments(route, name):
    for arg, values in INVALID[name].items():
        for x in values:
            got = outcome(name, **{arg: x})
            assert got[0] == M.MURMUR_EINVAL and got[1], (arg, x, got)
    for x in KV if "kv" in CALLS[name] else ():
        assert outcome(name, kv=x)[0] == M.MURMUR_EINVAL
    optional = {"ref_dev", "pos_dev", "seq_dev", "lse_dev"} - ({"pos_dev"} if name == "murmur_rope_append" else set())
    wide = {"q_dev", "k_tree_dev", "v_tree_dev", "out_dev", "q_out_dev"}
    for arg in CALLS[name]:
        if arg.endswith("_dev") and arg not in optional | {"block_table_dev"}:
            assert outcome(name, **{arg: None})[0] == M.MURMUR_EINVAL, arg
        if arg.endswith("_dev"):
            assert outcome(name, **{arg: FAKE + (128 if arg == "ws_dev" else 8 if arg in wide else 2)})[0] == M.MURMUR_EINVAL, arg
    if "ws_bytes" in CALLS[name]:
        assert outcome(name, ws_bytes=1)[0] == M.MURMUR_ENOSPACE


def test_unsupported_sizes(route):
    for over in (dict(D=64), dict(n_nodes=65), dict(Hq=68, Hkv=4), dict(max_keep=(1 << 28) + 1)):
        assert outcome("murmur_decode_attn_tree", **over)[0] == M.MURMUR_EUNSUPPORTED, over
    assert outcome("murmur_tree_accept", n_nodes=65)[0] == M.MURMUR_EUNSUPPORTED
    assert outcome("murmur_rope_append", D=256)[0] == M.MURMUR_EUNSUPPORTED


def test_caches_of_the_sequences_own(route):
    own = kv(stride_b=4096 * 512)
    assert outcome("murmur_decode_attn_tree", kv=own, block_table_dev=None, max_blocks=0, block_size=0)[0] == M.MURMUR_EHIP
    for over in (dict(max_blocks=1, block_size=0), dict(max_blocks=0, block_size=16)):
        assert outcome("murmur_decode_attn_tree", kv=own, block_table_dev=None, **over)[0] == M.MURMUR_EINVAL


def test_too_large_for_one_launch(route):
    assert outcome("murmur_decode_attn_tree", kv=kv(n_layers=1000), B=65535, ws_bytes=1 << 62)[0] == M.MURMUR_EINVAL
    assert outcome("murmur_rope_append", kv=kv(n_layers=1 << 20), n_tokens=1 << 20)[0] == M.MURMUR_EINVAL
    assert outcome("murmur_tree_accept", kv=kv(n_layers=1 << 17))[0] == M.MURMUR_EINVAL


def test_workspaces():
    assert M.murmur_paged_reserve_workspace(1) < M.murmur_paged_reserve_workspace(65535) < 1 << 20
    for args in ((0,), (65536,)):
        with pytest.raises(M.MurmurError):
            M.murmur_paged_reserve_workspace(*args)
    sizes = [M.murmur_decode_attn_tree_workspace(nl, B, 28, 4, T, keep) for nl in (1, 28) for B in (1, 12, 64, 400) for T in (1, 16, 64)
             for keep in (1, 200, 900, 40000)]
    assert min(sizes) == 0 and max(sizes) < 1 << 30 and all(x % 256 == 0 for x in sizes)
    for args in ((0, 1, 28, 4, 8, 100), (1, 0, 28, 4, 8, 100), (1, 1, 27, 4, 8, 100), (1, 1, 28, 4, 65, 100), (1, 1, 28, 4, 8, 0)):
        with pytest.raises(M.MurmurError):
            M.murmur_decode_attn_tree_workspace(*args)


def test_the_largest_workspace_serves_smaller_calls(route):
    """Sizes grow with the layers, the batch, the nodes and the lists: what a caller allocates once is enough for each call."""
    at = lambda nl, B, T, keep, hq=28, hkv=4: M.murmur_decode_attn_tree_workspace(nl, B, hq, hkv, T, keep)  # noqa: E731
    for sizes in ([(1, B, 16, 900) for B in range(1, 130)], [(1, 12, T, 2000) for T in range(1, 65)], [(nl, 3, 9, 700) for nl in range(1, 99)],
                  [(1, 12, 16, keep) for keep in range(1, 5000, 7)], [(1, 1, 31, 1 << i) for i in range(29)]):
        got = [at(*x) for x in sizes]
        assert got == sorted(got), sizes[0]
    rng = np.random.default_rng(3)
    for _ in range(3000):
        hkv = int(rng.integers(1, 9))
        hq = hkv * int(rng.integers(1, 17))
        large = [int(np.exp2(rng.uniform(0, top))) for top in (5, 8, 6, 17)]
        small = [int(rng.integers(1, x + 1)) for x in large]
        most = at(*large, hq, hkv)
        assert at(*small, hq, hkv) <= most <= 98 << 20, (small, large, hq, hkv)
        nl, B, T, keep = small
        got = outcome("murmur_decode_attn_tree", kv=kv(n_layers=nl), B=B, n_nodes=T, max_keep=keep, Hq=hq, Hkv=hkv, ws_dev=FAKE if most else None,
                      ws_bytes=most)
        assert got[0] == M.MURMUR_EHIP, (small, large, hq, hkv, got)


# ---- the rotation's table ------------------------------------------------------------------------------------------

def as_turns(freq):
    return [int(x) / 2.0 ** 64 for x in freq]


@pytest.mark.parametrize("rot", [2, 50, 64, 128])
@pytest.mark.parametrize("base", [1.5, 1e4, 5e5, 1e6])
def test_frequencies(rot, base):
    """To a 2^-50 of their own, or to the table's step of 2^-64."""
    i = np.arange(rot // 2)
    plain = np.array([math.exp(-2.0 * k / rot * math.log(base)) for k in i]) / (2 * math.pi)

    def close(kind, want, gain=1.0, **kw):
        f, g = M.murmur_rope_freqs_host(rot, base, kind, 8.0, 4096.0, **kw)
        assert f.dtype == np.uint64 and len(f) == rot // 2 and abs(g - gain) <= 2.0 ** -24 * gain
        assert np.all(np.abs(np.array(as_turns(f)) - want) <= 2.0 ** -46 * want + 2.0 ** -64)

    close(M.MURMUR_ROPE_PLAIN, plain)
    close(M.MURMUR_ROPE_LINEAR, plain / 8)
    if rot > 2:
        close(M.MURMUR_ROPE_BASE, plain * 8.0 ** (-2.0 * i / (rot - 2)))
    keep = np.clip((4096 * plain - 1) / 31, 0, 1)
    close(M.MURMUR_ROPE_BANDS, plain * (keep + (1 - keep) / 8))
    close(M.MURMUR_ROPE_YARN, plain * (keep + (1 - keep) / 8), gain=1 + 0.1 * math.log(8))
    keep = np.clip((4096 * plain - 0.5) / 3.5, 0, 1)
    close(M.MURMUR_ROPE_BANDS, plain * (keep + (1 - keep) / 8), slow_turns=0.5, fast_turns=4.0)


def in_60_digits(rot, base, kind, factor=1.0, original=0.0, slow=1.0, fast=32.0):
    """The table's entries in steps of 2^-64, unrounded."""
    with localcontext() as c:
        c.prec = 60
        pi = Decimal("3.14159265358979323846264338327950288419716939937510582097494")
        b, factor, slow, fast = Decimal(base), Decimal(factor), Decimal(slow), Decimal(fast)
        if kind == M.MURMUR_ROPE_BASE and rot > 2:
            b *= (factor.ln() * rot / (rot - 2)).exp()
        got = []
        for i in range(rot // 2):
            f = (b.ln() * -2 * i / rot).exp() / (2 * pi)
            if kind == M.MURMUR_ROPE_LINEAR:
                f /= factor
            if kind in (M.MURMUR_ROPE_BANDS, M.MURMUR_ROPE_YARN):
                keep = min(Decimal(1), max(Decimal(0), (Decimal(original) * f - slow) / (fast - slow)))
                f = f * keep + f / factor * (1 - keep)
            got.append(f * 2 ** 64)
        return got


@pytest.mark.parametrize("kind", [M.MURMUR_ROPE_PLAIN, M.MURMUR_ROPE_LINEAR, M.MURMUR_ROPE_BASE, M.MURMUR_ROPE_BANDS, M.MURMUR_ROPE_YARN])
@pytest.mark.parametrize("rot", [2, 50, 64, 128])
@pytest.mark.parametrize("base", [1.5, 1e4, 5e5, 1e6])
def test_frequencies_to_two_steps(rot, base, kind):
    """Within two steps of 2^-64, so that position 2^31 is turned to 2^-32 of a turn.  A value of at most 2^61.4 steps takes
    roundings of 2^-64 of it, 0.16 steps each: the power (an ulp, two of them), its argument (ln(base) x base^-x / (2 pi) of
    them, at most 0.06 steps; three times that where the base is a product of a power), two divisions; in the bands a share's
    six, of frequencies below 32 / 4096, and three more; the last rounding half a step.  0.5 + 0.32 + 0.18 + 0.32 + 0.48."""
    f, _ = M.murmur_rope_freqs_host(rot, base, kind, 8.0, 4096.0)
    off = [abs(int(x) - want) for x, want in zip(f, in_60_digits(rot, base, kind, 8.0, 4096.0))]
    assert max(off) <= 2, float(max(off))


def test_the_slowest_pair_takes_the_factor():
    plain, _ = M.murmur_rope_freqs_host(128, 1e4)
    scaled, _ = M.murmur_rope_freqs_host(128, 1e4, M.MURMUR_ROPE_BASE, 4.0)
    assert plain[0] == scaled[0] and abs(int(plain[-1]) / int(scaled[-1]) - 4.0) < 1e-9


@pytest.mark.parametrize("args", [(0, 1e4), (3, 1e4), (130, 1e4), (128, 1.0), (128, math.inf), (128, math.nan), (128, 1e4, 5),
                                  (128, 1e4, -1), (128, 1e4, 1, 0.5), (128, 1e4, 2, math.inf), (128, 1e4, 3, 2.0, 0.0),
                                  (128, 1e4, 4, 2.0, 4096.0, 2.0, 2.0), (128, 1e4, 4, 2.0, 4096.0, -1.0, 2.0),
                                  (128, 1e4, 4, 2.0, 4096.0, 1.0, math.inf), (4, 1e300, 2, 1e300)])
def test_frequencies_refused(args):
    with pytest.raises(M.MurmurError):
        M.murmur_rope_freqs_host(*args)


def test_projections_from_tensors():
    x = torch.zeros((2, 5, 12, 128), dtype=torch.bfloat16)
    got = M.qkv_from_tensors(x[:, :, :8], x[:, :, 8:10], x[:, :, 10:])
    assert (got.q_layer, got.q_token, got.kv_layer, got.kv_token) == (7680, 1536, 7680, 1536) and got.dtype == M.MURMUR_DTYPE_BF16
    assert got.k == x.data_ptr() + 8 * 256 and got.v == x.data_ptr() + 10 * 256
    for q, k, v in ((x.float(), x, x), (x, x, x[:, :, :6]), (x.half(), x.half(), x.half()), (x.transpose(1, 2), x, x), (x[..., ::2], x, x)):
        with pytest.raises(ValueError):
            M.qkv_from_tensors(q, k, v)


@pytest.mark.parametrize("shape", [(2, 5), (4, 5), (2, 3, 5), (15,), (3, 4), (0, 5)])
def test_policies_of_a_batch_of_trees(shape):
    """Records for another number of sequences would be read past their end, those of layers for sequences."""
    from paper_2606_01483_amd.decode import TreeBatch
    seg = np.array([[4, 30, 0, 1]] * 3)
    rest = dict(n_nodes=4, rope=rope(), n_layers=2, hq=8, hkv=2, block_size=8, n_blocks=16, max_len=64, max_keep=40, scale=1.0,
                device="cpu")
    with pytest.raises(ValueError):
        TreeBatch(seg, np.full(shape, -1), **rest)
    for good in ((5,), (1, 5), (3, 5)):
        assert TreeBatch(seg, np.full(good, -1), **rest).pol.shape[0] == (3 if good == (3, 5) else 1)
