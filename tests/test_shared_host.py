"""Argument checks and sizes of the calls on shared pages and shared prefixes (no GPU: every call here is refused, or
fails at its first HIP call, so the module is skipped where a GPU is visible)."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

from paper_2606_01483_amd import murmur as M

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="host-only checks run where no GPU is visible")

FAKE = 0x100000  # never dereferenced


def kv(**over):
    f = dict(k=FAKE, v=FAKE, n_layers=2, max_len=4096, stride_layer=4096 * 512, stride_b=0, stride_h=128, stride_pos=512)
    return M.murmur_kv(*{**f, **over}.values())


PAGES = dict(block_table_dev=FAKE, max_blocks=64, ref_dev=FAKE, n_blocks=256, free_stack_dev=FAKE, free_top_dev=FAKE,
             capacity=256)
WS = dict(ws_dev=FAKE, ws_bytes=1 << 30)
CALLS = {
    "murmur_paged_fork": dict(parent_dev=FAKE, B=12, **PAGES, **WS, stream=0),
    "murmur_paged_step_shared": dict(seg_dev=FAKE, pol_dev=FAKE, pol_per_seq=1, B=12, **PAGES, block_size=16,
                                     full_scan=False, copied_dev=FAKE, pool=kv(), Hkv=4, k_new_dev=FAKE,
                                     v_new_dev=FAKE, stream=0),
    "murmur_paged_compact": dict(B=12, **PAGES, block_size=16, map_dev=FAKE, pool=kv(), Hkv=4, **WS, stream=0),
    "murmur_shared_plan": dict(idx_dev=FAKE, ranges_dev=None, count_dev=FAKE, max_keep=900, B=12, group_dev=FAKE,
                               n_groups=3, shared_dev=FAKE, find_shared=True, n_layers=2, Hq=28, Hkv=4, plan_dev=FAKE,
                               plan_bytes=1 << 30, stream=0),
    "murmur_decode_attn_shared": dict(q_dev=FAKE, kv=kv(), idx_dev=FAKE, ranges_dev=None, max_keep=900, B=12,
                                      n_groups=3, Hq=28, Hkv=4, D=128, scale=1.0, out_dev=FAKE,
                                      out_dtype=M.MURMUR_DTYPE_BF16, lse_dev=None, plan_dev=FAKE, plan_bytes=1 << 30,
                                      **WS, stream=0),
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
        assert all(lib.per_step[n][2] is not None for n in M._PER_STEP_SHARED)
    else:
        monkeypatch.setattr(lib, "per_step", {n: (fn, at, None) for n, (fn, at, _) in lib.per_step.items()})


def test_exports_every_declared_function():
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "murmur_shared.h")).read()
    names = set(re.findall(r"^int (murmur_\w+)\(", header, re.M))
    assert names == set(CALLS) | {"murmur_paged_workspace", "murmur_decode_attn_shared_workspace"}
    for n in names:
        assert hasattr(ctypes.CDLL(M.LIB_PATH), n) and callable(getattr(M, n)), n


def test_every_call_is_here():
    assert sorted(CALLS) == sorted("murmur_" + n for n in M._PER_STEP_SHARED)


@pytest.mark.parametrize("name", sorted(CALLS))
def test_the_call_arrives(route, name):
    assert outcome(name)[0] == M.MURMUR_EHIP
    for arg, value in CALLS[name].items():
        if type(value) is int and not arg.endswith("_dev") and arg != "stream":
            assert outcome(name, **{arg: np.int64(value)})[0] == M.MURMUR_EHIP, arg


E, U, S = M.MURMUR_EINVAL, M.MURMUR_EUNSUPPORTED, M.MURMUR_ENOSPACE
PAGE_FAULTS = [("block_table_dev", None, E, "NULL"), ("ref_dev", None, E, "NULL"), ("free_stack_dev", None, E, "NULL"),
               ("free_top_dev", None, E, "NULL"), ("block_table_dev", FAKE + 2, E, "aligned"),
               ("ref_dev", FAKE + 2, E, "aligned"), ("free_stack_dev", FAKE + 1, E, "aligned"),
               ("free_top_dev", FAKE + 2, E, "aligned"), ("B", 0, E, "B must"), ("B", 65536, E, "B must"),
               ("max_blocks", 0, E, "max_blocks"), ("max_blocks", 1 << 27, E, "2^30"), ("n_blocks", 0, E, "n_blocks"),
               ("n_blocks", (1 << 30) + 1, E, "n_blocks"), ("n_blocks", 257, E, "capacity"), ("capacity", 255, E, "capacity")]
POOL_FAULTS = [("block_size", 0, E, "power of two"), ("block_size", 12, E, "power of two"),
               ("block_size", 1 << 21, E, "power of two"), ("block_size", 32, E, "below n_blocks"),
               ("pool", kv(k=None), E, "NULL"), ("pool", kv(n_layers=0), E, ">= 1"), ("pool", kv(max_len=4095), E, "below n_blocks"),
               ("pool", kv(stride_h=4), E, "multiples of 8"), ("pool", kv(stride_pos=64), E, "head_dim"),
               ("pool", kv(v=FAKE + 8), E, "aligned"), ("Hkv", 0, E, ">= 1"), ("Hkv", 1 << 27, E, "2^26")]
WS_FAULTS = [("ws_dev", None, E, "NULL"), ("ws_dev", FAKE + 64, E, "256-byte")]
SIZE_FAULTS = [("max_keep", 0, E, ">= 1"), ("B", 0, E, ">= 1"), ("n_groups", 0, E, "n_groups"),
               ("n_groups", 4097, E, "n_groups"), ("Hq", 27, E, "multiple"), ("Hq", 68, U, "exceeds 16"),
               ("max_keep", (1 << 28) + 1, U, "max_keep"), ("B", 4097, U, "4097 sequences"), ("plan_dev", None, E, "NULL"),
               ("plan_dev", FAKE + 8, E, "16-byte"), ("plan_bytes", 1000, S, "plan of 1000"),
               ("idx_dev", None, E, "idx_dev and ranges_dev"), ("idx_dev", FAKE + 2, E, "aligned")]
FAULTS = {
    "murmur_paged_fork": PAGE_FAULTS + WS_FAULTS + [("parent_dev", None, E, "NULL"), ("parent_dev", FAKE + 2, E, "aligned"),
                                                    ("ws_bytes", M.murmur_paged_workspace(12, 64, 256) - 1, S, "too small")],
    "murmur_paged_step_shared": PAGE_FAULTS + POOL_FAULTS + [
        ("seg_dev", None, E, "NULL"), ("pol_dev", None, E, "NULL"), ("copied_dev", None, E, "NULL"),
        ("copied_dev", FAKE + 2, E, "aligned"), ("pol_per_seq", 2, E, "pol_per_seq"), ("k_new_dev", None, E, "k_new_dev"),
        ("v_new_dev", FAKE + 8, E, "16-byte")],
    "murmur_paged_compact": PAGE_FAULTS + POOL_FAULTS + WS_FAULTS + [
        ("map_dev", None, E, "NULL"), ("map_dev", FAKE + 2, E, "aligned"), ("ws_bytes", M.murmur_paged_workspace(12, 64, 256) - 1, S, "too small")],
    "murmur_shared_plan": SIZE_FAULTS + [
        ("count_dev", None, E, "count_dev"), ("ranges_dev", FAKE, E, "find_shared"), ("group_dev", None, E, "NULL"),
        ("shared_dev", None, E, "NULL"), ("group_dev", FAKE + 2, E, "aligned"), ("shared_dev", FAKE + 2, E, "aligned"),
        ("n_layers", 0, E, ">= 1"), ("n_layers", 20000, E, "too large")],
    "murmur_decode_attn_shared": SIZE_FAULTS + WS_FAULTS + [
        ("q_dev", None, E, "NULL"), ("out_dev", None, E, "NULL"), ("kv", kv(k=None), E, "NULL"),
        ("kv", kv(n_layers=0), E, ">= 1"), ("kv", kv(max_len=0), E, ">= 1"), ("kv", kv(stride_b=4), E, "multiples of 8"),
        ("kv", kv(stride_pos=64), E, "head_dim"), ("kv", kv(k=FAKE + 8), E, "16-byte"), ("q_dev", FAKE + 8, E, "16-byte"),
        ("out_dev", FAKE + 8, E, "16-byte"), ("lse_dev", FAKE + 2, E, "4-byte"), ("D", 64, U, "head_dim"),
        ("out_dtype", 3, E, "out_dtype"), ("scale", float("inf"), E, "finite"), ("ws_bytes", 1000, S, "too small")],
}


@pytest.mark.parametrize("name", sorted(FAULTS))
def test_refusals(route, name):
    for arg, value, code, text in FAULTS[name]:
        got = outcome(name, **{arg: value})
        assert got[0] == code and text in got[1], (arg, value, got)


def test_optional_arguments():
    assert outcome("murmur_paged_step_shared", pool=None, Hkv=0, k_new_dev=None, v_new_dev=None)[0] == M.MURMUR_EHIP
    assert outcome("murmur_paged_compact", pool=None, Hkv=0)[0] == M.MURMUR_EHIP
    assert outcome("murmur_shared_plan", idx_dev=None, ranges_dev=FAKE, count_dev=None, find_shared=False)[0] == M.MURMUR_EHIP
    assert outcome("murmur_decode_attn_shared", idx_dev=None, ranges_dev=FAKE)[0] == M.MURMUR_EHIP


def test_sizes():
    assert M.murmur_paged_workspace(12, 64, 256) >= 8 * 256 + 16 * 12 * 64
    assert M.murmur_paged_workspace(1, 1, 1 << 20) >= 12 * (1 << 20)
    for bad in ((0, 1, 1), (65536, 1, 1), (1, 0, 1), (1, 1, 0), (1024, 1 << 21, 1)):
        with pytest.raises(M.MurmurError):
            M.murmur_paged_workspace(*bad)
    small = M.murmur_decode_attn_shared_workspace(1, 4, 28, 4, 200, 1)
    large = M.murmur_decode_attn_shared_workspace(28, 96, 28, 4, 4000, 12)
    assert all(x % 256 == 0 and 0 < x < y for x, y in zip(small, large))
    for bad in ((0, 1, 4, 4, 1, 1), (1, 1, 6, 4, 1, 1), (1, 1, 4, 4, 0, 1), (1, 1, 4, 4, 1, 0), (1, 1, 34, 2, 1, 1)):
        with pytest.raises(M.MurmurError):
            M.murmur_decode_attn_shared_workspace(*bad)
