"""Every form of murmur_decode_attn_shared in every instance of its kernels: index lists and range tables, rows within
32-bit offsets and beyond, fp32 and bf16 outputs, both schedules; against Equation 1 in fp64."""
import numpy as np
import pytest
import torch

import oracle
from oracle import shared as OS
from paper_2606_01483_amd import murmur as M
from _shared import attn_bounds
from test_gpu_shared_attn import CUT, bf16, i32

pytestmark = pytest.mark.gpu
D, NL, HQ, HKV, PROMPT, L = 128, 2, 28, 4, 75, 600
WIDTHS = [1, 3, 6]  # 7, 21 and 42 query rows a KV head: one, two and three row tiles


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    M.lib()
    yield
    torch.cuda.synchronize()
    assert M.murmur_device_error() == 0


def caches(rng, B, stride):
    """Two caches [NL, B, HKV, L, D] whose positions lie `stride` elements apart, and their murmur_kv."""
    got = []
    for _ in range(2):
        flat = torch.empty((L - 1) * stride + NL * B * HKV * D, dtype=torch.bfloat16, device="cuda")
        x = flat.as_strided((NL, B, HKV, L, D), (B * HKV * D, HKV * D, D, stride, 1))
        x.copy_(bf16(rng, NL, B, HKV, L, D))
        got.append(x)
    return got[0], got[1], M.make_kv(*got, NL, L, (B * HKV * D, HKV * D, D, stride))


# 33 groups: more workgroups than compute units, which the schedule of whole lists gives four wavefronts instead of eight
@pytest.mark.parametrize("extra_keep,times", [(0, 1), (CUT, 1), (0, 11)])
@pytest.mark.parametrize("f32", [True, False])
@pytest.mark.parametrize("stride", [0, 1 << 22, 1 << 23])  # the last two: over 4 GiB from first to last row
@pytest.mark.parametrize("form", ["ranges", "index", "pool"])
def test_forms(form, stride, f32, extra_keep, times):
    print(f"\n[case] {form}, stride {stride}, f32 {f32}, +{extra_keep}, {3 * times} groups", flush=True)
    rng = np.random.default_rng(61)
    group = np.concatenate([[0], np.cumsum(WIDTHS * times)])
    B, n = int(group[-1]), 3 * times
    stride = max(stride, NL * B * HKV * D)
    seg = np.stack([np.full(B, PROMPT), rng.integers(0, 400, B), rng.integers(0, 6, B), rng.integers(1, 90, B)], 1).astype(np.int32)
    pol = np.stack([np.resize([50, -1, 64, 33, -1, 7, 300], B), rng.integers(0, 40, B), rng.integers(0, 5, B),
                    np.resize([20, -1, 8, 5, -1, 30, 11], B), rng.integers(0, 3, B)], 1).astype(np.int32)
    idx, cnt = oracle.retained(seg, pol)
    keep = idx.shape[1] + extra_keep
    k, v, kv = caches(rng, B, stride)
    lead = np.repeat(group[:-1], np.diff(group))
    owner = np.arange(B)
    shared = [PROMPT, PROMPT - 5, PROMPT] * times
    d_idx, d_cnt, ranges = i32(np.zeros((B, keep))), i32(np.zeros(B)), i32(np.zeros((B, 6, 2)))
    M.murmur_evict_compact(i32(seg), i32(pol), 1, B, d_idx, keep, d_cnt, ranges)
    if form == "pool":  # one cache for all, the first sequence's
        owner[:] = 0
        kv = M.make_kv(k, v, NL, L, (B * HKV * D, 0, D, stride))
        shared = [OS.common([idx[b, :cnt[b]] for b in range(lo, hi)]) for lo, hi in zip(group[:-1], group[1:])]
    else:
        for x in (k, v):
            for b in range(B):
                x[:, b, :, :PROMPT] = x[:, lead[b], :, :PROMPT].clone()
    whole = [x.float().cpu().numpy() for x in (k, v)]
    if form != "pool":
        for x in (k, v):
            for b in range(B):
                if b != lead[b]:
                    x[:, b, :, :PROMPT - 5] = float("nan")
    q = bf16(rng, NL, B, HQ, D)
    ws_bytes, plan_bytes = M.murmur_decode_attn_shared_workspace(NL, B, HQ, HKV, keep, n)
    ws, plan = (torch.zeros(x // 4, dtype=torch.int32, device="cuda") for x in (ws_bytes, plan_bytes))
    out = torch.zeros((NL, B, HQ, D), dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
    lse, table = torch.zeros((NL, B, HQ), device="cuda"), ranges if form == "ranges" else None
    d_shared = i32(shared)
    M.murmur_shared_plan(d_idx, table, d_cnt, keep, B, i32(group), n, d_shared, form == "pool", NL, HQ, HKV, plan, plan_bytes)
    M.murmur_decode_attn_shared(q, kv, d_idx, table, keep, B, n, HQ, HKV, D, 0.11, out,
                                M.MURMUR_DTYPE_F32 if f32 else M.MURMUR_DTYPE_BF16, lse, plan, plan_bytes, ws, ws_bytes)
    torch.cuda.synchronize()
    assert M.murmur_device_error() == 0
    assert d_shared.cpu().tolist() == shared
    got, got_lse = out.float().cpu().numpy(), lse.cpu().numpy()
    for b in range(B) if times == 1 else [*range(10), *range(B - 10, B)]:
        at = idx[b, :cnt[b]]
        for layer in range(NL):
            rows = [x[layer, owner[b]][:, at].transpose(1, 0, 2) for x in whole]
            args = q[layer, b].float().cpu().numpy(), *rows, 0.11
            want, want_lse = OS.attend(*args)
            far, far_lse = attn_bounds(*args, want, want_lse)
            if not f32:  # the rounding to bf16 of a value that far off
                far = far + (np.abs(want) + far) * 2.0 ** -8
            assert (np.abs(got[layer, b] - want) <= far).all(), (b, layer)
            assert (np.abs(got_lse[layer, b] - want_lse) <= far_lse).all(), (b, layer)
