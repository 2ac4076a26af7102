"""Calls on shared pages and shared prefixes at the edge of what their arguments allow."""
import numpy as np
import pytest
import torch

from oracle import shared as OS
from paper_2606_01483_amd import murmur as M
from _shared import attn_bounds
from test_gpu_shared_attn import CUT, Case, bf16
from test_gpu_shared_pages import Device, grown_pool, i32

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


@pytest.mark.parametrize("block", [4, 9, 15])
def test_a_current_block_behind_the_pools_blocks(block):
    """An entry of n_blocks or more under the current token, in a pool that has rows there: reported, nothing written."""
    announce(f"current block {block} of 4, 16 in the pool")
    st = {"table": np.array([[0], [block], [1], [1]], dtype=np.int32), "stack": [2, 3]}
    st["ref"] = np.array([1, 2, 0, 0], dtype=np.int32)
    d = Device(st)
    k, v, kv = grown_pool(np.random.default_rng(2), 2, 64, 1)
    before = k.clone(), v.clone()
    seg = np.array([[0, 0, 0, 2], [0, 0, 0, 3], [0, 0, 0, 3], [0, 0, 0, 2]], dtype=np.int32)
    pol = np.tile(np.array([-1, 0, 0, -1, 0], dtype=np.int32), (4, 1))
    new = torch.full((2, 4, 1, 128), 77, dtype=torch.int16, device="cuda")
    d.step(i32(seg), i32(pol), 4, True, kv, 1, new, new)
    torch.cuda.synchronize()
    assert M.murmur_device_error() == M.MURMUR_DEVERR_BLOCK
    assert d.copied.cpu().tolist() == [-1, -2, -1, 1]
    assert d.table.cpu().tolist() == [[0], [block], [1], [3]]
    assert d.ref.cpu().tolist() == [1, 1, 0, 1] and int(d.top.item()) == 1
    for x, y in zip((k, v), before):
        y[:, 1] = 77
        y[:, 4 + 2] = 77
        y[:, 12] = y[:, 4]
        y[:, 12 + 1] = 77
        assert torch.equal(x, y)


def own_caches(lists, extra_keep, stride_b=True):
    """Lists of positions over sequence-ordered caches [1, B, 2, 64, 128] (one for all without stride_b)."""
    rng = np.random.default_rng(41)
    B, keep = len(lists), max(len(x) for x in lists) + extra_keep
    idx = np.full((B, keep), -1, dtype=np.int32)
    for b, x in enumerate(lists):
        idx[b, :len(x)] = x
    q, k, v = bf16(rng, 1, B, 4, 128), bf16(rng, 1, B, 2, 64, 128), bf16(rng, 1, B, 2, 64, 128)
    if not stride_b:
        k[:], v[:] = k[:, :1].clone(), v[:, :1].clone()
    kv = M.make_kv(k, v, 1, 64, (B * 2 * 64 * 128, 2 * 64 * 128 if stride_b else 0, 64 * 128, 128))
    return q, k, v, kv, i32(idx), i32([len(x) for x in lists]), keep


@pytest.mark.parametrize("extra_keep", [0, CUT])
@pytest.mark.parametrize("refused,group,find,stride_b", [
    (True, [0, 2, 3], True, True),     # equal positions of two caches: other rows
    (False, [0, 2, 3], False, True),   # the caller's promise
    (False, [0, 1, 2, 3], True, True),  # every sequence by itself
    (False, [0, 1, 3], True, True),    # two that share nothing
    (False, [0, 2, 3], True, False),   # one cache for all
])
def test_shares_found_in_caches_of_their_own(refused, group, find, stride_b, extra_keep):
    """Equal positions are the same rows in one cache only: found shares are refused where sequences have their own."""
    announce(f"groups {group}, find {find}, caches of their own {stride_b}, +{extra_keep}")
    lists = [list(range(40)), list(range(35)) + [50, 51], [9] + list(range(20, 45))]
    q, k, v, kv, idx, count, keep = own_caches(lists, extra_keep, stride_b)
    n = len(group) - 1
    ws_bytes, plan_bytes = M.murmur_decode_attn_shared_workspace(1, 3, 4, 2, keep, n)
    ws, plan = (torch.zeros(x // 4, dtype=torch.int32, device="cuda") for x in (ws_bytes, plan_bytes))
    out, lse, shared = torch.full((1, 3, 4, 128), 55.0, device="cuda"), torch.full((1, 3, 4), 55.0, device="cuda"), i32([20] + [0] * (n - 1))
    if not find:
        for x in (k, v):
            x[0, 1, :, :20] = x[0, 0, :, :20]
    M.murmur_shared_plan(idx, None, count, keep, 3, i32(group), n, shared, find, 1, 4, 2, plan, plan_bytes)
    M.murmur_decode_attn_shared(q, kv, idx, None, keep, 3, n, 4, 2, 128, 0.1, out, M.MURMUR_DTYPE_F32, lse, plan, plan_bytes,
                                ws, ws_bytes)
    torch.cuda.synchronize()
    if refused:
        assert M.murmur_device_error() == M.MURMUR_DEVERR_GROUP
        assert torch.isnan(out).all() and torch.isnan(lse).all()
        return
    assert M.murmur_device_error() == 0
    for b, x in enumerate(lists):
        rows = [y[0, b].float().cpu().numpy()[:, x].transpose(1, 0, 2) for y in (k, v)]
        args = q[0, b].float().cpu().numpy(), *rows, 0.1
        want, want_lse = OS.attend(*args)
        far, far_lse = attn_bounds(*args, want, want_lse)
        assert (np.abs(out[0, b].cpu().numpy() - want) <= far).all(), b
        assert (np.abs(lse[0, b].cpu().numpy() - want_lse) <= far_lse).all(), b


@pytest.mark.parametrize("extra_keep", [0, CUT])
@pytest.mark.parametrize("hq,hkv", [(28, 4), (3, 3)])
def test_logits_of_minus_infinity_weigh_nothing(hq, hkv, extra_keep):
    """Keys that a caller has set to minus infinity, whole passes of them, at the start of what is shared, of a rest and
    within both: the result is the attention over the other positions."""
    announce(f"logits of minus infinity, {hq}/{hkv}, +{extra_keep}")
    c = Case(42, [(400, [300, 0, 90, 5]), (0, [64, 200]), (33, [1])], NL=2, hq=hq, hkv=hkv, extra_keep=extra_keep)
    c.q[..., 0] = c.q[..., 0].abs() + 1
    out = set(c.lists[0][:130] + c.lists[0][200:300] + c.lists[0][400:490] + c.lists[2][400:440] + c.lists[5][:150])
    c.k[:, sorted(out), :, 0] = float("-inf")
    c.make_plan()
    c.attend()
    kept = [[x for x in xs if x not in out] for xs in c.lists]
    assert min(len(x) for x in kept) > 4
    c.lists = kept
    c.check()
    assert M.murmur_device_error() == 0


@pytest.mark.parametrize("extra_keep", [0, CUT])
@pytest.mark.parametrize("common", [40, 1500])
def test_groups_of_nothing_but_counts_too_large(common, extra_keep):
    """Counts above max_keep are errors of the count alone: a group without a valid list shares nothing and reads
    nothing, and one whose first list is too long shares what the others' lists have in common with it."""
    announce(f"counts too large, common {common}, +{extra_keep}")
    c = Case(43, [(common, [10]), (common, [3, 5, 9]), (20, [4, 0]), (7, [1, 2])], hq=8, hkv=2, extra_keep=extra_keep)
    for b in (0, 1, 4, 5):
        c.count[b] = c.keep + 1
    c.make_plan()
    c.attend()
    torch.cuda.synchronize()
    assert M.murmur_device_error() == M.MURMUR_DEVERR_COUNT
    assert c.shared.cpu().tolist() == [0, common, 0, 7]
    assert torch.isnan(c.out[:, [0, 1, 4, 5]]).all() and torch.isnan(c.lse[:, [0, 1, 4, 5]]).all()
    c.check([2, 3, 6, 7])
