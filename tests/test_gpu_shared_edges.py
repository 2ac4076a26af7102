"""Calls on shared pages and shared prefixes at the edge of what their arguments allow."""
import numpy as np
import pytest
import torch

from oracle import shared as OS
from paper_2606_01483_amd import murmur as M
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
