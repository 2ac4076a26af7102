"""The schedule of murmur_decode_attn_tree on the host: the ABI layer (csrc/draft.cpp) with stubs of the kernel launchers,
compiled with g++ into a small program that prints what each call would launch (no GPU).  Pins which sizes reach which
instance of the kernels, for the GPU tests that use them."""
import os
import shutil
import subprocess

import pytest

from _tree_forms import FEW, FORMS, PAIR, WIDE

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_01483_amd", "csrc")

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")

DRIVER = r"""
#include <stdio.h>
#include "internal.h"
#include "murmur_draft.h"
using namespace murmur;
static TreeLaunch got;
namespace murmur {
int launch_paged_reserve(const ReserveLaunch &, murmur_stream_t) { return 0; }
int launch_rope_append(const RopeLaunch &, murmur_stream_t) { return 0; }
int launch_decode_attn_tree(const TreeLaunch &a, murmur_stream_t) { got = a; return 0; }
int launch_tree_accept(const AcceptLaunch &, murmur_stream_t) { return 0; }
}  // namespace murmur
int main() {  // lines: layers batch Hq Hkv nodes max_keep
    void *f = (void *)0x100000;
    int nl, b, hq, hkv, nodes, keep;
    while (scanf("%d %d %d %d %d %d", &nl, &b, &hq, &hkv, &nodes, &keep) == 6) {
        size_t bytes = 0;
        murmur_decode_attn_tree_workspace(nl, b, hq, hkv, nodes, keep, &bytes);
        murmur_kv kv{f, f, nl, 1 << 20, 1LL << 40, 1LL << 32, 1LL << 28, 128};
        got = TreeLaunch{};
        const int rc = murmur_decode_attn_tree((const murmur_seg *)f, (const murmur_policy *)f, 0, (const int32_t *)f, 0, nodes, f, &kv, f, f, nullptr,
                                               0, 0, keep, b, hq, hkv, 128, 1.f, f, 1, nullptr, f, bytes, nullptr);
        printf("%d %d %d %d\n", rc, got.shape, got.n_split, got.row_sets);
    }
    return 0;
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    d = tmp_path_factory.mktemp("tree_plan")
    src, exe = d / "driver.cpp", d / "driver"
    src.write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-O1", f"-I{ROOT}/include", f"-I{CSRC}", str(src), os.path.join(CSRC, "api.cpp"),
                    os.path.join(CSRC, "draft.cpp"), os.path.join(ROOT, "tests", "sanitize", "launch_stub.cpp"), "-o", str(exe)], check=True)
    names = sorted(FORMS)
    lines = "".join(" ".join(map(str, FORMS[n][0])) + "\n" for n in names)
    out = subprocess.run([str(exe)], input=lines, text=True, capture_output=True, check=True).stdout.splitlines()
    return {n: tuple(map(int, x.split())) for n, x in zip(names, out, strict=True)}


@pytest.mark.parametrize("name", sorted(FORMS))
def test_plan(plans, name):
    assert plans[name] == (0, *FORMS[name][1])


def test_every_instance_is_there():
    """Both joins (up to eight splits and more) behind each shape, and no join."""
    assert {(shape, (splits > 1) + (splits > 8)) for _, (shape, splits, _) in FORMS.values()} == {(s, j) for s in (FEW, WIDE, PAIR)
                                                                                                 for j in range(3)}
