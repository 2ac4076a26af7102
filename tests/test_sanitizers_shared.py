"""AddressSanitizer / UndefinedBehaviorSanitizer run of the ABI layer of shared pages and shared prefixes (CPU only, with
stubs of the kernel launchers): random and extreme arguments of every entry point; buffers that hold what a launch is
given, and that grow with the batch."""
import os

from test_sanitizers import HERE, ROOT, SAN, build_and_run, pytestmark  # noqa: F401


def test_shared_abi_layer_under_sanitizers(tmp_path):
    csrc = os.path.join(ROOT, "paper_2606_01483_amd", "csrc")
    out = build_and_run(tmp_path, "shared_driver", [
        "g++", "-std=c++17", *SAN, f"-I{ROOT}/include", f"-I{csrc}", os.path.join(csrc, "api.cpp"),
        os.path.join(csrc, "shared.cpp"), os.path.join(HERE, "launch_stub.cpp"), os.path.join(HERE, "shared_driver.cpp")])
    assert "shared driver: ok" in out
