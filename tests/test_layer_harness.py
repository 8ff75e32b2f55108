"""The host code of the loss, the norms around a block and the kept activations over a stand-in for the HIP runtime (CPU), under
AddressSanitizer and UndefinedBehaviorSanitizer: layer_harness.hip compiles their sources for the host alone and runs one scenario per
test."""

import glob
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2503_19050_amd", "csrc")

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None or not glob.glob("/opt/rocm/llvm/lib/clang/*/lib/linux/libclang_rt.asan*"),
                                reason="needs hipcc and its sanitizers' runtime")


@pytest.fixture(scope="module")
def harness(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("harness")
    obj, exe = str(tmp / "layer_harness.o"), str(tmp / "layer_harness")
    sanitizers = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all"]
    subprocess.run(["hipcc", "--cuda-host-only", "--offload-arch=gfx950", "-std=c++17", "-O1", "-g", "-ffp-contract=off", "-w", *sanitizers,
                    "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", os.path.join(ROOT, "tests", "layer_harness.hip"), "-o", obj], check=True)
    # no HIP library: the object has the runtime it uses; there is no device code to register
    subprocess.run(["/opt/rocm/llvm/bin/clang++", obj, "-o", exe, *[f for f in sanitizers if f != "-Xarch_host"],
                    "-Wl,--unresolved-symbols=ignore-all"], check=True)
    return exe


@pytest.mark.parametrize("scenario", ["grids", "parts", "ranges"])
def test_scenario(harness, scenario):
    """What each one checks stands at its function in layer_harness.hip."""
    r = subprocess.run([harness, scenario], capture_output=True, text=True, timeout=300, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1"))
    assert r.returncode == 0, (r.returncode, (r.stdout + r.stderr)[-2000:])
