"""The low-bit kernels' rules on sizes under AddressSanitizer and
UndefinedBehaviorSanitizer (no GPU): tests/host_harness/lowbit_rules_harness.cpp,
built with g++ together with lowbit_plan.cpp and abi_lowbit.cpp."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_20940_amd", "csrc")


@pytest.fixture(scope="module")
def harness(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"):
        pytest.skip("g++ and the HIP headers are needed to build the host harness")
    exe = str(tmp_path_factory.mktemp("harness") / "lowbit_rules_harness")
    cmd = [gxx, "-std=c++17", "-g", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined",
           "-fno-omit-frame-pointer", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
           os.path.join(ROOT, "tests", "host_harness", "lowbit_rules_harness.cpp"),
           "-I" + os.path.join(ROOT, "include"), os.path.join(CSRC, "lowbit_plan.cpp"),
           os.path.join(CSRC, "abi_lowbit.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    return exe


def _run(exe, *args):
    return subprocess.run([exe, *map(str, args)], capture_output=True, text=True, timeout=300)


def test_rules_hold_under_sanitizers(harness):
    r = _run(harness)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
    assert " 0 failures" in r.stdout
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr


def test_wide_attention_cases_reach_the_kernel_of_eight_waves(harness):
    """Every GPU case that is to check that kernel gets it, some with a block an item, some with workers that share
    items and take more than one."""
    from test_gpu_mx_attention_wide import CASES

    whole = crossing = 0
    for case in CASES:
        r = _run(harness, "attention", *case)
        assert r.returncode == 0
        waves, items, workers = map(int, r.stdout.split())
        assert waves == 8, case
        whole += workers == 0
        # shares of the tiles, the first ones a tile larger: does a worker take tiles of two items?
        of_item = -(-case[5] // 64)
        each, more = divmod(items * case[0] * of_item, max(1, workers))
        first = [w * each + min(w, more) for w in range(workers + 1)]
        crossing += any(a // of_item != (b - 1) // of_item for a, b in zip(first, first[1:]))
    assert whole >= 10 and crossing >= 10
