"""The learned columns' host code (argument checks, the split of the work over workgroups,
workspace layouts) built with g++ under AddressSanitizer and UndefinedBehaviorSanitizer and
run on the CPU, the launches replaced by host stand-ins that read and write what the kernels do
(tests/host/fake_columns.cpp): each element once, inside its buffer, and no region of
the workspace over another."""
from __future__ import annotations

import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2606_28565_amd.abi import NFAM
from tests.test_fit_asan import offsets, run
from tests.test_host_asan import CSRC, HOST, ROCM_INCLUDE, ROOT


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.isdir(ROCM_INCLUDE):
        pytest.skip("g++ or the HIP runtime headers are not available")
    exe = str(tmp_path_factory.mktemp("host") / "ks_columns_driver")
    src = [os.path.join(CSRC, f) for f in ("ks_api.cpp", "ks_sim.cpp", "ks_fit.cpp", "ks_columns.cpp")]
    src += [os.path.join(HOST, f) for f in ("fake_device.cpp", "fake_fit.cpp", "fake_columns.cpp", "columns_driver.cpp")]
    cmd = [gxx, "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer",
           "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-ffp-contract=off",
           "-D__HIP_PLATFORM_AMD__", "-I", ROCM_INCLUDE, "-I", os.path.join(ROOT, "include"), "-I", CSRC, *src, "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    return exe


@pytest.mark.parametrize("bf16", [0, 1])
@pytest.mark.parametrize("cols", [1, 7, 8, 16, 67, 2049, 4100])
def test_columns(driver, bf16, cols):
    """One row to many parts of the order, one digit to three."""
    lines = [f"columns {n} {v} {cols} {pad} {bf16}" for n, v, pad in
             ((0, 3, 0), (1, 1, 2), (5, 300, 0), (128, 9, 5), (129, 1023, 0), (700, 1024, 1))]
    if cols <= 67:
        lines += [f"columns {n} {v} {cols} 3 {bf16}" for n, v in ((8193, 70), (40_001, 5), (3000, 70_000), (70_000, 1 << 20))]
    if cols == 1:
        lines += [f"columns 1300000 40 1 0 {bf16}"]
    assert run(driver, lines) == ["ok"] * len(lines)


def test_loss(driver):
    rng = np.random.default_rng(1)
    lines = [f"loss {n} {n % 2} {offsets(n, kind, rng)}" for n in (0, 1, 9, 4099, 8192, 8193, 90_001, 1_100_000)
             for kind in ("any", "one", "last")]
    assert run(driver, lines) == ["ok"] * len(lines)
    assert NFAM == 10
