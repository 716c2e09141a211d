"""The fitting entry points' host code (argument checks, the split of the rows over
workgroups, workspace layouts, AdamW's tables) built with g++ under AddressSanitizer and
UndefinedBehaviorSanitizer and run on the CPU, the launches replaced by host stand-ins
that write what the kernels write (tests/host/fake_fit.cpp): each row and element once,
inside its buffer, and no region of the workspace over another."""
from __future__ import annotations

import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2606_28565_amd.abi import NFAM
from tests.test_host_asan import CSRC, HOST, KS_EINVAL, KS_OK, ROCM_INCLUDE, ROOT, SAN_ENV


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.isdir(ROCM_INCLUDE):
        pytest.skip("g++ or the HIP runtime headers are not available")
    exe = str(tmp_path_factory.mktemp("host") / "ks_fit_driver")
    src = [os.path.join(CSRC, f) for f in ("ks_api.cpp", "ks_sim.cpp", "ks_fit.cpp")]
    src += [os.path.join(HOST, f) for f in ("fake_device.cpp", "fake_fit.cpp", "fit_driver.cpp")]
    cmd = [gxx, "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer",
           "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-ffp-contract=off",
           "-D__HIP_PLATFORM_AMD__", "-I", ROCM_INCLUDE, "-I", os.path.join(ROOT, "include"), "-I", CSRC, *src, "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    return exe


def run(exe, lines):
    r = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, env=dict(os.environ, **SAN_ENV),
                       timeout=300)
    assert r.returncode == 0, (r.returncode, r.stderr[-4000:])
    assert "ERROR: AddressSanitizer" not in r.stderr and "runtime error" not in r.stderr, r.stderr[-4000:]
    return r.stdout.splitlines()


def offsets(n, kind, rng):
    if kind == "one":
        cut = [0] * 4 + [n] * 5
    elif kind == "last":
        cut = [0] * 9
    else:
        cut = np.sort(rng.integers(0, n + 1, NFAM - 1)).tolist()
    return " ".join(str(int(v)) for v in cut)


@pytest.mark.parametrize("bf16", [0, 1])
@pytest.mark.parametrize("inp,hid", [(16, 1), (16, 64), (32, 67), (32, 128), (32, 129), (16, 200), (32, 256)])
def test_rows(driver, bf16, inp, hid):
    """One row to several steps of every workgroup; on both sides of the loss's switch to
    two launches."""
    rng = np.random.default_rng(hid)
    lines = [f"rows {n} {inp} {hid} {bf16} {pad} {offsets(n, kind, rng)}"
             for n, pad in ((0, 0), (1, 3), (9, 0), (128, 5), (129, 0), (4099, 8), (33_000, 0), (36_000, 1), (300_011, 0))
             for kind in ("any", "one", "last")]
    assert run(driver, lines) == ["ok"] * len(lines)


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw(driver, bits):
    """One tensor, one launch's, more; empty ones among them, off alignment too."""
    lines = []
    for g16, shift in ((0, 0), (1, 0), (1, 1)):
        for sizes in ([1], [63, 64, 65, 1024, 1025], [0, 0], [7 * i % 150 for i in range(199)],
                      [7 * i % 150 for i in range(200)], [1 + i % 3 for i in range(200)], [5] * 201, [i % 40 for i in range(650)],
                      [300_007, 0, 3]):
            lines.append(f"adam {bits} {g16} {shift} " + " ".join(map(str, sizes)))
    assert run(driver, lines) == ["ok"] * len(lines)


def test_features(driver):
    lines = [f"features {n} {s} {inp} {bf16} {pad}" for n, s in ((0, 3), (1, 1), (37, 5), (2000, 3))
             for inp in (16, 32) for bf16 in (0, 1) for pad in (0, 3)]
    assert run(driver, lines) == ["ok"] * len(lines)


EXPECTED = {
    "columns_apart": KS_OK, "columns_apart_before": KS_OK, "columns_far_apart": KS_OK, "columns_of_other_rows": KS_OK,
    "columns_meet": KS_EINVAL, "columns_meet_before": KS_EINVAL, "columns_run_into_the_next_row": KS_EINVAL,
    "columns_of_other_strides": KS_EINVAL, "same_rows": KS_EINVAL, "one_row_apart": KS_OK, "one_row_meets": KS_EINVAL,
    "behind_the_last": KS_OK,
}


def statuses(driver):
    return dict(line.split() for line in run(driver, ["args"]))


def test_rows_and_gradients_in_one_buffer(driver):
    """Rows and their gradients may be columns of one buffer of the same row stride; where
    an element belongs to both, or the strides differ, the call is refused."""
    got = statuses(driver)
    assert {k: int(got[k]) for k in EXPECTED} == EXPECTED


def test_workspace_of_an_unknown_precision(driver):
    got = statuses(driver)
    assert (got["workspace"], got["workspace_of_unknown_precision"]) == ("1", "0")
