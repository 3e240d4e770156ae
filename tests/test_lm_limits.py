"""Limits of the entry points of include/hmoe_lm.h (no GPU needed), and of what one launch holds."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_1704_06363_amd import hmoe
from tests.test_lm_abi import F, ROOT, lib, refused  # noqa: F401 (lib: the fixture)


@pytest.mark.parametrize("scale", [1.8e38, 2.4e38, 3.4e38])
def test_scales_whose_product_with_log2_e_may_overflow(lib, scale):  # noqa: F811
    refused(lib.hmoe_token_logprob(16, 64, None, 1, 10, 64, F(scale), 16, 3, 16, 16, 16, 16, 16, 16, None, 0, None), -1,
            "scale")
    refused(lib.hmoe_token_logprob_backward(16, 64, None, 1, 10, 64, F(scale), 16, 16, 16, 16, 16, 32, 64, None), -1,
            "scale")


@pytest.fixture(scope="module")
def slices(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("slices") / "slices_driver")
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", os.path.join(ROOT, "paper_1704_06363_amd", "csrc"),
                    os.path.join(ROOT, "tests", "slices_driver.cpp"), "-o", exe], check=True)
    return exe


@pytest.mark.parametrize("units,blocks,threads", [
    (0, 1, 256), (1, 1, 256), (512, 32768, 256),       # the second layer at 512 groups of 2^19 columns
    (512, 65536, 256), (1, 65536, 256), (511, 65535, 256),
    ((1 << 24) + 3, 1, 256),                           # narrow products of 2^28 rows of three adapters
    ((1 << 24) - 1, 1, 256), (1 << 24, 1, 256), ((1 << 24) + 4096, 1, 256),
    ((1 << 31) - 1, 1, 256), ((1 << 31) - 1, 64, 256), (9, 1 << 19, 256), (70, 1, 512)])
def test_slices_hold_fewer_than_2_to_32_threads(slices, units, blocks, threads):
    out = subprocess.run([slices], input=f"{units} {blocks} {threads}\n", capture_output=True, text=True,
                         check=True).stdout.split()
    parts, (rc, calls, third) = [tuple(map(int, p.split(":"))) for p in out[:-3]], map(int, out[-3:])
    assert rc == 0
    at = 0
    for first, count in parts:  # every unit once, in order
        assert first == at and count > 0 and count * blocks * threads < 1 << 32
        at += count
    assert at == units
    assert (calls, third) == ((3, -7) if len(parts) >= 3 else (len(parts), 0))


def test_workspaces_that_are_not_aligned(lib):  # noqa: F811
    big = 1 << 40
    refused(lib.hmoe_token_logprob(16, 100000, None, 1, 1, 100000, F(1.0), 16, 3, 16, 16, 16, 16, 16, 16, 24, big, None),
            -3, "workspace")
    few = hmoe.FewParams(8, 64, 128, 64, 2, 1, 0, 16, None, 16, None, 16, None)
    refused(lib.hmoe_moe_few(ctypes.byref(few), 4, 16, 16, 16, 16, 20, big, None), -3, "workspace")
    p = hmoe.Lora(8, 64, 128, 16, 1, 16, None, 16, 16, None)
    refused(lib.hmoe_lora_few(ctypes.byref(p), 4, 16, 16, 16, 17, big, None), -3, "workspace")
    refused(lib.hmoe_lora_forward(ctypes.byref(p), 400, 16, 16, None, 16, 16, 8, big, None), -3, "workspace")
    refused(lib.hmoe_lora_backward(ctypes.byref(p), 400, 16, 16, None, 16, 16, 16, 16, 16, 8, big, None), -3, "workspace")
