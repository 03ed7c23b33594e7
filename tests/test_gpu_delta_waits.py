"""Waits of the gated delta rule's gradients: a warp goes on with one answer, whatever its lanes saw."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2412_06355_gb300 import build as lib_build

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    so = str(tmp_path_factory.mktemp("probe") / "delta_probe.so")
    subprocess.run([lib_build.nvcc(), *lib_build.ARCH, *lib_build.NVCC_FLAGS, "-shared", "-o", so,
                    os.path.join(HERE, "delta_probe.cu")], check=True)
    lib = ctypes.CDLL(so)
    lib.run_split_warp.argtypes = [ctypes.c_void_p, ctypes.c_int]
    return lib


@pytest.mark.parametrize("which,goes_on", [(0, True), (1, False), (2, False)])
def test_a_warp_goes_on_together(probe, which, goes_on):
    """All lanes get one answer, so the election of an issuing lane, which names all 32, is never met by some of
    them alone: one lane issues, or none."""
    out = torch.zeros(33, dtype=torch.int32, device="cuda")
    assert probe.run_split_warp(out.data_ptr(), which) == 0
    assert out.tolist() == [int(goes_on)] * 33
