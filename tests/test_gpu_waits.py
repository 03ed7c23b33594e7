"""Waits between blocks that run out: the kernels return, and no finite state comes out of maps
that did not arrive. The sources' own device functions run in small kernels (wait_probe.cu)."""
import ctypes
import os
import subprocess
import time

import pytest
import torch

from paper_2412_06355_gb300 import build as lib_build

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    so = str(tmp_path_factory.mktemp("probe") / "wait_probe.so")
    subprocess.run([lib_build.nvcc(), *lib_build.ARCH, *lib_build.NVCC_FLAGS, "-shared", "-o", so,
                    os.path.join(HERE, "wait_probe.cu")], check=True)
    lib = ctypes.CDLL(so)
    lib.run_lost_maps.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int]
    lib.run_no_arrival.argtypes = [ctypes.c_void_p]
    lib.run_landing.argtypes = [ctypes.c_void_p]
    return lib


def run(probe, passes, silent):
    out = torch.zeros(2, passes, 16, 16, 2, device="cuda")
    began = time.time()
    assert probe.run_lost_maps(out.data_ptr(), passes, silent) == 0
    return out, time.time() - began


def test_scan_blocks_that_all_send(probe):
    """The probe itself: 16 segments of two blocks that double the state, pass after pass."""
    out, _ = run(probe, 3, -1)
    for rank in range(2):
        for p in range(3):
            want = [2.0 ** (32 * p + 16 * rank + seg) for seg in range(16)]
            if p == 2:                                     # both blocks start at their segment 12
                if rank:                                   # 5 doubled to the end of block 0
                    want = [5 * 2.0 ** (3 + seg) for seg in range(16)]
                want[13:] = [5.0, 10.0, 20.0]
            want = torch.tensor(want, dtype=torch.float64).view(16, 1, 1).expand(16, 16, 2)
            assert torch.equal(out[rank, p].double().cpu(), want), (rank, p)


@pytest.mark.parametrize("silent", [0, 1])
def test_scan_maps_that_do_not_come(probe, silent):
    """One wait of about a second, not one for each pass; NaN for every state that depends on the
    other block, also where its buffer holds a stale start; what a start of the block's own
    begins anew is as it should be."""
    out, seconds = run(probe, 6, silent)
    assert 0.5 < seconds < 5.0
    got = out[1 - silent]
    assert torch.isnan(got[:5]).all() and torch.isnan(got[5, :13]).all()
    assert torch.equal(got[5, 13:, 0, 0].cpu(), torch.tensor([5.0, 10.0, 20.0]))


def test_a_barrier_without_arrivals(probe):
    out = torch.zeros(1, dtype=torch.int32, device="cuda")
    began = time.time()
    assert probe.run_no_arrival(out.data_ptr()) == 0
    assert int(out) == 2 and 2.0 < time.time() - began < 10.0


def test_memory_is_given_back_late_after_a_wait_that_ran_out(probe):
    out = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert probe.run_landing(out.data_ptr()) == 0
    assert 10000 <= int(out) < 1000000
