"""The stages of shared memory that the delta rule's walks fetch chunks into, as a protocol on the CPU: the library's own
choice of barrier and phase (delta_plan.h), in every order in which fetches and products can follow each other."""
import ctypes
import subprocess

import pytest

from paper_2412_06355_gb300 import build

SOURCE = """
#include "seq/delta_plan.h"
extern "C" int at(int n, int stages) { return dendsn::stage_at(n, stages); }
extern "C" unsigned phase(int n, int stages) { return dendsn::free_phase(n, stages); }
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("stages")
    (d / "stages.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", f"-I{build.CSRC}", str(d / "stages.cpp"), "-o",
                    str(d / "stages.so")], check=True)
    lib = ctypes.CDLL(str(d / "stages.so"))
    lib.phase.restype = ctypes.c_uint
    return lib


def walk(chunks, stages, barrier, phase):
    """All states (chunks fetched, chunks done) that can be reached. A chunk's last product completes a phase of the
    barrier that `barrier` names; the fetch of chunk n >= stages goes on when a look at its barrier finds the parity of
    `phase` complete: the barrier is in a phase of the other parity. A look may come at any time, or late.
    Returns what went wrong, or None."""
    seen, todo = {(0, 0)}, [(0, 0)]
    while todo:
        fetched, done = todo.pop()
        nexts = []
        if done < fetched:
            nexts.append((fetched, done + 1))
        if fetched < chunks:
            ready = fetched < stages
            if not ready:
                complete = sum(barrier(c) == barrier(fetched) for c in range(done))
                ready = complete % 2 != phase(fetched) % 2
            if ready:
                if fetched >= stages and done <= fetched - stages:
                    return "overwritten", fetched, done
                nexts.append((fetched + 1, done))
        if not nexts and (fetched, done) != (chunks, chunks):
            return "stuck", fetched, done
        for s in nexts:
            if s not in seen:
                seen.add(s)
                todo.append(s)
    return None


@pytest.mark.parametrize("stages", [1, 2])
@pytest.mark.parametrize("chunks", [1, 2, 3, 4, 5, 9, 32])
def test_a_fetch_is_neither_lapped_nor_early(plan, stages, chunks):
    assert walk(chunks, stages, lambda n: plan.at(n, stages), lambda n: plan.phase(n, stages)) is None


def test_the_model_finds_a_lapped_wait():
    """One barrier for both stages: the chunk in the other stage completes it a second time."""
    assert walk(3, 1, lambda n: 0, lambda n: n - 1) is None
    assert walk(3, 2, lambda n: 0, lambda n: n - 2) == ("stuck", 2, 2)
    assert walk(5, 2, lambda n: n % 2, lambda n: n // 2) is not None
