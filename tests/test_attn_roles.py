"""The tensor-core attention kernel's barriers: no wait can pass too early or be overtaken, in whatever order its roles
run.  The phase arithmetic of the queries' barriers is the kernel's own (csrc/attn_phases.cuh, compiled for the host)."""
import ctypes
import os
import re
import subprocess

import pytest

from tests import attn_roles_model as model

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = """
#include "attn_phases.cuh"
extern "C" int q_buffers(int d) { return treewy::q_buffers(d); }
extern "C" unsigned q_barrier(unsigned i, int n) { return treewy::q_phase(i, n).barrier; }
extern "C" unsigned q_parity(unsigned i, int n) { return treewy::q_phase(i, n).parity; }
"""
# tiles of an item: one (a cut piece), two (up to 64 keys and the draft rows), more
BATCHES = [[1, 1, 1], [2, 2, 2], [2, 1, 2], [3, 2], [5, 1]]


@pytest.fixture(scope="module")
def phases(tmp_path_factory):
    path = tmp_path_factory.mktemp("phases")
    (path / "p.cpp").write_text(SRC)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2608_20961_b200", "csrc"), str(path / "p.cpp"),
                    "-o", str(path / "p.so")], check=True)
    return ctypes.CDLL(str(path / "p.so"))


def test_the_kernel_takes_its_phases_from_there():
    text = open(os.path.join(ROOT, "paper_2608_20961_b200", "csrc", "attn_sm100_tc.cu")).read()
    assert "q_buffers(D)" in text and len(re.findall(r"q_phase\(\w+, C::NQ\)", text)) == 2
    assert "NK = D == 256 ? 3 : 8, NV = D == 256 ? 2 : D == 128 ? 4 : 8;" in text and "NSB = D == 256 ? 2 : 4;" in text
    assert "ITEMS = 8;" in text


@pytest.mark.parametrize("rescale", [False, True])
@pytest.mark.parametrize("items", BATCHES, ids=str)
@pytest.mark.parametrize("d", [64, 128, 256])
def test_no_wait_is_misled(phases, d, items, rescale):
    phase = lambda i, n: (phases.q_barrier(i, n), phases.q_parity(i, n))
    n = phases.q_buffers(d)
    assert n == model.q_tm[d]
    assert model.walk(model.programs(d, items, phase, n, rescale)) is None


def test_the_model_sees_one_barrier_for_two_buffers():
    """Items of two tiles announced on one barrier: the second phase can overtake the first."""
    one = lambda i, n: (0, i & 1)
    found = model.walk(model.programs(128, [2, 2, 2], one, 1, False))
    assert found and "('q', 0) has been overtaken" in found
