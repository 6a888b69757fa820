"""The barriers of the tensor-core kernel of treewy_attn_chunk: no wait can pass too early or be overtaken, and nothing is overwritten
that is still read, in whatever order its roles run.  Who hands an output over is the kernel's own rule (csrc/chunk_phases.cuh,
compiled for the host)."""
import ctypes
import os
import re
import subprocess

import pytest

from tests import chunk_roles_model as model
from tests.chunk_roles_model import pair, single

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = """
#include "chunk_phases.cuh"
extern "C" int arrivals() { return treewy::O_FREE_ARRIVALS; }
extern "C" int frees(int apart, int strm, int which, int used) { return treewy::frees_output(apart, strm, which, used); }
"""
# runs of items of one CTA: two row tiles, one, streams without a tile (the first item's end, the last one's start)
BATCHES = {
    "pair, short single": lambda d: [pair(range(2), range(3)), single(d, 2), single(d, 1)],
    "singles": lambda d: [single(d, 3), single(d, 2), single(d, 5)],
    "singles of one tile": lambda d: [single(d, 1)] * 4 + [single(d, 4)],
    "pairs of one tile": lambda d: [pair([0], [0])] * 3 + [single(d, 2)],
    "a stream without a tile": lambda d: [pair([], [0]), single(d, 1), single(d, 2), pair([0], [])],
    "a stream without a tile, again and again": lambda d: [pair([], [0]), pair([], [0]), single(d, 1), pair([0, 1], []), pair([0], [])],
    "a window's hole": lambda d: [pair([0, 1, 4], [0, 2, 3, 4]), single(d, 3), pair([0, 2], [1, 2])],
    "more tiles than stages": lambda d: [single(d, 11), pair(range(7), range(8)), single(d, 1)],
    "more items than the ring": lambda d: [single(d, 2), pair([0], [0, 1])] * 5,
}


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    path = tmp_path_factory.mktemp("phases")
    (path / "p.cpp").write_text(SRC)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2608_20961_b200", "csrc"), str(path / "p.cpp"),
                    "-o", str(path / "p.so")], check=True)
    lib = ctypes.CDLL(str(path / "p.so"))
    assert lib.arrivals() % 4 == 0                   # (of a stream's four warps; the model has fewer)
    return model.Rule(lambda apart, s, which, used: lib.frees(apart, s, which, used), model.WARPS * lib.arrivals() // 4)


def _kernel():
    return open(os.path.join(ROOT, "paper_2608_20961_b200", "csrc", "chunk_sm100_tc.cu")).read()


def test_the_kernel_is_what_the_model_has():
    text = _kernel()
    assert "frees_output(apart, strm, s, apart ? taken > 0 : s < n)" in text and "mbar_init(&sh.o_free[i], O_FREE_ARRIVALS)" in text
    assert len(re.findall(r"mbar_arrive\(&sh\.o_free", text)) == 1 and len(re.findall(r"wait\(&sh\.o_free", text)) == 1
    assert "NB = D == 256 ? 4 : 2;" in text and "NK = D == 64 ? 10 : D == 128 ? 5 : 3, NV = D == 64 ? 10 : D == 128 ? 5 : 2;" in text
    assert "ITEMS = 8;" in text


@pytest.mark.parametrize("name", list(BATCHES))
@pytest.mark.parametrize("d", [64, 128])
def test_no_order_goes_wrong(rule, d, name):
    assert model.find(d, BATCHES[name](d), rule) is None
    assert model.find(d, BATCHES[name](d), rule, masked=False, rescale=True) is None


@pytest.mark.parametrize("name", ["pair, short single", "singles", "a stream without a tile"])
def test_what_a_tile_met_is_known_when_it_is_looked_for(rule, name):
    """NaN and infinity that a stream has taken out of the values, and pages out of range: the stream that writes the outputs of both knows
    of the other's too."""
    text = _kernel()
    wait, look = text.index("wait_warp(&sh.ml_full[w4]"), text.index("sh.nonfinite[ord % 8] == ord + 1")
    flags = "late" if wait < look < text.index("const bool writes = ") else "early"
    assert text.count("sh.nonfinite[ord % 8] == ") == 1 and text.count("sh.bad_item[ord % 8] == ") == 1
    assert model.find(128, BATCHES[name](128), rule, flags=flags) is None
    assert "is looked for before it is known" in model.find(128, BATCHES[name](128), rule, flags="early")


@pytest.mark.parametrize("tiles", [[3, 1, 6], [1] * 4, [5, 2] * 5], ids=str)
@pytest.mark.parametrize("rescale", [False, True])
def test_no_order_goes_wrong_with_one_stream(rule, tiles, rescale):
    assert model.find(256, [single(256, n) for n in tiles], rule, rescale=rescale) is None
    assert model.find(256, [single(256, n) for n in tiles], rule, masked=False, rescale=rescale) is None


@pytest.mark.parametrize("items", [[single(128, 1)] * 4, [pair([0], [0, 1]), pair([], [0]), single(128, 2)]], ids=["one tile", "no tile"])
def test_the_model_sees_a_phase_for_an_item(items):
    """As it was: a phase to an item, whether an output is used in it or not.  A stream without a tile can complete two phases ahead of
    the thread that waits for the first, which then waits for good."""
    W = model.WARPS
    both = model.Rule(lambda apart, s, which, used: (2 if s == which else 0) if apart else 1, 2 * W, by_use=False, waits=(0, 1))
    found = model.find(128, items, both)
    assert found and "('o_free', 1) has been overtaken" in found, found


def test_the_model_sees_outputs_overwritten():
    """An output that the first stream has to read, said to be free when the second has come to its end."""
    own = model.Rule(lambda apart, s, which, used: int(used and s == which), model.WARPS)
    found = model.find(128, [single(128, 2), pair([0], [0])], own)
    assert found and "('o', 1) holds 1, not 0" in found, found
