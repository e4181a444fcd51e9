"""The host arithmetic of esb_cache_attention (csrc/esb_attention_plan.h),
compiled by itself: whatever the lengths, no place outside of a page table is
looked up, and every place that a query sees is gone through."""
import ctypes
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SHIM = r"""
#include "esb_attention_plan.h"
extern "C" void tile(int64_t p0, int64_t p1, int seen, int window, int stage, int block, int* out)
{
    const esb::Tile t = esb::tile_places(p0, p1, seen, window, stage, block);
    out[0] = t.lo; out[1] = t.hi; out[2] = t.blocks;
}
extern "C" int first(int lo, int hi, int first, int warp, int warps, int stage) { return esb::first_place({lo, hi, 0}, first, warp, warps, stage); }
extern "C" int run(int seqs, int threads) { return esb::run_of(seqs, threads); }
extern "C" int end(int lo, int hi, int first, int blocks, int block) { return esb::end_place({lo, hi, 0}, first, blocks, block); }
"""
MOST = (1 << 31) - 1


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("plan")
    src, so = d / "plan.cpp", d / "plan.so"
    src.write_text(SHIM)
    subprocess.run([cxx, "-std=c++17", "-O1", "-fwrapv", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2109_03513_gb300", "csrc"), str(src),
                    "-o", str(so)], check=True)
    lib = ctypes.CDLL(str(so))
    lib.tile.argtypes = [ctypes.c_int64] * 2 + [ctypes.c_int] * 4 + [ctypes.c_void_p]
    return lib


@pytest.mark.parametrize("stage", [16, 32])
@pytest.mark.parametrize("held", [0, 16, 160, 4096, (1 << 30) - 16, 1 << 30])
def test_places_of_a_tile(shim, stage, held):
    warps, block = 4, 4 * stage
    for length in [0, 1, 2, 15, 16, 17, 100, 159, 160, 161, 5000, (1 << 30) - 1, 1 << 30, (1 << 30) + 100, MOST - 200, MOST - 64, MOST - 33, MOST - 1, MOST]:
        for queries in (1, 2, 8, 200):
            for window in (0, 1, 2, 31, 40, 64, 1000, 1 << 30, MOST):
                seen = min(length, held)
                p0, p1 = length - queries, length - 1
                out = (ctypes.c_int * 3)()
                shim.tile(p0, p1, seen, window, stage, block, out)
                lo, hi, blocks = out
                want_lo = max(0, p0 - window + 1) if window else 0
                want_hi = max(0, min(p1 + 1, seen))
                # what some query sees lies between lo and hi, and little else does
                assert hi == want_hi and lo % stage == 0 and 0 <= lo <= hi
                assert lo <= want_lo and (want_lo - lo < stage or want_lo >= hi)
                assert blocks == max(1, -(-(hi - lo) // block)) and (want_lo < hi or blocks == 1)
                for cut in {0, blocks // 2, blocks - 1}:
                    n = blocks - cut
                    end = shim.end(lo, hi, cut, n, block)
                    assert end == min(hi, lo + blocks * block)
                    for warp in range(warps):
                        place = shim.first(lo, hi, cut, warp, warps, stage)
                        assert place == lo + cut * block + warp * stage      # no wrap
                        stages = -(-(end - place) // block) if end > place else 0
                        if stages:                                           # all of its stages begin in the table
                            assert 0 <= place and place + (stages - 1) * block < min(held, end)


def test_runs_hold_every_sequence(shim):
    for seqs in (1, 2, 127, 128, 129, 1 << 20, MOST - 128, MOST - 127, MOST - 126, MOST):
        run = shim.run(seqs, 128)
        assert 128 * run >= seqs > 128 * (run - 1)
