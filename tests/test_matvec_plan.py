"""The host arithmetic of esb_matvec_groups (csrc/esb_matvec_plan.h), compiled
by itself: a row of the matrix is not read past its end, and the rings of the
tcgen05 kernel tell their uses apart."""
import ctypes
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SHIM = r"""
#include "esb_matvec_plan.h"
extern "C" int plan_tc(int64_t M, int64_t N, int64_t K, int planes, int r, int sms, int64_t* out)
{
    esb::MvTcPlan p;
    if (!esb::plan_matvec_tc(M, N, K, planes, r, sms, p)) return 0;
    const int64_t v[] = {p.nc, p.kc, p.mt, p.passes, p.stages, p.na, p.nd, (int64_t)p.smem, p.slot_first};
    for (int i = 0; i < 9; i++) out[i] = v[i];
    return 1;
}
extern "C" int64_t row_codes(int64_t K) { return esb::mv_row_codes(K); }
extern "C" int slice() { return esb::kSlice; }
extern "C" int end_words(int k, int t, int c, int codes) { return esb::mv_end_words(k, t, c, codes); }
"""


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("plan")
    src, so = d / "plan.cpp", d / "plan.so"
    src.write_text(SHIM)
    subprocess.run([cxx, "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2109_03513_gb300", "csrc"), str(src),
                    "-o", str(so)], check=True)
    lib = ctypes.CDLL(str(so))
    lib.plan_tc.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int] * 3 + [ctypes.c_void_p]
    lib.row_codes.argtypes, lib.row_codes.restype = [ctypes.c_int64], ctypes.c_int64
    return lib


def plan(shim, M, N, K, planes, r, sms=152):
    out = (ctypes.c_int64 * 9)()
    if not shim.plan_tc(M, N, K, planes, r, sms, out):
        return None
    return dict(zip(("nc", "kc", "mt", "passes", "stages", "na", "nd", "smem", "slot_first"), out))


def decoder_is_behind(stages, na, slot_first, c):
    """Whether the warps that decode step c (of two in a stage; they take every
    fourth) know, before they wait for its stage, that the use before this one
    of the stage's slot has landed: a wait for a parity is met by the phase two
    before.  Copies land in any order.  What these warps know: the stages of
    their own earlier steps, and, since the slot of A of step c - 4 was free,
    that the products of step c - 4 - na and of those before it are done, whose
    codes had landed; those of step c - na where they have waited for the slot
    of step c."""
    before = c // 2 - stages
    if before < 0:
        return True
    own = before in {s // 2 for s in range(c % 4, c, 4)}
    return own or 2 * before + 1 <= c - na - (0 if slot_first else 4)


def test_rings_of_stages_tell_their_uses_apart(shim):
    seen = set()
    for r in (1, 2, 4):
        for planes in (1, 2):
            for M in (1, 2, 5, 9, 11, 16, 17, 21, 24, 32, 33, 64, 500):
                for K in list(range(1, 6000, 127)) + [512, 1024, 1536, 1537, 2048, 2049, 4096, 4097, 4608, 4609, 5120, 5121, 16384, 20000]:
                    p = plan(shim, M, 65536, K, planes, r)
                    if p is None:
                        continue
                    assert K <= 5120
                    seen.add((p["stages"], p["na"], bool(p["slot_first"])))
                    assert p["kc"] >= K and p["kc"] % 512 == 0 and p["mt"] * planes <= p["nc"] and p["mt"] * p["passes"] >= M
                    assert p["smem"] <= 225 * 1024 and p["na"] * 64 + p["nd"] * r * p["nc"] <= 512
                    assert 4 <= p["na"] and 2 <= p["nd"]
    assert len(seen) > 4
    for stages, na, slot_first in sorted(seen):
        for c in range(64):
            assert decoder_is_behind(stages, na, slot_first, c), (stages, na, slot_first, c)
            assert c - 2 * na <= c - 4 - na      # the slot of A's own uses, by the products before step c - 4's


def test_rows_are_not_read_past_their_end(shim):
    size = shim.slice()
    for K in [*range(1, 1100), 4095, 4096, 4097, (1 << 18) - 1]:
        words = -(-K // 8)
        codes = shim.row_codes(K)
        # whole 16 bytes, no more than the smallest stride of such rows; the tcgen05 kernel's copies end there
        assert codes % 32 == 0 and codes // 8 == -(-words // 4) * 4
        # the warp-level kernel: every slice of a row but the last lies within it, and in the last one every lane's words
        k = (K - 1) // size * size
        for t in range(4):
            for c in range(4):
                at = k // 8 + 4 * t + (16 * c if k + size <= codes else shim.end_words(k, t, c, codes))
                assert 0 <= at and at + 4 <= codes // 8, (K, t, c)
                if 128 * c + 32 * t + k < K:             # codes of the row: in their place
                    assert at == k // 8 + 16 * c + 4 * t
