// esb_matvec_plan.h -- arithmetic of esb_matvec_groups that needs no CUDA:
// where a row of the matrix ends, which calls the tcgen05 kernel takes and the
// sizes of its rings.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

#ifdef __CUDACC__
#define ESB_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define ESB_HOST_DEVICE inline
#endif

namespace esb {

// Codes of a row of K that the kernels read: whole 16 bytes, which a row of ld
// words (a multiple of four) has.  Never by ld: a row may be the last of a
// matrix cut out of a wider one.
inline int64_t mv_row_codes(int64_t K) { return (K + 31) / 32 * 32; }

// The warp-level kernel's slice: four steps of 128 codes, 16 bytes of each for
// each of four lanes.
constexpr int kSteps = 4;
constexpr int kSlice = 128 * kSteps;
// Words from lane t's place in the slice that starts at code k to those of its
// step c that it reads, where the row of `codes` (mv_row_codes) ends within the
// slice: past the end its last words will do, x is 0 there.
ESB_HOST_DEVICE int mv_end_words(int k, int t, int c, int codes)
{
    const int last = codes / 8 - 4 - (k / 8 + t * 4);
    return c * 16 < last ? c * 16 : last;
}

constexpr int kTcStage = 256;                   // codes of a row in a stage: one TMA tile of 128 rows of 128 bytes, swizzled
constexpr int kTcStageBytes = 128 * kTcStage / 2;
constexpr int kTcStepsOfStage = kTcStage / 128;
constexpr int kTcMaxStages = 8, kTcMaxA = 5, kTcMaxD = 12;
constexpr size_t kTcSmem = 225 * 1024;

struct MvTcPlan {
    int nc, kc, mt;                             // columns of sums, codes of a row, rows of x in a pass
    int64_t passes;
    int stages, na, nd;                         // slots of the rings of code stages, of A and of sums
    bool slot_first;                            // decoding warps wait for their slot of A before their stage
    size_t smem;
};

inline size_t mv_tc_smem(int nc, int kc, int r, int stages)
{
    return 1024 + (size_t)(kc / 64) * nc * 128 + (size_t)stages * kTcStageBytes + (size_t)(kc / 128) * r * nc * 4 + 2 * nc * 128 * 4;
}

// The plan of a call: false where the warp-level kernel takes it.  planes: of
// each row of x; r: groups of a step of 128 codes.
inline bool plan_matvec_tc(int64_t M, int64_t N, int64_t K, int planes, int r, int sms, MvTcPlan& p)
{
    // Where the other kernel would take more than one pass of 32 columns, or
    // nearly fills one with rows alone (times in esb_matvec_tc.cu).
    const int64_t columns = M * planes * r;
    if (columns <= 32 && !(r == 1 && columns > 20)) return false;
    const int64_t tiles = (N + 127) / 128;
    const int64_t kc = (K + 511) / 512 * 512;   // steps in fours
    p.kc = (int)kc;
    // 32 columns where the rows need them and x then fits, else 16.  At least
    // four slots of A: the decoding warps of step c know from their last step,
    // c - 4, that what lay in its slot before is done, so all steps to c - 4 - na
    // are, and the use before the last of c's own slot, c - 2 na, must be among
    // them for a barrier's parity to tell its uses apart.
    // (groups of 32 have sums for two steps only with 32 columns: 16 then)
    p.nc = M * planes <= 16 || r == 4 ? 16 : 32;
    p.smem = 0;
    for (;; p.nc = 16) {
        for (p.stages = kTcMaxStages; p.stages >= 2; p.stages--) {
            p.smem = mv_tc_smem(p.nc, p.kc, r, p.stages);
            if (p.smem <= kTcSmem) break;
        }
        if (p.stages >= 2 || p.nc == 16) break;
    }
    if (p.stages < 2) return false;             // K above 5120: x leaves no room for two stages
    p.mt = (int)std::min<int64_t>(M, p.nc / planes);
    p.passes = (M + p.mt - 1) / p.mt;
    if (p.passes > 65535) return false;
    p.mt = (int)((M + p.passes - 1) / p.passes);
    p.na = p.nc == 16 ? 5 : 4;
    p.nd = std::min(kTcMaxD, (512 - p.na * 64) / (r * p.nc));
    // The ring of stages: copies land in any order, and a decoding warp takes
    // every second stage.  In an even ring it has waited for the last use of its
    // slot itself; with five or seven stages the products up to step c - 4 - na
    // tell it that this use had landed.  With three, steps c - 7 to c - 5, only
    // the products up to step c - na do, which the slot of A of step c itself
    // brings: its wait then comes first.  (Otherwise last, behind the loads of
    // the codes.  24 rows times 50000 x 4608: 115 us so, 138 with two stages.)
    p.slot_first = p.stages == 3;
    // Too few tiles for the SMs: the other kernel splits rows among warps.
    return tiles * p.passes * 5 >= (int64_t)sms * 4;
}

}  // namespace esb
