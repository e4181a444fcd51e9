// esb_matvec_tc.cu -- esb_matvec_groups for many columns (rows of x, times
// their planes, times the groups of a step): the same decoding, with the
// products on tcgen05.
//
// The warp-level matrix instruction of esb_matvec.cu holds its warp's issue
// for about 11 cycles, and once for every 8 columns.  Here the decoded codes
// go to tensor memory (a thread owns a row: it reads 16 bytes of it at a time
// from shared memory, where TMA puts tiles of 128 rows by 256 codes, and
// stores fp16 pairs to its lane), one thread issues tcgen05.mma kind::f16 (A
// in tensor memory, B the rows of x in shared memory, 128 x NC x 16), and
// eight warps scale each step's sums by the group's and the column's scales
// into fp32 registers.  Instructions bound it, about 29 a word of which 13
// decode: 65536 x 4096 with 32 rows of bf16 takes 103 us in groups of 128
// (133 by the other kernel) and 216 in groups of 32 (302), with 16 rows 65
// and 132 (63 and 159), with 4 rows 55 and 108 (45 and 61).  It takes calls of
// more columns than the other kernel's one pass (esb_matvec_plan.h), where x
// leaves shared memory for two code stages (K to 5120) and the matrix has tiles
// for four SMs of five.
//
// Roles of a block (one on an SM, tiles of 128 matrix rows in turn): warps
// 0..15 decode, steps of 128 codes c to the four warps c % 4; 16..23 scale,
// two teams of four that take the steps in turn (the second hands its sums to
// the first, which stores); 24 copies; 25 issues.  Steps go through two rings
// of tensor memory: 64 columns of A, and NC columns of sums for each group.
#include <algorithm>
#include <cstdint>
#include <mutex>

#include <cuda.h>
#include <cuda_runtime.h>

#include "esb_internal.h"
#include "esb_matvec.cuh"
#include "esb_matvec_plan.h"
#include "esb_tc.cuh"

namespace esb {

namespace {

constexpr int kTcDecode = 16, kTcScale = 8, kTcCopy = kTcDecode + kTcScale, kTcIssue = kTcCopy + 1, kTcWarps = kTcIssue + 1;
constexpr int kTcThreads = kTcWarps * 32;

// Where stage_x puts x: K-major rows of 128 bytes (64 values) in 8-row atoms
// with the 128-byte swizzle, and the columns' scales of every step and group.
template <int NC>
struct TcPlace {
    unsigned char* xs;
    float* fx;
    int r_of_step;
    __device__ __forceinline__ uint4* values(int row, int b) const
    {
        return reinterpret_cast<uint4*>(xs + (size_t)(b >> 3) * (NC * 128) + (row >> 3) * 1024 + (row & 7) * 128 + (((b & 7) ^ (row & 7)) << 4));
    }
    __device__ __forceinline__ float* scale(int row, int step, int r) const { return fx + (step * r_of_step + r) * NC + row; }
};

struct TcArgs {
    MvArgs a;
    int r;                                      // groups of a step: 1, 2 or 4
    int stages, na, nd;                         // slots of the three rings
    int slot_first;                             // the decoding warps' order of waits
    int* status;
};

__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
          "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
          "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
          "r"(r[30]), "r"(r[31])
        : "memory");
}

// D[tmem] (+)= A[tmem] B[smem]^T, kind::f16 (both operands fp16); issued as
// mma_f8f6f4 is.
__device__ __forceinline__ void mma_f16_ts(uint32_t d, uint32_t a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate, uint32_t leader)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d), "r"(a), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(leader)
        : "memory");
}

// A place in a ring: index and the parity of its use.
struct Ring {
    int at = 0;
    uint32_t parity = 0u;
    __device__ __forceinline__ void go(int by, int size)
    {
        at += by;
        while (at >= size) {
            at -= size;
            parity ^= 1u;
        }
    }
};

template <int NC>
__global__ void __launch_bounds__(kTcThreads, 1) matvec_tc_kernel(const __grid_constant__ CUtensorMap codes, const TcArgs ta)
{
    extern __shared__ unsigned char tc_raw[];
    __shared__ uint64_t full[kTcMaxStages], empty[kTcMaxStages], afull[kTcMaxA], afree[kTcMaxA], dfull[kTcMaxD], dfree[kTcMaxD], drain;
    __shared__ uint32_t tmem_slot;
    __shared__ int err_word;
    __shared__ uint16_t xtab[256];
    volatile int* err = &err_word;
    const MvArgs& a = ta.a;
    const int lane = threadIdx.x & 31, warp = warp_index();
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(tc_raw) + 1023) & ~(uintptr_t)1023);
    unsigned char* xs = smem;
    unsigned char* ring = xs + (size_t)(a.kc / 64) * NC * 128;
    float* fx = reinterpret_cast<float*>(ring + ta.stages * kTcStageBytes);
    float* hand = fx + (a.kc / 128) * ta.r * NC;        // the second team's sums, twice NC x 128
    if ((uint32_t)(reinterpret_cast<unsigned char*>(hand + 2 * NC * 128) - tc_raw) > dynamic_smem_bytes()) {
        if (threadIdx.x == 0) record_status(ta.status, ESB_ERR_INTERNAL);
        return;
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < ta.stages; i++) {
            mbar_init(&full[i], 1);                     // the copying thread's expectation, then the bytes
            mbar_init(&empty[i], 4 * kTcStepsOfStage);  // four warps read each of its steps
        }
        for (int i = 0; i < ta.na; i++) {
            mbar_init(&afull[i], 4);                    // the four warps of a step
            mbar_init(&afree[i], 1);                    // the MMAs' commit
        }
        for (int i = 0; i < ta.nd; i++) {
            mbar_init(&dfull[i], 1);                    // the MMAs' commit
            mbar_init(&dfree[i], 4);                    // the team that takes the step
        }
        mbar_init(&drain, 1);
        err_word = 0;
        fence_mbar_init();
    }
    if (warp == kTcIssue) {
        tmem_alloc(&tmem_slot, 512);
        tc_fence_before();
    }
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    griddep_wait();
    griddep_launch_dependents();

    const int64_t m0 = (int64_t)blockIdx.y * a.mt;
    const int mt = (int)min((int64_t)a.mt, a.M - m0), cols = mt * a.planes;
    const int N = (int)a.N, tiles = (N + 127) / 128;
    const int my_tiles = tiles > (int)blockIdx.x ? (tiles - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x : 0;
    const int stages_of_tile = a.kc / kTcStage, steps_of_tile = stages_of_tile * kTcStepsOfStage;
    const uint32_t sums = tmem + ta.na * 64;            // the ring of sums behind that of A

    if (warp == kTcCopy) {
        // ------------------------------------------------------- copies
        // One thread, one tile a stage.  Rows past N and words past the row's
        // last code read as zeros (which decode to numbers; x is 0 there).
        // 128 bulk copies of a row segment each went out too slowly (137 us
        // for 65536 x 4096), 16-byte asynchronous copies by four warps took 57.
        if (lane == 0) {
            Ring st;
            int issued = 0;
            for (int i = 0; i < my_tiles && !*err; i++) {
                const int row0 = ((int)blockIdx.x + i * (int)gridDim.x) * 128;
                for (int s = 0; s < stages_of_tile; s++) {
                    if (!wait_or_abort(&empty[st.at], st.parity ^ 1u, err)) { *err = 1; break; }
                    mbar_arrive_expect_tx(&full[st.at], kTcStageBytes);
                    asm volatile(
                        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                        ::"r"(smem_u32(ring + st.at * kTcStageBytes)), "l"(&codes), "r"(s * (kTcStage / 8)), "r"(row0),
                          "r"(smem_u32(&full[st.at])) : "memory");
                    st.go(1, ta.stages);
                    issued++;
                }
            }
            if (*err) {
                // given up: no copy may be under way when the block ends
                volatile int never = 0;
                const int n = min(issued, ta.stages);
                Ring q;
                q.go(issued - n, ta.stages);
                for (int i = 0; i < n; i++, q.go(1, ta.stages)) (void)wait_or_abort(&full[q.at], q.parity, &never);
            }
        }
    } else {
        // x, by all the other warps (the last of them takes the copying one's place)
        const int order = warp < kTcCopy ? warp : kTcCopy, others = kTcWarps - 1;
        const int tid = order * 32 + lane, nthreads = others * 32;
        // (rows of B that are no plane of x hold whatever is there: their
        // columns' sums are not read)
        if (a.x_type == ESB_CODES) {
            for (int i = tid; i < 256; i += nthreads) xtab[i] = x_code_half(i, a.xc.fmt.k);
            asm volatile("barrier.sync 1, %0;" ::"n"((kTcWarps - 1) * 32) : "memory");
        }
        const TcPlace<NC> place{xs, fx, ta.r};
        if (ta.r == 1) stage_x<1>(a, m0, mt, 0, place, xtab, others, order);
        else if (ta.r == 2) stage_x<2>(a, m0, mt, 0, place, xtab, others, order);
        else stage_x<4>(a, m0, mt, 0, place, xtab, others, order);
        fence_proxy_async_smem();                       // the MMAs read x by the async proxy
        asm volatile("barrier.sync 1, %0;" ::"n"((kTcWarps - 1) * 32) : "memory");

        if (warp < kTcDecode) {
            // --------------------------------------------------- decoding
            const int quarter = warp & 3, first = warp >> 2;
            const uint32_t my_row = smem_u32(ring) + (quarter * 32 + lane) * 128;
            const uint32_t my_lanes = tmem + ((uint32_t)(quarter * 32) << 16);
            Ring st, sl;
            st.go(first / kTcStepsOfStage, ta.stages);
            sl.go(first, ta.na);
            // 16 bytes j of a row of 128 lie at j xor (row mod 8)
            const uint32_t half = (uint32_t)(first % kTcStepsOfStage) * 4u, turn = (uint32_t)lane & 7u;
            bool ok = true;
            for (int q = 0; q < my_tiles * steps_of_tile / 4 && ok; q++) {
                ok = (!ta.slot_first || warp_wait(&afree[sl.at], sl.parity ^ 1u, err)) && warp_wait(&full[st.at], st.parity, err);
                if (!ok) break;
                const uint32_t at = my_row + st.at * kTcStageBytes;
                uint32_t w[16];
#pragma unroll
                for (int i = 0; i < 4; i++)
                    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                                 : "=r"(w[4 * i]), "=r"(w[4 * i + 1]), "=r"(w[4 * i + 2]), "=r"(w[4 * i + 3]) : "r"(at + (((half + i) ^ turn) << 4)) : "memory");
                ok = warp_wait(&afree[sl.at], sl.parity ^ 1u, err);
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    uint32_t d[32];
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        uint32_t p[4];
                        decode8(w[8 * h + i], a.tab, p);
#pragma unroll
                        for (int j = 0; j < 4; j++) d[4 * i + j] = p[j];
                    }
                    tmem_st32(my_lanes + sl.at * 64 + 32 * h, d);
                }
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&empty[st.at]);
                    mbar_arrive(&afull[sl.at]);
                }
                st.go(4 / kTcStepsOfStage, ta.stages);
                sl.go(4, ta.na);
            }
            if (!ok) *err = 1;
        } else if (warp == kTcIssue) {
            // --------------------------------------------------- MMAs
            const uint32_t idesc = idesc_e4m3_f32(NC);  // format fields 0: fp16 in kind::f16
            const uint32_t leader = elect_one();
            const uint64_t bdesc = smem_desc_sw128(smem_u32(xs));
            Ring as, ds;
            bool ok = true;
            for (int i = 0; i < my_tiles && ok; i++)
                for (int c = 0; c < steps_of_tile; c++) {
                    ok = warp_wait(&dfree[ds.at], ds.parity ^ 1u, err) && warp_wait(&afull[as.at], as.parity, err);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t A = tmem + as.at * 64, D = sums + ds.at * ta.r * NC;
                    const uint64_t B = bdesc + (uint64_t)(2 * c) * (NC * 128 >> 4);
                    // 8 steps of 16 codes, 32 bytes along a swizzled row of 64
#pragma unroll
                    for (int j = 0; j < 8; j++)
                        mma_f16_ts(D + (j * ta.r / 8) * NC, A + 8 * j, B + (uint64_t)(j >> 2) * (NC * 128 >> 4) + 2 * (j & 3), idesc,
                                   (j * ta.r) % 8 != 0, leader);
                    mma_commit(&afree[as.at], leader);
                    mma_commit(&dfull[ds.at], leader);
                    as.go(1, ta.na);
                    ds.go(1, ta.nd);
                }
            if (!ok) *err = 1;
            ws_drain(&drain, err, leader);
        } else {
            // --------------------------------------------------- scaling
            const int quarter = warp & 3, team = (warp - kTcDecode) >> 2;
            const uint32_t my_lanes = sums + ((uint32_t)(quarter * 32) << 16);
            // the scales of this team's steps, 8 groups ahead of their use (and
            // on into the next tile)
            int f_tile = 0, f_step = team, f_r = 0;
            const float* f_row = nullptr;
            auto fetch = [&]() {
                if (f_step == team && f_r == 0)
                    f_row = a.w.scales + min(((int)blockIdx.x + f_tile * (int)gridDim.x) * 128 + quarter * 32 + lane, N - 1) * a.w.lds;
                const uint32_t k32 = (uint32_t)(f_step * ta.r + f_r) * (4 / ta.r);
                const uint32_t gi = a.gmagic ? __umulhi(k32, a.gmagic) : k32;
                const float v = gi < (uint32_t)a.ngroups ? __ldg(f_row + gi) : 0.0f;
                if (++f_r == ta.r) {
                    f_r = 0;
                    f_step += 2;
                    if (f_step >= steps_of_tile) {
                        f_step = team;
                        f_tile++;
                    }
                }
                return v;
            };
            float ahead[8];
#pragma unroll
            for (int u = 0; u < 8; u++) ahead[u] = fetch();
            Ring ds;
            ds.go(team, ta.nd);
            bool ok = true;
            for (int i = 0; i < my_tiles; i++) {        // every tile, for the barrier below, also after a wait has given up
                const int row = ((int)blockIdx.x + i * (int)gridDim.x) * 128 + quarter * 32 + lane;
                float acc[NC];
#pragma unroll
                for (int j = 0; j < NC; j++) acc[j] = 0.0f;
                for (int c = team; c < steps_of_tile && ok; c += 2) {
                    ok = warp_wait(&dfull[ds.at], ds.parity, err);
                    if (!ok) break;
                    tc_fence_after();
                    for (int r = 0; r < ta.r; r++) {
                        uint32_t d[NC];
#pragma unroll
                        for (int j = 0; j < NC; j += 16) tmem_ld16_nw(my_lanes + (ds.at * ta.r + r) * NC + j, d + j);
                        const float s = ahead[0];
#pragma unroll
                        for (int u = 0; u < 7; u++) ahead[u] = ahead[u + 1];
                        ahead[7] = fetch();
                        tmem_wait_ld(d);
                        if (r == ta.r - 1) {
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(&dfree[ds.at]);
                        }
                        const float4* f = reinterpret_cast<const float4*>(fx + (c * ta.r + r) * NC);
#pragma unroll
                        for (int j = 0; j < NC; j += 4) {
                            if (j >= cols) break;       // the rest are not columns of x
                            const float4 v = f[j / 4];
                            acc[j] = fmaf(__uint_as_float(d[j]) * s, v.x, acc[j]);
                            if (j + 1 < cols) acc[j + 1] = fmaf(__uint_as_float(d[j + 1]) * s, v.y, acc[j + 1]);
                            if (j + 2 < cols) acc[j + 2] = fmaf(__uint_as_float(d[j + 2]) * s, v.z, acc[j + 2]);
                            if (j + 3 < cols) acc[j + 3] = fmaf(__uint_as_float(d[j + 3]) * s, v.w, acc[j + 3]);
                        }
                    }
                    ds.go(2, ta.nd);
                }
                if (!ok) *err = 1;
                // the second team's sums to the first, by way of the half of
                // `hand` that the last tile did not use
                float* h = hand + (i & 1) * NC * 128 + quarter * 32 + lane;
                if (team) {
#pragma unroll
                    for (int j = 0; j < NC; j++)
                        if (j < cols) h[j * 128] = acc[j];
                }
                asm volatile("barrier.sync %0, 64;" ::"r"(2 + quarter) : "memory");
                if (team || row >= N || !ok) continue;
#pragma unroll
                for (int j = 0; j < NC; j++)
                    if (j < cols) acc[j] += h[j * 128];
#pragma unroll
                for (int j = 0; j < NC; j++) {
                    if (a.planes == 1) {
                        if (j < mt) put_y(a, m0 + j, row, acc[j]);
                    } else if (j % 2 == 0 && j / 2 < mt) {
                        put_y(a, m0 + j / 2, row, acc[j] + acc[j + 1 < NC ? j + 1 : j]);
                    }
                }
            }
        }
    }
    __syncthreads();
    if (*err && threadIdx.x == 0) record_status(ta.status, ESB_ERR_TIMEOUT);
    if (warp == kTcIssue) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

using EncodeTiled = decltype(&cuTensorMapEncodeTiled);
EncodeTiled encode_tiled()
{
    static EncodeTiled fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiled>(f);
    });
    return fn;
}

}  // namespace

bool launch_matvec_tc(const MvArgs& args, int r, cudaStream_t st, cudaError_t* err)
{
    const int64_t sms = device_sm_count(), tiles = (args.N + 127) / 128;
    MvTcPlan p;
    if (!plan_matvec_tc(args.M, args.N, args.K, args.planes, r, (int)sms, p)) return false;
    TcArgs t;
    t.a = args;
    t.r = r;
    t.a.kc = p.kc;
    t.a.mt = p.mt;
    t.stages = p.stages;
    t.na = p.na;
    t.nd = p.nd;
    t.slot_first = p.slot_first;
    t.status = device_status_ptr();
    CUtensorMap map;
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    // rows ld words apart, of the words that are read
    const cuuint64_t dims[2] = {(cuuint64_t)args.row_codes / 8, (cuuint64_t)args.N}, strides[1] = {(cuuint64_t)args.w.ld * 4};
    const cuuint32_t box[2] = {kTcStage / 8, 128}, steps[2] = {1, 1};
    if (strides[0] >= (cuuint64_t)1 << 40 ||
        encode(&map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, const_cast<uint32_t*>(args.w.codes), dims, strides, box, steps,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return false;
    using Kernel = void (*)(const CUtensorMap, const TcArgs);
    const Kernel kernel = p.nc == 16 ? matvec_tc_kernel<16> : matvec_tc_kernel<32>;
    *err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kTcSmem);
    if (*err != cudaSuccess) return true;
    const unsigned gx = (unsigned)std::min<int64_t>(tiles, std::max<int64_t>(1, sms / p.passes));
    *err = launch_pdl(kernel, dim3(gx, (unsigned)p.passes), dim3(kTcThreads), p.smem, st, map, t);
    return true;
}

}  // namespace esb
