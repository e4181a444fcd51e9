// esb_matvec.cu -- few rows times a matrix of 4-bit ESB codes with group
// scales: y[m][n] = bias[n] + sum_g s[n][g] sum_{k in g} q(W[n][k]) x[m][k].
//
// The matrix is read once for every 8 to 32 rows, so HBM sets the floor: at
// the measured copy rate an SM receives about 43 codes a clock, which leaves
// some 20 instruction slots of its lanes for a word of 8 codes.  A
// multiply-add per code and row does not fit into that; the warp-level matrix
// instruction (m16n8k16, fp16 in, fp32 sums) takes a decoded word of two
// matrix rows for 8 rows of x at once, so the code is the operand with the 16
// rows and decoding it is the work: 13 instructions a word, and 11 issue
// cycles for each matrix instruction.  No pipe is full (1 x 65536 x 4096: issue
// 48%, ALU 55%, tensor 18%): a warp decodes and multiplies in turn, and 16 warps
// on an SM do not hide the one behind the other.  65536 x 4096 in groups of 128
// takes 40 us with one row of bf16 (21 at the copy rate), 46 with 8 and 62 with
// 16; 4096 x 4096 with one row 7 us, launch and latencies.  For more columns
// esb_matvec_tc.cu has the products on tcgen05, whose operand has to go
// through tensor memory first.
//
// fp16 holds both operands exactly.  Every element of a 4-bit set is a
// number with at most 2 fraction bits, so its fp16 high byte is a table entry
// (8 bytes in two registers: one byte permutation looks four codes up) and
// its low byte is 0.  fp16 rows of x are taken as they are; bf16 and fp32 rows
// are scaled by a power of two for every 128 values (64, 32 where groups are
// that short), so that the largest lies in [2^14, 2^15): bf16's 8 bits fit, and a value loses bits only below 2^-39 of
// the largest.  fp32 rows become two such planes (11 bits each, 2^-22 of the
// value remains); 8-bit codes are exact and bring their own scales.
//
// The sum over a group is one chain of matrix instructions and is scaled as
// fp32.  A group shorter than the 128 codes of a step gets a column of its
// own: lane t of four holds codes 32 t .. 32 t + 31 of the step, so with x
// zeroed in the other lanes a column sums one group (columns that a few rows
// leave unused anyway).
#include <algorithm>
#include <cstdint>
#include <cuda_runtime.h>

#include "esb_internal.h"
#include "esb_matvec.cuh"
#include "esb_matvec_plan.h"

namespace esb {

namespace {

constexpr int kMvWarps = 16, kMvThreads = kMvWarps * 32;   // of a block, one on an SM
constexpr int kRedLd = 20;          // floats between columns of a warp's 16 sums
// (kSteps: steps of 128 codes of a row, 16 bytes a lane and row, that a warp has
// in flight; kSlice: their codes)

__device__ __forceinline__ uint4 ldg_stream(const uint32_t* p)
{
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ uint4 lds16(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
// The warps that share a tile wait for one another.
__device__ __forceinline__ void group_barrier(int id, int threads) { asm volatile("barrier.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// c = a b, or c += a b.
template <bool ADD>
__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    if constexpr (ADD)
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
            : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}

// Shared memory: for every plane of every row kc halves -- 8 at a time in the
// pair order above, the four lanes' eights of a word next to each other --
// and 64 bytes of padding (lanes of neighbouring columns read other banks), a
// row of zeros where some lanes have no x, the columns' scales of every step,
// and the warps' sums, twice.
__host__ __device__ inline int xs_stride(int kc) { return kc * 2 + 64; }
__host__ inline size_t mv_x_bytes(int rows, int kc, int nt) { return (size_t)rows * xs_stride(kc) + (size_t)(kc / 128) * 8 * nt * 4; }
__host__ inline size_t mv_sums(int cols) { return (size_t)2 * kMvWarps * cols * kRedLd * 4; }

__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ float ld_cluster(const float* p, int rank)
{
    uint32_t a;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
    return v;
}

// Where stage_x puts a plane's eights and a column's scales.
template <int NT, int R>
struct XsPlace {
    unsigned char* xs;
    float* fx;
    int stride;
    __device__ __forceinline__ uint4* values(int row, int b) const
    {
        const int i = b & 15;
        return reinterpret_cast<uint4*>(xs + (size_t)row * stride + (size_t)(b >> 4) * 256 + ((i & 3) * 4 + (i >> 2)) * 16);
    }
    __device__ __forceinline__ float* scale(int row, int step, int r) const { return fx + step * 8 * NT + row * R + r; }
};

template <int NT, int R>
__global__ void __launch_bounds__(kMvThreads, 1) matvec_kernel(const MvArgs a)
{
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ uint16_t xtab[256];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int64_t m0 = (int64_t)blockIdx.z * a.mt;
    const int mt = (int)min((int64_t)a.mt, a.M - m0);
    const int cols = mt * a.planes * R;
    const int k0 = (int)blockIdx.y * a.kc;
    const int slices = min(a.kc / kSlice, ((int)a.K - k0 + kSlice - 1) / kSlice);   // may be <= 0 in the last block of a row
    unsigned char* xs = smem;
    unsigned char* zeros = xs + (size_t)a.mt * a.planes * xs_stride(a.kc);
    float* fx = reinterpret_cast<float*>(zeros + (a.zrow ? xs_stride(a.kc) : 0));
    float* red = fx + (a.kc / 128) * 8 * NT;
    const int part = a.mt * a.planes * R * kRedLd;      // floats of a warp's sums of a tile
    const int batch = kMvWarps * part;

    const int wn = kMvWarps / a.wk;                     // tiles of 16 rows in work at once
    const int wi = warp / a.wk, wj = warp % a.wk;       // this warp's tile of them, and its place along the row
    const int N = (int)a.N, tiles = (N + 15) / 16, stride = (int)gridDim.x * wn;
    const int first = (int)blockIdx.x * wn;

    griddep_wait();
    griddep_launch_dependents();
    // Loads of the slice after the one in work go into each step's registers as
    // soon as that step is done.
    uint4 buf[kSteps][2];
    float sc[2][R];                                     // scales of step t of the slice, rows g and g + 8
    const uint32_t* pw[2];                              // this lane's place in the slice that is loaded next
    const float* ps[2];
    int p_k = k0 + wj * kSlice, p_base = first;         // its first code, its tile
    auto rows_of = [&]() {
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const int n = min((p_base + wi) * 16 + 8 * i + g, N - 1);
            pw[i] = a.w.codes + n * a.w.ld + (p_k / 8 + t * 4);
            ps[i] = a.w.scales + n * a.w.lds;
        }
    };
    auto load_step = [&](int c) {
        if (p_k + kSlice <= (int)a.row_codes) {
            buf[c][0] = ldg_stream(pw[0] + c * 16);
            buf[c][1] = ldg_stream(pw[1] + c * 16);
        } else {
            const int o = mv_end_words(p_k, t, c, (int)a.row_codes);
            buf[c][0] = ldg_stream(pw[0] + o);
            buf[c][1] = ldg_stream(pw[1] + o);
        }
    };
    auto load_scales = [&]() {
#pragma unroll
        for (int j = 0; j < R; j++) {
            const uint32_t k32 = (uint32_t)p_k / 32 + (t % kSteps) * 4 + j * (4 / R);
            const uint32_t gi = a.gmagic ? __umulhi(k32, a.gmagic) : k32;
            const bool in = gi < (uint32_t)a.ngroups;
            sc[0][j] = in ? __ldg(ps[0] + gi) : 0.0f;
            sc[1][j] = in ? __ldg(ps[1] + gi) : 0.0f;
        }
    };
    rows_of();
    if (wj < slices) {
#pragma unroll
        for (int c = 0; c < kSteps; c++) load_step(c);
        load_scales();
    }

    for (int i = threadIdx.x; i < (a.kc / 128) * 8 * NT; i += kMvThreads)
        if (i % (8 * NT) >= cols) fx[i] = 0.0f;
    if (a.zrow)
        for (int i = threadIdx.x * 16; i < a.kc * 2; i += kMvThreads * 16) *reinterpret_cast<uint4*>(zeros + i) = make_uint4(0u, 0u, 0u, 0u);
    if (a.x_type == ESB_CODES) {
        for (int i = threadIdx.x; i < 256; i += kMvThreads) xtab[i] = x_code_half(i, a.xc.fmt.k);
        __syncthreads();
    }
    stage_x<R>(a, m0, mt, k0, XsPlace<NT, R>{xs, fx, xs_stride(a.kc)}, xtab, kMvWarps, warp);
    __syncthreads();

    // where this lane reads x for column 8 i + g: its row's plane, or zeros
    uint32_t xp[NT];
#pragma unroll
    for (int i = 0; i < NT; i++) {
        const int col = 8 * i + g;
        const bool on = col < cols && (t * R) / 4 == col % R;
        xp[i] = smem_u32((on ? xs + (size_t)(col / R) * xs_stride(a.kc) : zeros) + t * 16);
    }
    const uint32_t fp = smem_u32(fx) + t * 8;

    auto put = [&](int n, int m, float v) { put_y(a, m0 + m, n, v); };

    int flip = 0, held = 0;                             // held: tiles whose sums wait in red's half
    for (int base = first; base < tiles; base += stride) {
        float acc[NT][4];
#pragma unroll
        for (int i = 0; i < NT; i++) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.0f;
#pragma unroll 1
        for (int sl = wj; sl < slices; sl += a.wk) {
            float cur[2][R];
#pragma unroll
            for (int j = 0; j < R; j++) {
                cur[0][j] = sc[0][j];
                cur[1][j] = sc[1][j];
            }
            bool more = true;
            if (sl + a.wk < slices) {
                p_k += a.wk * kSlice;
                pw[0] += a.wk * (kSlice / 8);
                pw[1] += a.wk * (kSlice / 8);
            } else {
                p_k = k0 + wj * kSlice;
                p_base += stride;
                more = p_base < tiles;
                rows_of();
            }
            if (more) load_scales();
            const uint32_t xo = (uint32_t)sl * (256u * kSteps), fo = fp + (uint32_t)sl * (32u * kSteps * NT);
#pragma unroll
            for (int c = 0; c < kSteps; c++) {
                const uint32_t wa[4] = {buf[c][0].x, buf[c][0].y, buf[c][0].z, buf[c][0].w};
                const uint32_t wb[4] = {buf[c][1].x, buf[c][1].y, buf[c][1].z, buf[c][1].w};
                float sum[NT][4];
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    uint32_t da[4], db[4];
                    decode8(wa[q], a.tab, da);
                    decode8(wb[q], a.tab, db);
#pragma unroll
                    for (int i = 0; i < NT; i++) {
                        const uint4 b = lds16(xp[i] + xo + c * 256 + q * 64);
                        if (q == 0) mma_16816<false>(sum[i], da[0], db[0], da[1], db[1], b.x, b.y);
                        else mma_16816<true>(sum[i], da[0], db[0], da[1], db[1], b.x, b.y);
                        mma_16816<true>(sum[i], da[2], db[2], da[3], db[3], b.z, b.w);
                    }
                }
                if (more) load_step(c);
                // this lane's sums: rows g and g + 8, columns 2 t and 2 t + 1 of each eight
                float s[2][2];
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    float q[R];
#pragma unroll
                    for (int j = 0; j < R; j++) q[j] = __shfl_sync(0xffffffffu, cur[h][j], (lane & 28) | c);
                    const bool up = R == 4 && (t & 1);
                    s[h][0] = up ? q[2 % R] : q[0];
                    s[h][1] = up ? q[3 % R] : q[1 % R];
                }
#pragma unroll
                for (int i = 0; i < NT; i++) {
                    float2 fc;
                    asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(fc.x), "=f"(fc.y) : "r"(fo + (c * NT + i) * 32) : "memory");
                    acc[i][0] = fmaf(sum[i][0] * s[0][0], fc.x, acc[i][0]);
                    acc[i][1] = fmaf(sum[i][1] * s[0][1], fc.y, acc[i][1]);
                    acc[i][2] = fmaf(sum[i][2] * s[1][0], fc.x, acc[i][2]);
                    acc[i][3] = fmaf(sum[i][3] * s[1][1], fc.y, acc[i][3]);
                }
            }
        }
        // the warps' parts wait until `hold` tiles are there; then they are
        // added up, in their order.  A half of red is written again behind the
        // other half's barrier.
        float* rw = red + (flip * a.hold + held) * batch + warp * part;
#pragma unroll
        for (int i = 0; i < NT; i++)
#pragma unroll
            for (int e = 0; e < 2; e++) {
                const int col = 8 * i + 2 * t + e;
                float* p = rw + col * kRedLd + g;
                if (col < cols) {
                    p[0] = acc[i][e];
                    p[8] = acc[i][2 + e];
                }
            }
        if (++held < a.hold && base + stride < tiles) continue;
        group_barrier(wi, a.wk * 32);
        const int each = 16 * mt;
        for (int o = wj * 32 + lane; o < held * each; o += a.wk * 32) {
            const int h = o / each, u = o - h * each, row = u & 15, m = u >> 4;
            float* p = red + (flip * a.hold + h) * batch + wi * a.wk * part + m * a.planes * R * kRedLd + row;
            float v = 0.0f;
            for (int j = 0; j < a.wk; j++)
                for (int q = 0; q < a.planes * R; q++) v += p[j * part + q * kRedLd];
            const int n = (base - (held - 1 - h) * stride + wi) * 16 + row;
            if (a.split > 1) p[0] = v;                  // this block's part, at the first of the numbers it sums
            else if (n < N) put(n, m, v);
        }
        if (a.split > 1) {
            cluster_barrier();
            for (int o = wj * 32 + lane; o < held * each; o += a.wk * 32) {
                const int h = o / each, u = o - h * each, row = u & 15, m = u >> 4;
                const int n = (base - (held - 1 - h) * stride + wi) * 16 + row;
                if (m % a.split != (int)blockIdx.y || n >= N) continue;   // the blocks take the rows of x in turn
                const float* p = red + (flip * a.hold + h) * batch + wi * a.wk * part + m * a.planes * R * kRedLd + row;
                float v = 0.0f;
                for (int j = 0; j < a.split; j++) v += ld_cluster(p, j);
                put(n, m, v);
            }
        }
        flip ^= 1;
        held = 0;
    }
    if (a.split > 1) cluster_barrier();                 // no block leaves while another reads its sums
}

// fp16 high bytes of the non-negative elements by the code's low 3 bits.
void element_bytes(int k, uint32_t& lo, uint32_t& hi)
{
    uint32_t b[8];
    const int n = fmt_N(4, k);
    for (int c = 0; c < 8; c++) {
        const int e = (c >> k) & n, f = c & ((1 << k) - 1);
        const double v = e == n ? (double)f / (1 << k) : (1.0 + (double)f / (1 << k)) * (1 << e);
        int ex = 0;
        double m = v;
        if (v != 0.0) {
            while (m >= 2.0) { m *= 0.5; ex++; }
            while (m < 1.0) { m *= 2.0; ex--; }
        }
        b[c] = v == 0.0 ? 0u : (uint32_t)((ex + 15) << 2) | (uint32_t)((m - 1.0) * 4.0);
    }
    lo = b[0] | (b[1] << 8) | (b[2] << 16) | (b[3] << 24);
    hi = b[4] | (b[5] << 8) | (b[6] << 16) | (b[7] << 24);
}

using MvKernel = void (*)(const MvArgs);
constexpr size_t kMvSmem = 225 * 1024;
template <int R> MvKernel mv_kernel(int nt)
{
    return nt == 1 ? matvec_kernel<1, R> : (nt == 2 ? matvec_kernel<2, R> : matvec_kernel<4, R>);
}

}  // namespace

cudaError_t launch_matvec_groups(int64_t M, int64_t N, int64_t K, const void* x, int x_type, int64_t ldx, const esb_coded* xc,
                                 const esb_coded& w, const float* bias, void* y, int y_type, int64_t ldy, cudaStream_t st)
{
    MvArgs a;
    a.M = M; a.N = N; a.K = K;
    a.x = x; a.ldx = ldx;
    a.xc = xc ? *xc : esb_coded{};
    a.w = w;
    const int64_t whole = (K + 127) / 128 * 128;
    if (a.w.group <= 0 || a.w.group >= K) a.w.group = whole;
    a.ngroups = (K + a.w.group - 1) / a.w.group;
    a.xgroup = xc && xc->group > 0 && xc->group < K ? xc->group : whole;
    const int64_t g32 = a.w.group / 32;                 // k / group for k / 32 < 2^13: one high product
    a.gmagic = g32 == 1 ? 0u : (uint32_t)(((1ll << 32) + g32 - 1) / g32);
    a.bias = bias; a.y = y; a.ldy = ldy;
    a.x_type = x_type; a.y_type = y_type;
    a.xvec = x && (reinterpret_cast<uintptr_t>(x) & 15u) == 0 && ldx * type_bytes(x_type) % 16 == 0;
    element_bytes(w.fmt.k, a.tab.lo, a.tab.hi);
    a.tab.by16 = 1u << 16;
    a.tab.by4 = 1u << 4;
    const int r = a.w.group % 128 == 0 ? 1 : (a.w.group % 64 == 0 ? 2 : 4);
    a.planes = x_type == ESB_F32 ? 2 : 1;
    a.row_codes = mv_row_codes(K);

    cudaError_t e = cudaSuccess;
    if (launch_matvec_tc(a, r, st, &e)) return e;

    // Rows a block takes at once: up to 32 columns' worth, fewer where x would
    // not fit; the row's codes over up to 8 blocks (a cluster) where that
    // makes x fit.  Also over four where the matrix is wider than high and
    // has a tile a warp at most: preparing x is what takes long there (4 x
    // 4096 x 9216, x in 8-bit codes, groups of 64: 14 us, 17 without; 4 rows of
    // bf16 times 1024 x 14336: 11 and 14).  Each tile's sums then cross the
    // cluster, which costs more for high matrices (4 x 8192 x 4096 bf16: 10.9
    // and 10.7; 12000 x 4096, several tiles a warp: 23 and 15) and for one row
    // of x is as long as what it saves.
    const int sms = device_sm_count();
    const int most = 32 / (a.planes * r);
    const int64_t tiles = (N + 15) / 16, all = (K + 511) / 512;
    int64_t passes = (M + most - 1) / most;
    MvKernel kernel;
    size_t smem;
    for (;; passes *= 2) {
        a.mt = (int)((M + passes - 1) / passes);
        const int cols = a.mt * a.planes * r, nt = cols <= 8 ? 1 : (cols <= 16 ? 2 : 4);
        kernel = r == 1 ? mv_kernel<1>(nt) : (r == 2 ? mv_kernel<2>(nt) : mv_kernel<4>(nt));
        a.zrow = r > 1 || cols < 8 * nt;
        const bool spread = K >= 4096 && N <= K && a.mt * a.planes >= 4 && tiles <= kMvWarps * sms / (4 * passes);
        for (a.split = spread ? 4 : 1;; a.split *= 2) {
            a.kc = (int)((all + a.split - 1) / a.split) * 512;
            const size_t sums = mv_sums(cols);
            smem = mv_x_bytes(a.mt * a.planes + a.zrow, a.kc, nt) + sums;
            a.hold = 1;
            while (a.hold < 4 && (a.hold + 1) * sums <= 16 * 1024) a.hold++;
            smem += (a.hold - 1) * sums;
            if (a.split == 8 || smem <= kMvSmem) break;
        }
        if (smem <= kMvSmem || a.mt == 1) break;
    }
    passes = (M + a.mt - 1) / a.mt;
    const int64_t at_once = std::max<int64_t>(1, sms / (a.split * std::min<int64_t>(passes, sms)));   // blocks of a pass on the SMs
    // Warps along a row: as few rounds as possible of tiles of so many slices,
    // each with a quarter slice's worth of work besides.
    const int64_t slices = a.kc / kSlice;
    double best = 0.0;
    a.wk = 0;
    for (int wk = 1; wk <= kMvWarps && wk <= slices; wk *= 2) {
        const int64_t wn = kMvWarps / wk, rounds = (tiles + wn * at_once - 1) / (wn * at_once);
        const double cost = (double)rounds * ((double)((slices + wk - 1) / wk) + 0.25);
        if (!a.wk || cost < best) { best = cost; a.wk = wk; }
    }
    const int64_t want = (tiles + kMvWarps / a.wk - 1) / (kMvWarps / a.wk), cap = at_once;
    if (smem > 47 * 1024) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMvSmem);
    if (e != cudaSuccess) return e;
    for (int64_t p0 = 0; p0 < passes; p0 += 65535) {    // grid.z holds 65535 passes
        const int64_t np = passes - p0 < 65535 ? passes - p0 : 65535;
        MvArgs b = a;
        b.M = M - p0 * a.mt;
        b.y = static_cast<char*>(y) + p0 * a.mt * ldy * type_bytes(y_type);
        if (xc) {
            b.xc.codes += p0 * a.mt * xc->ld;
            b.xc.scales += p0 * a.mt * xc->lds;
        } else {
            b.x = static_cast<const char*>(x) + p0 * a.mt * ldx * type_bytes(x_type);
        }
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(want < cap ? want : cap), (unsigned)a.split, (unsigned)np);
        cfg.blockDim = dim3(kMvThreads);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = st;
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = 1;
        attr[1].val.clusterDim.y = (unsigned)a.split;
        attr[1].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = a.split > 1 ? 2 : 1;
        e = cudaLaunchKernelEx(&cfg, kernel, b);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace esb
