// esb_matvec.cu -- few rows times a matrix of 4-bit ESB codes with group
// scales: y[m][n] = bias[n] + sum_g s[n][g] sum_{k in g} q(W[n][k]) x[m][k].
//
// The matrix is read once for every 8 to 32 rows, so HBM bounds the call: at
// the measured copy rate an SM receives about 43 codes a clock, which leaves
// some 20 instruction slots of its lanes for a word of 8 codes.  A
// multiply-add per code and row does not fit into that; the warp-level matrix
// instruction (m16n8k16, fp16 in, fp32 sums) takes a decoded word of two
// matrix rows for 8 rows of x at once, so the code is the operand with the 16
// rows and decoding it is the work.  (tcgen05 would need the decoded matrix
// in shared memory first, four bytes written and read there for every byte
// from HBM, for a tile of 8 to 32 columns.)
//
// fp16 holds both operands exactly.  Every element of a 4-bit set is a
// number with at most 2 fraction bits, so its fp16 high byte is a table entry
// (8 bytes in two registers: one byte permutation looks four codes up) and
// its low byte is 0.  Rows of x are scaled by a power of two for every 128
// values (64, 32 where groups are that short), so that the largest lies in
// [2^14, 2^15): bf16's 8 bits fit, and a value loses bits only below 2^-39 of
// the largest.  fp32 rows become two such planes (11 bits each, 2^-22 of the
// value remains); 8-bit codes are exact and bring their own scales.
//
// The sum over a group is one chain of matrix instructions and is scaled as
// fp32.  A group shorter than the 128 codes of a step gets a column of its
// own: lane t of four holds codes 32 t .. 32 t + 31 of the step, so with x
// zeroed in the other lanes a column sums one group (columns that a few rows
// leave unused anyway).
#include <cstdint>
#include <cuda_runtime.h>

#include "esb_internal.h"
#include "esb_rows.cuh"

namespace esb {

namespace {

constexpr int kMvWarps = 8;
constexpr int kMvThreads = kMvWarps * 32;
constexpr int kSlice = 512;         // codes of a row in flight per warp: 16 bytes a lane, 4 steps
constexpr int kRedLd = 20;          // floats between columns of a warp's 16 sums

struct MvArgs {
    int64_t M, N, K;
    const void* x;
    int64_t ldx;
    esb_coded xc;                   // for x_type ESB_CODES
    esb_coded w;
    int64_t xgroup, ngroups;
    const float* bias;
    void* y;
    int64_t ldy;
    uint32_t tab_lo, tab_hi;        // fp16 high bytes of elements 0..7 of the code's low 3 bits
    int x_type, y_type, xvec;
    int mt, planes;                 // rows of x in a block, planes of each
    int kc;                         // codes of a row in a block (a multiple of kSlice)
    int wk;                         // warps along a row (the others take other tiles)
    int split;                      // blocks along a row (a cluster)
};

__device__ __forceinline__ uint4 ldg_stream(const uint32_t* p)
{
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Eight codes as four fp16 pairs {0,2} {1,3} {4,6} {5,7}: the order in which
// a word's sign bits lie at the top of alternate bytes.
__device__ __forceinline__ void decode8(uint32_t w, uint32_t lo, uint32_t hi, uint32_t (&p)[4])
{
    const uint32_t sel = w & 0x77777777u;
    const uint32_t m03 = __byte_perm(lo, hi, sel), m47 = __byte_perm(lo, hi, sel >> 16);
    const uint32_t odd = __byte_perm(m03, m47, 0x7531) | (w & 0x80808080u);
    const uint32_t even = __byte_perm(m03, m47, 0x6420) | ((w << 4) & 0x80808080u);
    p[0] = __byte_perm(even, 0u, 0x1404);
    p[1] = __byte_perm(odd, 0u, 0x1404);
    p[2] = __byte_perm(even, 0u, 0x3424);
    p[3] = __byte_perm(odd, 0u, 0x3424);
}

__device__ __forceinline__ uint32_t half2_of(float a, float b) { return pack2<__half>(a, b); }

// Shared memory: 256 zero bytes (x of columns that are not there), then for
// every plane of every row kc halves -- 8 at a time in the pair order above,
// the four lanes' eights of a word next to each other -- and 64 bytes of
// padding (lanes of neighbouring columns read other banks), the columns'
// scales of every step, and the warps' sums, twice.
__host__ __device__ inline int xs_stride(int kc) { return kc * 2 + 64; }
__host__ inline size_t mv_smem(int rows, int kc, int nt)
{
    return 256 + (size_t)rows * xs_stride(kc) + (size_t)(kc / 128) * 8 * nt * 4 + 2u * kMvWarps * 8 * nt * kRedLd * 4;
}

__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float ld_cluster(const float* p, int rank)
{
    uint32_t a;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
    return v;
}

// Rows m0 .. m0 + mt - 1 of x, codes k0 .. k0 + kc - 1, into shared memory.
template <int NT, int R>
__device__ __forceinline__ void stage_x(const MvArgs& a, int64_t m0, int mt, int64_t k0, unsigned char* xs, float* fx, const uint16_t* xtab)
{
    constexpr int LANES = 16 / R;                       // lanes that share a scale
    const int stride = xs_stride(a.kc), blocks = a.kc / 8;
    for (int m = 0; m < mt; m++) {
        for (int b = threadIdx.x; b < blocks; b += kMvThreads) {   // blocks is a multiple of 64: warps stay whole
            const int64_t k = k0 + (int64_t)b * 8;
            const int64_t n = a.K - k;
            const int i = b & 15, step = b >> 4, r = i / LANES;
            unsigned char* at = xs + (size_t)(m * a.planes) * stride + (size_t)(step * 128 + ((i & 3) * 4 + (i >> 2)) * 8) * 2;
            float* f = fx + step * 8 * NT + m * a.planes * R + r;
            uint4 out;
            if (a.x_type == ESB_CODES) {
                uint32_t h[8];
                const uint32_t* xw = a.xc.codes + (m0 + m) * a.xc.ld + k / 4;
                const uint32_t w0 = n > 0 ? xw[0] : 0u, w1 = n > 4 ? xw[1] : 0u;
#pragma unroll
                for (int j = 0; j < 8; j++) h[j] = j < n ? xtab[((j < 4 ? w0 : w1) >> (8 * (j & 3))) & 255u] : 0u;
                out = make_uint4(h[0] | (h[2] << 16), h[1] | (h[3] << 16), h[4] | (h[6] << 16), h[5] | (h[7] << 16));
                if (i % LANES == 0)
                    *f = n > 0 ? a.xc.scales[(m0 + m) * a.xc.lds + k / a.xgroup] * (a.xc.fmt.k == 2 ? 65536.0f : 1.0f) : 0.0f;
            } else {
                float v[8];
                load8_any(a.x, a.x_type, (m0 + m) * a.ldx + k, n, a.xvec, v);
                float s = 1.0f, back = 1.0f;
                if (a.x_type != ESB_F16) {
                    uint32_t mx = 0u;
#pragma unroll
                    for (int j = 0; j < 8; j++) {
                        const uint32_t u = __float_as_uint(v[j]) & 0x7fffffffu;
                        mx = max(mx, u < 0x7f800000u ? u : 0u);
                    }
#pragma unroll
                    for (int o = LANES / 2; o > 0; o >>= 1) mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, o));
                    const int e = max((int)(mx >> 23), 15);          // exponent field; 2^(14 - (e - 127)) <= 2^126
                    s = __uint_as_float((uint32_t)(268 - e) << 23);
                    back = __uint_as_float((uint32_t)(e - 14) << 23);
#pragma unroll
                    for (int j = 0; j < 8; j++) v[j] *= s;
                }
                if (a.planes == 2) {
                    float lo[8];
#pragma unroll
                    for (int j = 0; j < 8; j++) {
                        const float hi = __half2float(__float2half_rn(v[j]));
                        lo[j] = fabsf(hi) < __int_as_float(0x7f800000) ? (v[j] - hi) * 2048.0f : 0.0f;
                        v[j] = hi;
                    }
                    *reinterpret_cast<uint4*>(at + stride) = make_uint4(half2_of(lo[0], lo[2]), half2_of(lo[1], lo[3]),
                                                                        half2_of(lo[4], lo[6]), half2_of(lo[5], lo[7]));
                    if (i % LANES == 0) f[R] = back * (1.0f / 2048.0f);
                }
                out = make_uint4(half2_of(v[0], v[2]), half2_of(v[1], v[3]), half2_of(v[4], v[6]), half2_of(v[5], v[7]));
                if (i % LANES == 0) *f = back;
            }
            *reinterpret_cast<uint4*>(at) = out;
        }
    }
}

template <int NT, int R>
__global__ void __launch_bounds__(kMvThreads, 2) matvec_kernel(const MvArgs a)
{
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ uint16_t xtab[256];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int64_t m0 = (int64_t)blockIdx.z * a.mt;
    const int mt = (int)min((int64_t)a.mt, a.M - m0);
    const int cols = mt * a.planes * R;
    const int64_t k0 = (int64_t)blockIdx.y * a.kc;
    const int slices = (int)min((int64_t)(a.kc / kSlice), (a.K - k0 + kSlice - 1) / kSlice);   // may be <= 0 in the last block of a row
    unsigned char* xs = smem + 256;
    float* fx = reinterpret_cast<float*>(xs + (size_t)a.mt * a.planes * xs_stride(a.kc));
    float* red = fx + (a.kc / 128) * 8 * NT;

    const int wn = kMvWarps / a.wk;                     // tiles of 16 rows in work at once
    const int wi = warp / a.wk, wj = warp % a.wk;       // this warp's tile of them, and its place along the row
    const int64_t tiles = (a.N + 15) / 16, step = (int64_t)gridDim.x * wn;
    const int mine = slices > wj ? (slices - wj + a.wk - 1) / a.wk : 0;

    griddep_wait();
    griddep_launch_dependents();
    uint4 buf[4][2];
    float sc[2][R];                                     // scales of step t of the slice, rows g and g + 8
    const uint32_t *pa = nullptr, *pb = nullptr;
    const float *sa = nullptr, *sb = nullptr;
    auto rows_of = [&](int64_t tile) {
        const int64_t na = min(tile * 16 + g, a.N - 1), nb = min(tile * 16 + 8 + g, a.N - 1);
        pa = a.w.codes + na * a.w.ld;
        pb = a.w.codes + nb * a.w.ld;
        sa = a.w.scales + na * a.w.lds;
        sb = a.w.scales + nb * a.w.lds;
    };
    auto load_step = [&](int sl, int c, bool ok) {
        const int64_t at = (k0 + (int64_t)sl * kSlice + c * 128) / 8 + t * 4;
        ok = ok && at < a.w.ld;                         // ld is a multiple of 4: all 16 bytes are the row's
        buf[c][0] = buf[c][1] = make_uint4(0u, 0u, 0u, 0u);
        if (ok) {
            buf[c][0] = ldg_stream(pa + at);
            buf[c][1] = ldg_stream(pb + at);
        }
    };
    auto load_scales = [&](int sl, bool ok) {
#pragma unroll
        for (int i = 0; i < R; i++) {
            const uint32_t k = (uint32_t)(k0 + (int64_t)sl * kSlice + t * 128 + i * (128 / R));
            const uint32_t gi = k / (uint32_t)a.w.group;
            const bool in = ok && gi < (uint32_t)a.ngroups;
            sc[0][i] = in ? __ldg(sa + gi) : 0.0f;
            sc[1][i] = in ? __ldg(sb + gi) : 0.0f;
        }
    };
    int64_t base = (int64_t)blockIdx.x * wn;
    rows_of(base + wi);
#pragma unroll
    for (int c = 0; c < 4; c++) load_step(wj, c, mine > 0);
    load_scales(wj, mine > 0);

    if (threadIdx.x < 16) reinterpret_cast<uint4*>(smem)[threadIdx.x] = make_uint4(0u, 0u, 0u, 0u);
    for (int i = threadIdx.x; i < (a.kc / 128) * 8 * NT; i += kMvThreads)
        if (i % (8 * NT) >= cols) fx[i] = 0.0f;
    if (a.x_type == ESB_CODES) {
        // k = 2 reaches 1.75 * 2^30; its elements are scaled by 2^-16
        const float v = code_value(threadIdx.x, 8, a.xc.fmt.k) * (a.xc.fmt.k == 2 ? 1.0f / 65536.0f : 1.0f);
        const __half h = __float2half_rn(v);
        xtab[threadIdx.x] = *reinterpret_cast<const uint16_t*>(&h);
        __syncthreads();
    }
    stage_x<NT, R>(a, m0, mt, k0, xs, fx, xtab);
    __syncthreads();

    // where this lane reads x for column 8 i + g: its row's plane, or zeros
    const unsigned char* xp[NT];
    uint32_t xmask[NT];
#pragma unroll
    for (int i = 0; i < NT; i++) {
        const int col = 8 * i + g;
        const bool on = col < cols && (t * R) / 4 == col % R;
        xp[i] = on ? xs + (size_t)(col / R) * xs_stride(a.kc) + t * 16 : smem;
        xmask[i] = on ? 0xffffffffu : 0u;
    }

    int flip = 0;
    for (; base < tiles; base += step) {
        float acc[NT][4];
#pragma unroll
        for (int i = 0; i < NT; i++) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.0f;
        for (int j = 0; j < mine; j++) {
            const int sl = wj + j * a.wk;
            const bool last = j == mine - 1;
            const bool more = !last || base + step < tiles;
            const int nsl = last ? wj : sl + a.wk;
            if (last) rows_of(base + step + wi);
            float cur[2][R];
#pragma unroll
            for (int i = 0; i < R; i++) {
                cur[0][i] = sc[0][i];
                cur[1][i] = sc[1][i];
            }
            load_scales(nsl, more);
#pragma unroll
            for (int c = 0; c < 4; c++) {
                const uint32_t wa[4] = {buf[c][0].x, buf[c][0].y, buf[c][0].z, buf[c][0].w};
                const uint32_t wb[4] = {buf[c][1].x, buf[c][1].y, buf[c][1].z, buf[c][1].w};
                load_step(nsl, c, more);
                float sum[NT][4];
#pragma unroll
                for (int i = 0; i < NT; i++) sum[i][0] = sum[i][1] = sum[i][2] = sum[i][3] = 0.0f;
                const uint32_t off = (uint32_t)(sl * 4 + c) * 256u;
#pragma unroll
                for (int w = 0; w < 4; w++) {
                    uint32_t da[4], db[4];
                    decode8(wa[w], a.tab_lo, a.tab_hi, da);
                    decode8(wb[w], a.tab_lo, a.tab_hi, db);
#pragma unroll
                    for (int i = 0; i < NT; i++) {
                        const uint4 b = *reinterpret_cast<const uint4*>(xp[i] + (off & xmask[i]) + w * 64);
                        mma_16816(sum[i], da[0], db[0], da[1], db[1], b.x, b.y);
                        mma_16816(sum[i], da[2], db[2], da[3], db[3], b.z, b.w);
                    }
                }
                // this lane's sums: rows g and g + 8, columns 2 t and 2 t + 1 of each eight
                float s0[2], s1[2];
                if constexpr (R == 1) {
                    s0[0] = s0[1] = __shfl_sync(0xffffffffu, cur[0][0], (lane & 28) | c);
                    s1[0] = s1[1] = __shfl_sync(0xffffffffu, cur[1][0], (lane & 28) | c);
                } else {
                    float q0[R], q1[R];
#pragma unroll
                    for (int i = 0; i < R; i++) {
                        q0[i] = __shfl_sync(0xffffffffu, cur[0][i], (lane & 28) | c);
                        q1[i] = __shfl_sync(0xffffffffu, cur[1][i], (lane & 28) | c);
                    }
                    const bool up = R == 4 && (t & 1);
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        s0[i] = up ? q0[(i + 2) % R] : q0[i];
                        s1[i] = up ? q1[(i + 2) % R] : q1[i];
                    }
                }
                const float* f = fx + (sl * 4 + c) * 8 * NT + 2 * t;
#pragma unroll
                for (int i = 0; i < NT; i++) {
                    const float2 fc = *reinterpret_cast<const float2*>(f + 8 * i);
                    acc[i][0] = fmaf(sum[i][0] * s0[0], fc.x, acc[i][0]);
                    acc[i][1] = fmaf(sum[i][1] * s0[1], fc.y, acc[i][1]);
                    acc[i][2] = fmaf(sum[i][2] * s1[0], fc.x, acc[i][2]);
                    acc[i][3] = fmaf(sum[i][3] * s1[1], fc.y, acc[i][3]);
                }
            }
        }
        // the warps' parts of each tile, in their order
        float* rw = red + (size_t)(flip * kMvWarps + warp) * 8 * NT * kRedLd;
#pragma unroll
        for (int i = 0; i < NT; i++) {
            float* p = rw + (8 * i + 2 * t) * kRedLd + g;
            p[0] = acc[i][0];
            p[kRedLd] = acc[i][1];
            p[8] = acc[i][2];
            p[kRedLd + 8] = acc[i][3];
        }
        __syncthreads();
        for (int o = threadIdx.x; o < wn * 16 * mt; o += kMvThreads) {
            const int row = o & 15, m = (o >> 4) % mt, ti = (o >> 4) / mt;
            float* p = red + (size_t)(flip * kMvWarps + ti * a.wk) * 8 * NT * kRedLd + row;
            float v = 0.0f;
            for (int j = 0; j < a.wk; j++)
                for (int c = 0; c < a.planes * R; c++) v += p[(size_t)j * 8 * NT * kRedLd + (m * a.planes * R + c) * kRedLd];
            if (a.split > 1) {
                p[m * a.planes * R * kRedLd] = v;       // this block's part, at the first of the numbers it sums
                continue;
            }
            const int64_t n = (base + ti) * 16 + row;
            if (n < a.N) {
                if (a.bias) v += a.bias[n];
                const int64_t at = (m0 + m) * a.ldy + n;
                if (a.y_type == ESB_F32) static_cast<float*>(a.y)[at] = v;
                else if (a.y_type == ESB_F16) static_cast<__half*>(a.y)[at] = __float2half_rn(v);
                else static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v);
            }
        }
        if (a.split > 1) {
            // the blocks' parts, in their order.  A part is written again two
            // tiles on, behind the next barrier.
            cluster_barrier();
            for (int o = threadIdx.x; o < wn * 16 * mt; o += kMvThreads) {
                if (o % a.split != (int)blockIdx.y) continue;
                const int row = o & 15, m = (o >> 4) % mt, ti = (o >> 4) / mt;
                const int64_t n = (base + ti) * 16 + row;
                if (n >= a.N) continue;
                const float* p = red + (size_t)(flip * kMvWarps + ti * a.wk) * 8 * NT * kRedLd + row + m * a.planes * R * kRedLd;
                float v = 0.0f;
                for (int j = 0; j < a.split; j++) v += ld_cluster(p, j);
                if (a.bias) v += a.bias[n];
                const int64_t at = (m0 + m) * a.ldy + n;
                if (a.y_type == ESB_F32) static_cast<float*>(a.y)[at] = v;
                else if (a.y_type == ESB_F16) static_cast<__half*>(a.y)[at] = __float2half_rn(v);
                else static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v);
            }
        }
        flip ^= 1;
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
template <int R> MvKernel mv_kernel(int nt) { return nt == 1 ? matvec_kernel<1, R> : (nt == 2 ? matvec_kernel<2, R> : matvec_kernel<4, R>); }

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
    a.bias = bias; a.y = y; a.ldy = ldy;
    a.x_type = x_type; a.y_type = y_type;
    a.xvec = x && (reinterpret_cast<uintptr_t>(x) & 15u) == 0 && ldx * type_bytes(x_type) % 16 == 0;
    element_bytes(w.fmt.k, a.tab_lo, a.tab_hi);
    const int r = a.w.group % 128 == 0 ? 1 : (a.w.group % 64 == 0 ? 2 : 4);
    a.planes = x_type == ESB_F32 ? 2 : 1;

    // Rows a block takes at once: up to 32 columns' worth, fewer where x would
    // not fit; the row's codes over up to 8 blocks (a cluster) where that
    // makes it fit twice into an SM, or gives the SMs work.
    const int sms = device_sm_count();
    const int most = 32 / (a.planes * r);
    const int64_t tiles = (N + 15) / 16, all = (K + kSlice - 1) / kSlice;
    int64_t passes = (M + most - 1) / most;
    int nt;
    size_t smem;
    for (;; passes *= 2) {
        a.mt = (int)((M + passes - 1) / passes);
        const int cols = a.mt * a.planes * r;
        nt = cols <= 8 ? 1 : (cols <= 16 ? 2 : 4);
        for (a.split = 1;; a.split *= 2) {
            a.kc = (int)((all + a.split - 1) / a.split) * kSlice;
            smem = mv_smem(a.mt * a.planes, a.kc, nt);
            if (a.split == 8) break;
            if (smem <= 100 * 1024 && (tiles * a.split >= sms || a.kc <= 8 * kSlice)) break;
        }
        if (smem <= 200 * 1024 || a.mt == 1) break;
    }
    passes = (M + a.mt - 1) / a.mt;
    const int sl = a.kc / kSlice;
    a.wk = sl > 4 ? 8 : (sl > 2 ? 4 : sl);
    const int64_t want = (tiles + kMvWarps / a.wk - 1) / (kMvWarps / a.wk);
    int64_t cap = 2 * sms / (a.split * (passes < 8 ? passes : 8));
    if (cap < 1) cap = 1;
    const MvKernel kernel = r == 1 ? mv_kernel<1>(nt) : (r == 2 ? mv_kernel<2>(nt) : mv_kernel<4>(nt));
    cudaError_t e = cudaSuccess;
    if (smem > 47 * 1024) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
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
