// esb_matvec.cuh -- what the two matrix-vector kernels (esb_matvec.cu,
// esb_matvec_tc.cu) share: arguments, the decoding of 4-bit codes to fp16, and
// the preparation of the rows of x.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

#include "esb_internal.h"
#include "esb_rows.cuh"

namespace esb {

// fp16 high bytes of the elements by the code's low 3 bits; 2^16 and 2^4.
struct MvTable {
    uint32_t lo, hi, by16, by4;
};

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
    MvTable tab;
    int x_type, y_type, xvec;
    uint32_t gmagic;                // 2^32 / (group / 32) rounded up, 0 for groups of 32
    int mt, planes;                 // rows of x in a block, planes of each
    int kc;                         // codes of a row in a block (a multiple of 512)
    int zrow;                       // whether some lanes read zeros in place of x
    int64_t row_codes;              // codes of a row of the matrix that are read (mv_row_codes)
    int wk;                         // warps along a row (the others take other tiles)
    int split;                      // blocks along a row (a cluster)
    int hold;                       // tiles whose sums wait for one barrier
};

// Eight codes as four fp16 pairs {0,2} {1,3} {4,6} {5,7}: the order in which
// a word's sign bits lie at the top of alternate bytes.  The two shifts are
// products with powers of two that the compiler does not know: they go to the
// multiply-add pipe, the other eleven instructions to the ALU pipe, which is
// the busier one (55% of its cycles in 1 x 65536 x 4096, the other 11%).
__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t sel)
{
    uint32_t r;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(sel));
    return r;
}
__device__ __forceinline__ void decode8(uint32_t w, const MvTable& tb, uint32_t (&p)[4])
{
    const uint32_t sel = w & 0x77777777u;
    const uint32_t m03 = prmt(tb.lo, tb.hi, sel), m47 = prmt(tb.lo, tb.hi, __umulhi(sel, tb.by16));
    const uint32_t odd = prmt(m03, m47, 0x7531u) | (w & 0x80808080u);
    const uint32_t even = prmt(m03, m47, 0x6420u) | ((w * tb.by4) & 0x80808080u);
    p[0] = prmt(even, 0u, 0x1404u);
    p[1] = prmt(odd, 0u, 0x1404u);
    p[2] = prmt(even, 0u, 0x3424u);
    p[3] = prmt(odd, 0u, 0x3424u);
}

__device__ __forceinline__ uint32_t half2_of(float a, float b) { return pack2<__half>(a, b); }

// Eight values of row m of x, the b-th eight: scaled, split into planes, in
// pair order, to where the kernel keeps a plane's eights and a step's scales.
// All 32 lanes take part.
template <int R, int TYPE, class Where>
__device__ __forceinline__ void put_x8(const Where& where, float (&v)[8], int m, int b)
{
    const int i = b & 15;
    constexpr int LANES = 16 / R;                       // lanes that share a scale
    float back = 1.0f;
    if constexpr (TYPE != ESB_F16) {
        uint32_t mx = 0u;
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const uint32_t u = __float_as_uint(v[j]) & 0x7fffffffu;
            mx = max(mx, u < 0x7f800000u ? u : 0u);
        }
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        const int e = max((int)(mx >> 23), 15);         // exponent field; 2^(14 - (e - 127)) <= 2^126
        const float s = __uint_as_float((uint32_t)(268 - e) << 23);
        back = __uint_as_float((uint32_t)(e - 14) << 23);
#pragma unroll
        for (int j = 0; j < 8; j++) v[j] *= s;
    }
    if constexpr (TYPE == ESB_F32) {
        float lo[8];
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const float hi = __half2float(__float2half_rn(v[j]));
            lo[j] = fabsf(hi) < __int_as_float(0x7f800000) ? (v[j] - hi) * 2048.0f : 0.0f;
            v[j] = hi;
        }
        *where.values(2 * m + 1, b) = make_uint4(half2_of(lo[0], lo[2]), half2_of(lo[1], lo[3]), half2_of(lo[4], lo[6]), half2_of(lo[5], lo[7]));
        if (i % LANES == 0) *where.scale(2 * m + 1, b >> 4, i / LANES) = back * (1.0f / 2048.0f);
    }
    const int row = TYPE == ESB_F32 ? 2 * m : m;
    *where.values(row, b) = make_uint4(half2_of(v[0], v[2]), half2_of(v[1], v[3]), half2_of(v[4], v[6]), half2_of(v[5], v[7]));
    if (i % LANES == 0) *where.scale(row, b >> 4, i / LANES) = back;
}

// Rows m0 .. m0 + mt - 1 of x, codes k0 .. k0 + kc - 1, into shared memory: a
// warp takes 256 values of a row at a time, several such parts in flight.
template <int R, int TYPE, class Where>
__device__ __forceinline__ void stage_x_of(const MvArgs& a, int64_t m0, int mt, int64_t k0, const Where& where, const uint16_t* xtab, int warps, int warp)
{
    constexpr int U = TYPE == ESB_F32 ? 4 : 8, WORDS = TYPE == ESB_F32 ? 8 : (TYPE == ESB_CODES ? 2 : 4);
    const int parts = a.kc / 256, total = mt * parts;
    const int lane = threadIdx.x & 31, i = lane & 15;
    for (int q0 = warp; q0 < total; q0 += U * warps) {
        uint32_t raw[U][WORDS];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int q = q0 + u * warps;
            if (q >= total) break;
            const int m = q / parts;
            const int64_t k = k0 + (q - m * parts) * 256 + lane * 8, n = a.K - k;
            if constexpr (TYPE == ESB_CODES) {
                const uint32_t* xw = a.xc.codes + (m0 + m) * a.xc.ld + k / 4;
                raw[u][0] = n > 0 ? __ldg(xw) : 0u;
                raw[u][1] = n > 4 ? __ldg(xw + 1) : 0u;
            } else {
                using T = Elem<TYPE>;
                const T* p = static_cast<const T*>(a.x) + (m0 + m) * a.ldx + k;
                if (a.xvec && n >= 8) {
#pragma unroll
                    for (int j = 0; j < WORDS; j += 4) {
                        const uint4 v = __ldg(reinterpret_cast<const uint4*>(p) + j / 4);
                        raw[u][j] = v.x; raw[u][j + 1] = v.y; raw[u][j + 2] = v.z; raw[u][j + 3] = v.w;
                    }
                } else if constexpr (TYPE == ESB_F32) {
#pragma unroll
                    for (int j = 0; j < 8; j++) raw[u][j] = j < n ? __float_as_uint(p[j]) : 0u;
                } else {
                    const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
                    for (int j = 0; j < 4; j++)
                        raw[u][j] = (2 * j < n ? h[2 * j] : 0u) | ((2 * j + 1 < n ? (uint32_t)h[2 * j + 1] : 0u) << 16);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int q = q0 + u * warps;
            if (q >= total) break;
            const int m = q / parts, b = (q - m * parts) * 32 + lane;
            if constexpr (TYPE == ESB_CODES) {
                const int64_t k = k0 + (int64_t)b * 8, n = a.K - k;
                uint32_t h[8];
#pragma unroll
                for (int j = 0; j < 8; j++) h[j] = j < n ? xtab[(raw[u][j >> 2] >> (8 * (j & 3))) & 255u] : 0u;
                *where.values(m, b) = make_uint4(h[0] | (h[2] << 16), h[1] | (h[3] << 16), h[4] | (h[6] << 16), h[5] | (h[7] << 16));
                if (i % (16 / R) == 0)
                    *where.scale(m, b >> 4, i / (16 / R)) = n > 0 ? a.xc.scales[(m0 + m) * a.xc.lds + k / a.xgroup] * (a.xc.fmt.k == 2 ? 65536.0f : 1.0f) : 0.0f;
            } else {
                float v[8];
                if constexpr (TYPE == ESB_F32) {
#pragma unroll
                    for (int j = 0; j < 8; j++) v[j] = __uint_as_float(raw[u][j]);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; j++) unpack2<Elem<TYPE>>(raw[u][j], v[2 * j], v[2 * j + 1]);
                }
                put_x8<R, TYPE>(where, v, m, b);
            }
        }
    }
}

// By the type of x, by warp `warp` of `warps`.
template <int R, class Where>
__device__ __forceinline__ void stage_x(const MvArgs& a, int64_t m0, int mt, int64_t k0, const Where& where, const uint16_t* xtab, int warps, int warp)
{
    if (a.x_type == ESB_BF16) stage_x_of<R, ESB_BF16>(a, m0, mt, k0, where, xtab, warps, warp);
    else if (a.x_type == ESB_CODES) stage_x_of<R, ESB_CODES>(a, m0, mt, k0, where, xtab, warps, warp);
    else if (a.x_type == ESB_F16) stage_x_of<R, ESB_F16>(a, m0, mt, k0, where, xtab, warps, warp);
    else stage_x_of<R, ESB_F32>(a, m0, mt, k0, where, xtab, warps, warp);
}

// fp16 images of the 8-bit codes: k = 2 reaches 1.75 * 2^30, so its elements
// are scaled by 2^-16 (and their rows' scales by 2^16).
__device__ __forceinline__ uint16_t x_code_half(int code, int k)
{
    const __half h = __float2half_rn(code_value(code, 8, k) * (k == 2 ? 1.0f / 65536.0f : 1.0f));
    return *reinterpret_cast<const uint16_t*>(&h);
}

// A result to y.
__device__ __forceinline__ void put_y(const MvArgs& a, int64_t m, int n, float v)
{
    if (a.bias) v += a.bias[n];
    const int64_t at = m * a.ldy + n;
    if (a.y_type == ESB_F32) static_cast<float*>(a.y)[at] = v;
    else if (a.y_type == ESB_F16) static_cast<__half*>(a.y)[at] = __float2half_rn(v);
    else static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v);
}

// The tcgen05 kernel (esb_matvec_tc.cu) where it takes the call: false if it
// does not.  r: groups of a step of 128 codes.
bool launch_matvec_tc(const MvArgs& args, int r, cudaStream_t st, cudaError_t* err);

}  // namespace esb
