// esb_rows.cuh -- typed rows, reductions and the projection with a scale of
// its own for every group, shared by the language-model kernels of libesb
// (esb_groups.cu, esb_matvec.cu, esb_norm.cu, esb_logprobs.cu).
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "esb.h"
#include "esb_common.cuh"

namespace esb {

__host__ __device__ inline int type_bytes(int type) { return type == ESB_F32 ? 4 : 2; }

template <int TYPE> struct ElemOf;
template <> struct ElemOf<ESB_F32> { using T = float; };
template <> struct ElemOf<ESB_F16> { using T = __half; };
template <> struct ElemOf<ESB_BF16> { using T = __nv_bfloat16; };
template <int TYPE> using Elem = typename ElemOf<TYPE>::T;

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Two 16-bit values of a 32-bit word.
template <class T> __device__ __forceinline__ void unpack2(uint32_t w, float& a, float& b);
template <> __device__ __forceinline__ void unpack2<__nv_bfloat16>(uint32_t w, float& a, float& b)
{
    a = __uint_as_float(w << 16);
    b = __uint_as_float(w & 0xffff0000u);
}
template <> __device__ __forceinline__ void unpack2<__half>(uint32_t w, float& a, float& b)
{
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    a = f.x;
    b = f.y;
}
template <class T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b)
{
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b)
{
    const __half2 p = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
}

// Eight consecutive values as fp32, by 16-byte loads.  p is 16-byte aligned.
// Plain loads, not those of read-only memory: a norm may write its row in place.
template <class T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8])
{
    if constexpr (sizeof(T) == 4) {
        const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
        const uint4 a = *reinterpret_cast<const uint4*>(p);
        unpack2<T>(a.x, v[0], v[1]);
        unpack2<T>(a.y, v[2], v[3]);
        unpack2<T>(a.z, v[4], v[5]);
        unpack2<T>(a.w, v[6], v[7]);
    }
}

template <class T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8])
{
    if constexpr (sizeof(T) == 4) {
        reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        *reinterpret_cast<uint4*>(p) =
            make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
    }
}

// The same for the first `n` of eight values (n may be <= 0), one by one
// unless all eight are there and `vec` says that p is 16-byte aligned.
// Values past n read as 0.
template <class T>
__device__ __forceinline__ void load8_to(const T* p, int64_t n, bool vec, float (&v)[8])
{
    if (vec && n >= 8) {
        load8<T>(p, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = i < n ? to_f32(p[i]) : 0.0f;
}

template <class T>
__device__ __forceinline__ void store8_to(T* p, int64_t n, bool vec, const float (&v)[8])
{
    if (vec && n >= 8) {
        store8<T>(p, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; i++)
        if (i < n) p[i] = from_f32<T>(v[i]);
}

// Values of a type that the kernel learns at run time (uniform branches).
__device__ __forceinline__ void load8_any(const void* p, int type, int64_t at, int64_t n, bool vec, float (&v)[8])
{
    if (type == ESB_F32) load8_to(static_cast<const float*>(p) + at, n, vec, v);
    else if (type == ESB_F16) load8_to(static_cast<const __half*>(p) + at, n, vec, v);
    else load8_to(static_cast<const __nv_bfloat16*>(p) + at, n, vec, v);
}
__device__ __forceinline__ void store8_any(void* p, int type, int64_t at, int64_t n, bool vec, const float (&v)[8])
{
    if (type == ESB_F32) store8_to(static_cast<float*>(p) + at, n, vec, v);
    else if (type == ESB_F16) store8_to(static_cast<__half*>(p) + at, n, vec, v);
    else store8_to(static_cast<__nv_bfloat16*>(p) + at, n, vec, v);
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// ------------------------------------------------ projection, own scales

// Projection constants of a format with b = 4 or 8.
struct QuantFmt {
    int k, is_signed, even, linear;   // linear: the set has one spacing
    uint32_t zero_code, rotate;       // added to places, it gives codes (modulo the sign bit)
    float C, Ck, pk, ipk;             // largest value, 2^k times it, 2^k and 2^-k
};

__host__ inline QuantFmt make_quant_fmt(const esb_format& f, int rounding)
{
    const ProjParams p = make_proj_params(f.b, f.k, f.is_signed, rounding);
    QuantFmt q;
    q.k = f.k; q.is_signed = f.is_signed; q.even = rounding;
    q.linear = p.N <= 1;
    q.zero_code = p.zero_code;
    q.rotate = p.zero_code * (f.b == 4 ? 0x11111111u : 0x01010101u);
    q.C = fmt_C(f.b, f.k);
    q.pk = (float)(1 << f.k);
    q.Ck = q.C * q.pk;
    q.ipk = 1.0f / q.pk;
    return q;
}

// A group's scale with what its divisions need.
struct GroupScale {
    float alpha, step, rcp; // step = alpha 2^-k, rcp = 1 / step
    bool fast;              // alpha far from the ends of fp32
};

__device__ __forceinline__ GroupScale make_scale(float alpha, const QuantFmt& f)
{
    GroupScale s;
    s.alpha = alpha;
    s.fast = alpha > 0x1p-60f && alpha < 0x1p60f;
    s.step = alpha * f.ipk;
    s.rcp = s.fast ? __frcp_rn(s.step) : 0.0f;
    return s;
}

// |x| / alpha (max(x, 0) / alpha for the unsigned set) times 2^k, rounded to
// nearest as IEEE division (the power of two is exact).  Many values share
// alpha, so its correctly rounded reciprocal y is found once; q = a y is then
// within two units of a / alpha, one step with the exact remainder makes it
// faithful, and by Markstein's theorem (Computation of elementary functions on
// the IBM RISC System/6000 processor, 1990) a second one rounds it correctly.
// A scale at the ends of fp32, where a remainder could underflow, takes the
// division.
__device__ __forceinline__ float scaled_value(float x, const GroupScale& s, const QuantFmt& f)
{
    const float a = f.is_signed ? fabsf(x) : fmaxf(x, 0.0f);
    if (!s.fast) return __fdiv_rn(a, s.alpha) * f.pk;
    float q = __fmul_rn(a, s.rcp);
    q = __fmaf_rn(__fmaf_rn(-q, s.step, a), s.rcp, q);
    return __fmaf_rn(__fmaf_rn(-q, s.step, a), s.rcp, q);
}

// Eight values to codes: their places in the ascending non-negative set (and
// the sign bits), then the words.  Place j has the code (j - 2^k) mod 2^(b-1),
// so the words take one add and a mask; zero keeps sign 0.  Places are found
// with t = 2^k |x| / alpha: below 2^k (values below 1) the place is t rounded;
// above, the k leading fraction bits are kept, and a carry into the next
// binade is the next place.  q receives the numbers that the codes stand for.
// An alpha of 0 (a group of zeros) or one that is not finite gives zero codes;
// otherwise no value of the group is NaN.
template <int B>
__device__ __forceinline__ void quantise8(const float (&x)[8], const GroupScale& s, const QuantFmt& f, uint32_t (&w)[B / 4], float (&q)[8])
{
    constexpr int PER = 32 / B;
    constexpr uint32_t TOP = B == 4 ? 0x88888888u : 0x80808080u;   // the codes' sign bits
    constexpr uint32_t ONES = B == 4 ? 0x11111111u : 0x01010101u;
    uint32_t S[B / 4];
#pragma unroll
    for (int i = 0; i < B / 4; i++) w[i] = S[i] = 0u;
    const bool dead = !(s.alpha > 0.0f && s.alpha < __int_as_float(0x7f800000));
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const float t = fminf(scaled_value(x[i], s, f), f.Ck);
        uint32_t j;
        float r;
        // rounded to nearest by the addition of 2^23; half away from zero as
        // the floor of t + 1/2, both sums truncated
        const float big = f.even ? __fadd_rn(t, 8388608.0f) : __fadd_rz(__fadd_rz(t, 0.5f), 8388608.0f);
        j = __float_as_uint(big) - 0x4B000000u;
        r = big - 8388608.0f;
        if (!f.linear) {
            const uint32_t u = __float_as_uint(t);
            const int sh = 23 - f.k;
            const uint32_t odd = f.k ? (u >> sh) & 1u : 1u;          // k = 0: the one significant bit
            const uint32_t h = (u + (f.even ? (1u << (sh - 1)) - 1u + odd : 1u << (sh - 1))) >> sh;
            const bool above = t >= f.pk;
            // place 2^k is t = 2^k, whose leading bits are (127 + k) 2^k
            j = above ? h - (((126u + (uint32_t)f.k) << f.k)) : j;
            r = above ? __uint_as_float(h << sh) : r;
        }
        w[i / PER] += j << (B * (i % PER));
        S[i / PER] |= ((__float_as_uint(x[i]) >> 31) & (uint32_t)f.is_signed) << (B * (i % PER) + B - 1);
        r = dead ? 0.0f : r;
        r = s.fast ? __fmul_rn(s.step, r) : __fmul_rn(s.alpha, r * f.ipk);
        q[i] = x[i] < 0.0f ? -r : r;
    }
#pragma unroll
    for (int i = 0; i < B / 4; i++) {
        if (dead) w[i] = 0u;
        const uint32_t nz = (w[i] + (TOP - ONES)) & TOP;
        w[i] = ((w[i] + f.rotate) & ~TOP) | (S[i] & nz);
    }
}

// The words of eight codes of which only the first n are a row's: the rest
// become the zero code.
template <int B>
__device__ __forceinline__ void zero_past(uint32_t (&w)[B / 4], int64_t n, const QuantFmt& f)
{
    constexpr int PER = 32 / B;
    constexpr uint32_t ONES = B == 4 ? 0x11111111u : 0x01010101u;
#pragma unroll
    for (int i = 0; i < B / 4; i++) {
        const int64_t k = n - i * PER;
        if (k >= PER) continue;
        const uint32_t keep = k <= 0 ? 0u : (1u << (B * (int)k)) - 1u;
        w[i] = (w[i] & keep) | ((f.zero_code * ONES) & ~keep);
    }
}

// Magnitude of x that a group's largest value is taken over, as bits: those
// of |x|, or of max(x, 0) for the unsigned set.  They order like the numbers,
// with NaN above infinity, so a NaN in a group becomes its scale.
__device__ __forceinline__ uint32_t magnitude_bits(float x, int is_signed)
{
    const uint32_t u = __float_as_uint(x), a = u & 0x7fffffffu;
    return (is_signed || a > 0x7f800000u || !(u >> 31)) ? a : 0u;
}

}  // namespace esb
