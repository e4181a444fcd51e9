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

// What is left of `cols` values from place e on, as a count of a few of them.
__device__ __forceinline__ int left_of(int64_t cols, int64_t e)
{
    const int64_t n = cols - e;
    return n > 64 ? 64 : (n < 0 ? 0 : (int)n);
}

// The same for the first `n` of eight values (n may be <= 0), one by one
// unless all eight are there and `vec` says that p is 16-byte aligned.
// Values past n read as 0.
template <class T>
__device__ __forceinline__ void load8_to(const T* p, int n, bool vec, float (&v)[8])
{
    if (vec && n >= 8) {
        load8<T>(p, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = i < n ? to_f32(p[i]) : 0.0f;
}

template <class T>
__device__ __forceinline__ void store8_to(T* p, int n, bool vec, const float (&v)[8])
{
    if (vec && n >= 8) {
        store8<T>(p, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; i++)
        if (i < n) p[i] = from_f32<T>(v[i]);
}

// Eight consecutive values as they lie in memory: loads that are waiting take
// half the registers of fp32 values.
template <class T>
struct Raw8 {
    uint32_t w[2 * sizeof(T)];
    __device__ __forceinline__ void load(const T* p, int n, bool vec)
    {
        if (vec && n >= 8) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; i++) {
                const uint4 v = reinterpret_cast<const uint4*>(p)[i];
                w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
            }
        } else if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 8; i++) w[i] = i < n ? __float_as_uint(p[i]) : 0u;
        } else {
            const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
            for (int i = 0; i < 4; i++) w[i] = (2 * i < n ? h[2 * i] : 0u) | ((2 * i + 1 < n ? (uint32_t)h[2 * i + 1] : 0u) << 16);
        }
    }
    __device__ __forceinline__ void values(float (&v)[8]) const
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = __uint_as_float(w[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++) unpack2<T>(w[i], v[2 * i], v[2 * i + 1]);
        }
    }
};

// Values of a type that the kernel learns at run time (uniform branches).
__device__ __forceinline__ void load8_any(const void* p, int type, int64_t at, int n, bool vec, float (&v)[8])
{
    if (type == ESB_F32) load8_to(static_cast<const float*>(p) + at, n, vec, v);
    else if (type == ESB_F16) load8_to(static_cast<const __half*>(p) + at, n, vec, v);
    else load8_to(static_cast<const __nv_bfloat16*>(p) + at, n, vec, v);
}
__device__ __forceinline__ void store8_any(void* p, int type, int64_t at, int n, bool vec, const float (&v)[8])
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

// Two fp32 numbers in one instruction of the multiply-add pipe.
struct Pair {
    unsigned long long v;
};
__device__ __forceinline__ Pair pair_of(float a, float b)
{
    Pair p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p.v) : "f"(a), "f"(b));
    return p;
}
__device__ __forceinline__ void split(const Pair& p, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p.v)); }
__device__ __forceinline__ Pair add2(const Pair& a, const Pair& b)
{
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Pair mul2(const Pair& a, const Pair& b)
{
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Pair fma2(const Pair& a, const Pair& b, const Pair& c)
{
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ Pair add2_rz(const Pair& a, const Pair& b)
{
    Pair r;
    asm("add.rz.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}

// ------------------------------------------------ projection, own scales

// Projection constants of a format with b = 4 or 8.
struct QuantFmt {
    int k, is_signed, even;
    int linear, plain;                // the set has one spacing; signed with ties away from zero
    uint32_t zero_code, rotate;       // added to places, it gives codes (modulo the sign bit)
    float C, rC, Ck, pk, ipk;         // largest value, its rounded reciprocal, 2^k times it, 2^k and 2^-k
};

__host__ inline QuantFmt make_quant_fmt(const esb_format& f, int rounding)
{
    const ProjParams p = make_proj_params(f.b, f.k, f.is_signed, rounding);
    QuantFmt q;
    q.k = f.k; q.is_signed = f.is_signed; q.even = rounding;
    q.linear = p.N <= 1;
    q.plain = f.is_signed && rounding == ESB_ROUND_HALF_AWAY;
    q.zero_code = p.zero_code;
    q.rotate = p.zero_code * (f.b == 4 ? 0x11111111u : 0x01010101u);
    q.C = fmt_C(f.b, f.k);
    q.rC = 1.0f / q.C;
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

// The scale of a group with this largest magnitude: it over C, rounded to
// nearest (in the middle of fp32's range as fast_quotients below).
__device__ __forceinline__ float absmax_scale(uint32_t mx, const QuantFmt& f)
{
    const float a = __uint_as_float(mx);
    if (!(a > 0x1p-60f && a < 0x1p60f) || f.C > 0x1p60f) return __fdiv_rn(a, f.C);
    float q = __fmul_rn(a, f.rC);
    q = __fmaf_rn(__fmaf_rn(-q, f.C, a), f.rC, q);
    return __fmaf_rn(__fmaf_rn(-q, f.C, a), f.rC, q);
}

// 2^k |x| / alpha for two values, rounded to nearest as IEEE division of |x|
// by alpha (the power of two is exact).  Many values share alpha, so the
// correctly rounded reciprocal y of the step is found once; q = a y is then
// within two units of the quotient, one step with the exact remainder makes it
// faithful, and by Markstein's theorem (Computation of elementary functions on
// the IBM RISC System/6000 processor, 1990) a second one rounds it correctly.
__device__ __forceinline__ Pair fast_quotients(const Pair& a, const Pair& rcp, const Pair& minus_step)
{
    Pair q = mul2(a, rcp);
    q = fma2(fma2(q, minus_step, a), rcp, q);
    return fma2(fma2(q, minus_step, a), rcp, q);
}

// t = 2^k |x| / alpha on the set: r receives the element (times 2^k), the
// return value its place among the non-negative elements.  Places are t
// rounded below 2^k (values below 1); above, the k leading fraction bits are
// kept, and a carry into the next binade is the next place.
__device__ __forceinline__ uint32_t round_away(float t, bool linear, int k, float pk, float& r)
{
    // half away from zero as the floor of t + 1/2, both sums truncated
    const float big = __fadd_rz(__fadd_rz(t, 0.5f), 8388608.0f);
    uint32_t j = __float_as_uint(big) - 0x4B000000u;
    r = big - 8388608.0f;
    if (!linear) {
        const int sh = 23 - k;
        const uint32_t h = (__float_as_uint(t) + (1u << (sh - 1))) >> sh;
        const bool above = t >= pk;
        // place 2^k is t = 2^k, whose leading bits are (127 + k) 2^k
        j = above ? h - ((126u + (uint32_t)k) << k) : j;
        r = above ? __uint_as_float(h << sh) : r;
    }
    return j;
}

// The general case of one value: unsigned sets, the other tie rule, scales at
// the ends of fp32 (where a remainder could underflow) by division, and groups
// whose scale is 0 or not finite, which have zero codes.
static __device__ __noinline__ uint2 place_any(float x, float alpha, const QuantFmt& f)
{
    float r = 0.0f;
    if (!(alpha > 0.0f && alpha < __int_as_float(0x7f800000))) return make_uint2(0u, 0u);
    const float a = f.is_signed ? fabsf(x) : fmaxf(x, 0.0f);
    const float t = fminf(__fdiv_rn(a, alpha) * f.pk, f.Ck);
    if (!f.even) {
        const uint32_t j = round_away(t, f.linear, f.k, f.pk, r);
        return make_uint2(j, __float_as_uint(r));
    }
    if (f.linear || t < f.pk) {
        const float big = __fadd_rn(t, 8388608.0f);
        return make_uint2(__float_as_uint(big) - 0x4B000000u, __float_as_uint(big - 8388608.0f));
    }
    const int sh = 23 - f.k;
    const uint32_t u = __float_as_uint(t), odd = f.k ? (u >> sh) & 1u : 1u;   // k = 0: the one significant bit
    const uint32_t h = (u + (1u << (sh - 1)) - 1u + odd) >> sh;
    return make_uint2(h - ((126u + (uint32_t)f.k) << f.k), h << sh);
}

// Eight values to codes: their places (a nibble or byte each) and sign bits,
// then the words.  Place j has the code (j - 2^k) mod 2^(b-1), so a word takes
// one add and a mask; zero keeps sign 0.  r receives the elements' magnitudes
// times 2^k (element_values turns them into numbers).  In a group with a
// finite scale no value is NaN.
// CLAMP: quotients may be past the largest element.  (Under a group's own
// absmax scale they pass it by a unit in the last place at most, which the
// rounding to the set takes back.)  MAG: x are magnitudes.
template <int B, bool LINEAR, bool CLAMP, bool MAG = false>
__device__ __forceinline__ void places8(const float (&x)[8], const GroupScale& s, const QuantFmt& f, uint32_t (&w)[B / 4], float (&r)[8])
{
    constexpr int PER = 32 / B;
    constexpr uint32_t ONES = B == 4 ? 0x11111111u : 0x01010101u;
    const Pair rcp = pair_of(s.rcp, s.rcp), minus_step = pair_of(-s.step, -s.step);
    const Pair half = pair_of(0.5f, 0.5f), whole = pair_of(8388608.0f, 8388608.0f), minus_whole = pair_of(-8388608.0f, -8388608.0f);
#pragma unroll
    for (int i = 0; i < B / 4; i++) w[i] = LINEAR ? 0u - 0x4B000000u * ONES : 0u;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        Pair t = fast_quotients(MAG ? pair_of(x[i], x[i + 1]) : pair_of(fabsf(x[i]), fabsf(x[i + 1])), rcp, minus_step);
        float t0, t1;
        if constexpr (CLAMP || !LINEAR) split(t, t0, t1);
        if constexpr (CLAMP) {
            t0 = fminf(t0, f.Ck);
            t1 = fminf(t1, f.Ck);
            t = pair_of(t0, t1);
        }
        if constexpr (LINEAR) {
            // the place is the low bits of the sum; what lies above them is
            // taken off the word at once
            const Pair big = add2_rz(add2_rz(t, half), whole);
            split(big, t0, t1);
            w[i / PER] += __float_as_uint(t0) * (1u << (B * (i % PER)));
            w[i / PER] += __float_as_uint(t1) * (1u << (B * (i % PER + 1)));
            split(add2(big, minus_whole), r[i], r[i + 1]);
        } else {
            w[i / PER] += round_away(t0, false, f.k, f.pk, r[i]) << (B * (i % PER));
            w[i / PER] += round_away(t1, false, f.k, f.pk, r[i + 1]) << (B * (i % PER + 1));
        }
    }
}
// The sign bits of eight values at the tops of their codes.
template <int B>
__device__ __forceinline__ void signs8(const float (&x)[8], uint32_t (&S)[B / 4])
{
    uint32_t u[8];
#pragma unroll
    for (int i = 0; i < 8; i++) u[i] = __float_as_uint(x[i]);
    auto tops = [&](int a, int b, int c, int d) {       // the values' top bytes
        return __byte_perm(__byte_perm(u[a], u[b], 0x0073), __byte_perm(u[c], u[d], 0x0073), 0x5410) & 0x80808080u;
    };
    if constexpr (B == 8) {
        S[0] = tops(0, 1, 2, 3);
        S[1] = tops(4, 5, 6, 7);
    } else {
        S[0] = tops(1, 3, 5, 7) | (tops(0, 2, 4, 6) >> 4);
    }
}
// The same from four pairs of 16-bit numbers.
template <int B>
__device__ __forceinline__ void signs8(const uint32_t (&x)[4], uint32_t (&S)[B / 4])
{
    if constexpr (B == 8) {
        S[0] = __byte_perm(x[0], x[1], 0x7531) & 0x80808080u;
        S[1] = __byte_perm(x[2], x[3], 0x7531) & 0x80808080u;
    } else {
        const uint32_t a = __byte_perm(x[0], x[1], 0x7351), b = __byte_perm(x[2], x[3], 0x7351);
        S[0] = (__byte_perm(a, b, 0x7632) & 0x80808080u) | ((__byte_perm(a, b, 0x5410) & 0x80808080u) >> 4);
    }
}
// Places to codes, with the signs of x (eight numbers, or four pairs of 16 bits).
template <int B, class X>
__device__ __forceinline__ void codes8(const X& x, const QuantFmt& f, uint32_t (&w)[B / 4])
{
    constexpr uint32_t TOP = B == 4 ? 0x88888888u : 0x80808080u;   // the codes' sign bits
    constexpr uint32_t ONES = B == 4 ? 0x11111111u : 0x01010101u;
    uint32_t S[B / 4];
    signs8<B>(x, S);
#pragma unroll
    for (int i = 0; i < B / 4; i++) {
        const uint32_t nz = (w[i] + (TOP - ONES)) & TOP;
        w[i] = ((w[i] + f.rotate) & ~TOP) | (S[i] & nz);
    }
}
template <int B, bool CLAMP>
__device__ __forceinline__ void quantise8(const float (&x)[8], const GroupScale& s, const QuantFmt& f, uint32_t (&w)[B / 4], float (&r)[8])
{
    constexpr int PER = 32 / B;
    if (s.fast && f.plain) {
        if (f.linear) places8<B, true, CLAMP>(x, s, f, w, r);
        else places8<B, false, CLAMP>(x, s, f, w, r);
    } else {
#pragma unroll
        for (int i = 0; i < B / 4; i++) w[i] = 0u;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const uint2 p = place_any(x[i], s.alpha, f);
            w[i / PER] += p.x << (B * (i % PER));
            r[i] = __uint_as_float(p.y);
        }
    }
    codes8<B>(x, f, w);
}

// The numbers that the codes of x stand for, alpha q, from r.
__device__ __forceinline__ void element_values(const float (&x)[8], const GroupScale& s, const QuantFmt& f, float (&r)[8])
{
    const float by = s.fast ? s.step : s.alpha;
    if (!s.fast) {
#pragma unroll
        for (int i = 0; i < 8; i++) r[i] *= f.ipk;
    }
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        split(mul2(pair_of(by, by), pair_of(r[i], r[i + 1])), r[i], r[i + 1]);
        r[i] = __uint_as_float(__float_as_uint(r[i]) ^ (__float_as_uint(x[i]) & 0x80000000u));
        r[i + 1] = __uint_as_float(__float_as_uint(r[i + 1]) ^ (__float_as_uint(x[i + 1]) & 0x80000000u));
    }
}

// The words of eight codes of which only the first n are a row's: the rest
// become the zero code.
template <int B>
__device__ __forceinline__ void zero_past(uint32_t (&w)[B / 4], int n, const QuantFmt& f)
{
    constexpr int PER = 32 / B;
    constexpr uint32_t ONES = B == 4 ? 0x11111111u : 0x01010101u;
#pragma unroll
    for (int i = 0; i < B / 4; i++) {
        const int k = n - i * PER;
        if (k >= PER) continue;
        const uint32_t keep = k <= 0 ? 0u : (1u << (B * k)) - 1u;
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
// The largest magnitude_bits of eight values, up to NaN's bits: the maximum
// of three numbers is one instruction, and NaN where one of them is.
__device__ __forceinline__ float max_nan(float a, float b, float c)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float max_nan_abs(float a, float b, float c)
{
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ uint32_t largest_of8(const float (&v)[8], int is_signed)
{
    float m = 0.0f;
    if (is_signed) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) m = max_nan_abs(m, v[i], v[i + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i += 2) m = max_nan(m, v[i], v[i + 1]);
    }
    return __float_as_uint(m) & 0x7fffffffu;
}

}  // namespace esb
