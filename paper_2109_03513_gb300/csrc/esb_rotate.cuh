// esb_rotate.cuh -- the position rotation of heads, shared by the kernels of a
// decoder's attention (esb_headnorm.cu, esb_cache.cu, esb_attention.cu).
//
// A pair (a, b) of a head's values is turned by its position's angle:
//   (a c - b s, b c + a s),  c and s from a table in fp32.
// Pairs are (i, i + dim/2), or neighbours (2 i, 2 i + 1).
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

#include "esb.h"
#include "esb_rows.cuh"

namespace esb {

struct RotArgs {
    const float* table;
    int64_t positions, ld;
    int dim, inter;
    int vec;            // eight values of a head and of the table are whole vectors of one half
};

__host__ inline RotArgs make_rot(const esb_rotation* r, int head_dim)
{
    RotArgs a = {};
    if (!r || r->dim == 0) return a;
    a.table = r->table; a.positions = r->positions; a.ld = r->ld; a.dim = r->dim; a.inter = r->interleaved != 0;
    a.vec = r->dim % 16 == 0 && r->ld % 4 == 0 && (reinterpret_cast<uintptr_t>(r->table) & 15u) == 0 && head_dim % 8 == 0;
    return a;
}

// a c + b s rounded once, but for some 2^-22 of the cases, where it is off by a
// unit in the last place: both products and their sum with their errors.
__device__ __forceinline__ float dot2_rn(float a, float c, float b, float s)
{
    const float p = __fmul_rn(a, c), q = __fmul_rn(b, s);
    const float pe = __fmaf_rn(a, c, -p), qe = __fmaf_rn(b, s, -q);
    const float r = __fadd_rn(p, q), z = __fsub_rn(r, p);
    const float e = __fadd_rn(__fsub_rn(p, __fsub_rn(r, z)), __fsub_rn(q, z));
    return __fadd_rn(r, __fadd_rn(e, __fadd_rn(pe, qe)));
}

__device__ __forceinline__ Pair dot2_rn(const Pair& a, const Pair& c, const Pair& b, const Pair& s)
{
    const Pair minus = pair_of(-1.0f, -1.0f);
    const Pair p = mul2(a, c), q = mul2(b, s);
    const Pair pe = fma2(a, c, mul2(p, minus)), qe = fma2(b, s, mul2(q, minus));
    const Pair r = add2(p, q), z = fma2(p, minus, r);
    const Pair e = add2(fma2(fma2(z, minus, r), minus, p), fma2(z, minus, q));
    return add2(r, add2(e, add2(pe, qe)));
}

// cos and sin of pair j of a position (NaN for a position that the table lacks).
__device__ __forceinline__ void rot_at(const RotArgs& r, int64_t pos, int j, float& c, float& s)
{
    if (pos < 0 || pos >= r.positions) {
        c = s = __int_as_float(0x7fffffff);
        return;
    }
    const float* t = r.table + pos * r.ld;
    c = __ldg(t + j);
    s = __ldg(t + r.dim / 2 + j);
}

// Eight values of a head from d on, rotated.  x: the head's first value, n: its
// values.  Values past the head read as 0.
template <class T>
__device__ __forceinline__ void rotated8(const T* x, int n, int d, bool xvec, const RotArgs& r, int64_t pos, float (&v)[8])
{
    load8_to(x + d, n - d, xvec, v);
    if (d >= r.dim) return;
    const int half = r.dim >> 1;
    if (r.vec && xvec) {
        // one side of the halves, or four whole pairs
        float c[8], s[8];
        const bool in = pos >= 0 && pos < r.positions;
        const float* t = r.table + (in ? pos : 0) * r.ld;
        if (r.inter) {
            const float4 c4 = __ldg(reinterpret_cast<const float4*>(t + d / 2)), s4 = __ldg(reinterpret_cast<const float4*>(t + half + d / 2));
            c[0] = c[1] = c4.x; c[2] = c[3] = c4.y; c[4] = c[5] = c4.z; c[6] = c[7] = c4.w;
            s[1] = s4.x; s[3] = s4.y; s[5] = s4.z; s[7] = s4.w;
            float w[8];
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                w[i] = dot2_rn(v[i], c[i], v[i + 1], -s[i + 1]);
                w[i + 1] = dot2_rn(v[i + 1], c[i], v[i], s[i + 1]);
            }
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = in ? w[i] : __int_as_float(0x7fffffff);
        } else {
            const bool upper = d >= half;
            const int j = upper ? d - half : d;
            float p[8];
            load8<T>(x + (upper ? j : d + half), p);
            const float4 c0 = __ldg(reinterpret_cast<const float4*>(t + j)), c1 = __ldg(reinterpret_cast<const float4*>(t + j + 4));
            const float4 s0 = __ldg(reinterpret_cast<const float4*>(t + half + j)), s1 = __ldg(reinterpret_cast<const float4*>(t + half + j + 4));
            c[0] = c0.x; c[1] = c0.y; c[2] = c0.z; c[3] = c0.w; c[4] = c1.x; c[5] = c1.y; c[6] = c1.z; c[7] = c1.w;
            s[0] = s0.x; s[1] = s0.y; s[2] = s0.z; s[3] = s0.w; s[4] = s1.x; s[5] = s1.y; s[6] = s1.z; s[7] = s1.w;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                v[i] = dot2_rn(v[i], c[i], p[i], upper ? s[i] : -s[i]);
                if (!in) v[i] = __int_as_float(0x7fffffff);
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const int e = d + i;
        if (e >= r.dim || e >= n) continue;
        const bool second = r.inter ? (e & 1) : e >= half;
        const int other = r.inter ? e ^ 1 : (second ? e - half : e + half);
        float c, s;
        rot_at(r, pos, r.inter ? e >> 1 : (second ? e - half : e), c, s);
        v[i] = dot2_rn(v[i], c, to_f32(x[other]), second ? s : -s);
    }
}

}  // namespace esb
