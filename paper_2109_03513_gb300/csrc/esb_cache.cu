// esb_cache.cu -- keys (rotated by their positions) and values of new tokens
// onto 4-bit ESB codes with a scale for each token and head, into the pages of
// a cache.
//
// A lane holds 16 values of a head, two words of codes; a head's lanes (8 for 128
// values) find its largest magnitude or its spread together.
// The rotated key is rounded once to fp32 (both products and their sum carry
// their errors), so that its code is that of the exact rotation: on a set of
// 15 values a last place is a step of the set now and then.
#include <algorithm>
#include <cstdint>
#include <cuda_runtime.h>

#include "esb_internal.h"
#include "esb_heads.cuh"

namespace esb {

namespace {

constexpr int kApThreads = 256;

struct AppendSide {
    const void* x;
    int64_t ldx;
    uint32_t* codes;
    float* scales;
    void* q;                            // the values, or NULL
    int64_t ldq;
    float astar;
    int xvec, qvec;
    QuantFmt f;
};

struct AppendArgs {
    AppendSide side[2];                 // keys, values
    const int64_t *slots, *positions;
    int64_t tokens, places, page_ld, page_lds;
    int heads, page_size, D, words, q_type, rule, tvec;
    RotArgs rot;
    HeadWork work;
};

// The scale of a head's 16 values in each of L lanes (the rest of them 0).
template <int L>
__device__ __forceinline__ float scale_of(const AppendArgs& a, const AppendSide& s, const float (&u)[8], const float (&v)[8], int left_u, int left_v)
{
    if (a.rule == ESB_SCALE_ABSMAX) {
        uint32_t mx = max(largest_of8(u, 1), largest_of8(v, 1));
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        return absmax_scale(mx, s.f);
    }
    auto total = [&](float x) {
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        return x;
    };
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; i++) s1 += u[i] + v[i];
    const float mean = total(s1) / (float)a.D;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const float x = i < left_u ? u[i] - mean : 0.0f, y = i < left_v ? v[i] - mean : 0.0f;
        s2 = fmaf(x, x, fmaf(y, y, s2));
    }
    return __fmul_rn(s.astar, __fadd_rn(__fsqrt_rn(total(s2) / (float)a.D), 1e-7f));
}

// Heads of whole vectors: a lane holds 8 pairs of a key as the rotation pairs
// them, or 16 of a value's numbers, the next head's ahead; a warp keeps a
// token's cos and sin for several heads.
template <int TYPE, int L>
__global__ void __launch_bounds__(kApThreads, TYPE == ESB_F32 ? 2 : 3) append_pairs_kernel(const AppendArgs a)
{
    using T = Elem<TYPE>;
    griddep_wait();
    RotArgs none = {};
    const int j0 = (threadIdx.x % L) * 8;
    const PairPlace pk(j0, a.D / 2, a.rot), pv(j0, a.D / 2, none);
    float c[8], sn[8];
    HeadWalk<L, kApThreads / 32> at = {}, to = {};
    RawPairs<T, true> next;
    int64_t next_slot = -1, next_pos = 0, slot, pos;
    auto load = [&]() {
        const AppendSide& s = a.side[to.part];
        if (to.it == 0) {
            next_slot = to.token < a.work.tokens && to.on ? __ldg(a.slots + to.token) : -1;
            next_pos = a.rot.dim && to.part == 0 && to.on ? __ldg(a.positions + to.token) : 0;
        }
        const T* x = static_cast<const T*>(s.x) + (to.on ? to.token * s.ldx + (int64_t)to.head * a.D : 0);
        if (to.part) next.load(x, pv, none, to.on);
        else next.load(x, pk, a.rot, to.on);
    };
    to.start(a.work);
    load();
    at = to;
    while (at.more(a.work)) {
        const RawPairs<T, true> raw = next;
        slot = next_slot;
        pos = next_pos;
        to.next(a.work);
        load();
        const bool key = at.part == 0;
        if (at.it == 0 && key && a.rot.dim) load_turn(a.rot, a.tvec, pk, pos, c, sn);
        const bool on = at.on && slot >= 0 && slot < a.places;
        const bool rows = key ? pk.rows : true;
        float u[8], v[8];
        if (key) {
            raw.values(pk, u, v);
            if (a.rot.dim && pk.j0 < pk.half) {
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const float x = u[i];
                    u[i] = dot2_rn(x, c[i], v[i], -sn[i]);
                    v[i] = dot2_rn(v[i], c[i], x, sn[i]);
                }
            }
            if (pk.rows) {
                float x[8], y[8];
#pragma unroll
                for (int i = 0; i < 8; i++) { x[i] = u[i]; y[i] = v[i]; }
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    u[i] = (i & 1) ? y[i / 2] : x[i / 2];
                    v[i] = (i & 1) ? y[4 + i / 2] : x[4 + i / 2];
                }
            }
        } else {
            raw.u.values(u);
            raw.w.values(v);
        }
        const AppendSide& s = a.side[at.part];
        const int there = pv.count > 0 ? 8 : 0;
        const float alpha = scale_of<L>(a, s, u, v, there, there);
        if (on) {
            const int64_t page = slot / a.page_size;
            const int place = (int)(slot - page * a.page_size);
            if (j0 == 0) s.scales[page * a.page_lds + (int64_t)at.head * a.page_size + place] = alpha;
            const GroupScale g = make_scale(alpha, s.f);
            uint32_t w0[1], w1[1];
            float q0[8], q1[8];
            quantise8<4, true>(u, g, s.f, w0, q0);
            quantise8<4, true>(v, g, s.f, w1, q1);
            uint32_t* codes = s.codes + page * a.page_ld + ((int64_t)at.head * a.page_size + place) * a.words;
            const int d0 = rows ? 2 * j0 : j0, d1 = rows ? d0 + 8 : j0 + pk.half;
            if (pv.count > 0) {
                if (rows) *reinterpret_cast<uint2*>(codes + d0 / 8) = make_uint2(w0[0], w1[0]);
                else { codes[d0 / 8] = w0[0]; codes[d1 / 8] = w1[0]; }
                if (s.q) {
                    element_values(u, g, s.f, q0);
                    element_values(v, g, s.f, q1);
                    const int64_t row = at.token * s.ldq + (int64_t)at.head * a.D;
                    store8_any(s.q, a.q_type, row + d0, 8, s.qvec, q0);
                    store8_any(s.q, a.q_type, row + d1, 8, s.qvec, q1);
                }
            } else if (2 * j0 < a.words * 8) {              // the words behind the values
                const uint32_t z = s.f.zero_code * 0x11111111u;
                *reinterpret_cast<uint2*>(codes + j0 / 4) = make_uint2(z, z);
            }
        }
        at = to;
    }
}

// Any heads: a lane holds 16 consecutive values, and reads a pair's other half again.
template <int TYPE, int L>
__global__ void __launch_bounds__(kApThreads) append_kernel(const AppendArgs a)
{
    using T = Elem<TYPE>;
    griddep_wait();
    const int part = threadIdx.x % L, per = 2 * a.heads;
    const int64_t rows = a.tokens * per, step = (int64_t)gridDim.x * (kApThreads / L);
    for (int64_t r = (int64_t)blockIdx.x * (kApThreads / L) + threadIdx.x / L; __any_sync(0xffffffffu, r < rows); r += step) {
        const int64_t token = r < rows ? r / per : 0;
        const int h = r < rows ? (int)(r - token * per) : 0;
        const bool value = h >= a.heads;
        const int head = value ? h - a.heads : h;
        const AppendSide& s = a.side[value];
        const int64_t slot = r < rows ? __ldg(a.slots + token) : -1;
        const bool on = slot >= 0 && slot < a.places;
        const int d0 = part * 16, n = on ? a.D : 0;
        const T* x = static_cast<const T*>(s.x) + (on ? token * s.ldx + (int64_t)head * a.D : 0);
        float v[2][8];
        const int64_t pos = on && !value && a.rot.dim ? __ldg(a.positions + token) : 0;
#pragma unroll
        for (int i = 0; i < 2; i++) {
            if (on && !value && a.rot.dim && d0 + 8 * i < a.D) rotated8<T>(x, n, d0 + 8 * i, s.xvec, a.rot, pos, v[i]);
            else load8_to(x + d0 + 8 * i, n - d0 - 8 * i, s.xvec, v[i]);
        }
        const float alpha = scale_of<L>(a, s, v[0], v[1], a.D - d0, a.D - d0 - 8);
        if (!on) continue;
        const int64_t page = slot / a.page_size;
        const int place = (int)(slot - page * a.page_size);
        if (part == 0) s.scales[page * a.page_lds + (int64_t)head * a.page_size + place] = alpha;
        if (part * 2 >= a.words) continue;
        const GroupScale g = make_scale(alpha, s.f);
        uint32_t w[2];
#pragma unroll
        for (int i = 0; i < 2; i++) {
            uint32_t word[1];
            float q[8];
            quantise8<4, true>(v[i], g, s.f, word, q);
            const int left = a.D - d0 - 8 * i;
            if (left < 8) zero_past<4>(word, left, s.f);
            w[i] = word[0];
            if (s.q && left > 0) {
                element_values(v[i], g, s.f, q);
                store8_any(s.q, a.q_type, token * s.ldq + (int64_t)head * a.D + d0 + 8 * i, left, s.qvec, q);
            }
        }
        uint32_t* to = s.codes + page * a.page_ld + ((int64_t)head * a.page_size + place) * a.words + part * 2;
        *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
    }
}

using ApKernel = void (*)(const AppendArgs);
template <int TYPE> ApKernel append_of(int L, bool pairs)
{
    switch (L) {
    case 4: return pairs ? append_pairs_kernel<TYPE, 4> : append_kernel<TYPE, 4>;
    case 8: return pairs ? append_pairs_kernel<TYPE, 8> : append_kernel<TYPE, 8>;
    default: return pairs ? append_pairs_kernel<TYPE, 16> : append_kernel<TYPE, 16>;
    }
}

}  // namespace

cudaError_t launch_cache_append(int64_t tokens, const esb_kv_cache& c, const esb_append& n, double alpha_star_k, double alpha_star_v,
                                cudaStream_t st)
{
    AppendArgs a = {};
    for (int i = 0; i < 2; i++) {
        AppendSide& s = a.side[i];
        s.x = i ? n.v : n.k; s.ldx = i ? n.ldv : n.ldk;
        s.codes = i ? c.v_codes : c.k_codes; s.scales = i ? c.v_scales : c.k_scales;
        s.q = i ? n.vq : n.kq; s.ldq = i ? n.ldvq : n.ldkq;
        s.astar = (float)(i ? alpha_star_v : alpha_star_k);
        s.xvec = rows16(s.x, s.ldx, n.x_type);
        s.qvec = s.q && rows16(s.q, s.ldq, n.q_type);
        s.f = make_quant_fmt(i ? c.v_fmt : c.k_fmt, n.rounding);
    }
    a.slots = n.slots; a.positions = n.positions; a.tokens = tokens; a.places = c.pages * c.page_size;
    a.page_ld = c.page_ld; a.page_lds = c.page_lds;
    a.heads = c.heads; a.page_size = c.page_size; a.D = c.head_dim; a.words = (c.head_dim + 31) / 32 * 4;
    a.q_type = n.q_type; a.rule = n.rule; a.rot = make_rot(n.rotation, c.head_dim);
    a.tvec = a.rot.vec;
    const int L = lanes_of(a.D);
    static ApKernel (*const pick[3])(int, bool) = {append_of<ESB_F32>, append_of<ESB_F16>, append_of<ESB_BF16>};
    const bool pairs = pairs_of_vectors(a.D, a.rot.dim, a.rot.inter) && a.side[0].xvec && a.side[1].xvec;
    int64_t blocks;
    if (pairs) {
        const int64_t most = (int64_t)device_sm_count() * (n.x_type == ESB_F32 ? 2 : 3), warps = kApThreads / 32;
        a.work = split_heads(tokens, c.heads, c.heads, L, most * warps);
        blocks = std::min((a.work.part[0].items + a.work.part[1].items + warps - 1) / warps, most);
    } else {
        const int64_t per = kApThreads / L;
        blocks = std::min<int64_t>((tokens * 2 * c.heads + per - 1) / per, 8ll * device_sm_count());
    }
    return launch_pdl(pick[n.x_type](L, pairs), dim3((unsigned)blocks), dim3(kApThreads), 0, st, a);
}

}  // namespace esb
