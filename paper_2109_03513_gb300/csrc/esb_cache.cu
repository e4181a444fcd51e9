// esb_cache.cu -- keys (rotated by their positions) and values of new tokens
// onto 4-bit ESB codes with a scale for each token and head, into the pages of
// a cache.
//
// A lane holds 16 consecutive values of a head, two words of codes; a head's
// lanes (8 for 128 values) find its largest magnitude or its spread together.
// The rotated key is rounded once to fp32 (both products and their sum carry
// their errors), so that its code is that of the exact rotation: on a set of
// 15 values a last place is a step of the set now and then.
#include <algorithm>
#include <cstdint>
#include <cuda_runtime.h>

#include "esb_internal.h"
#include "esb_rotate.cuh"
#include "esb_rows.cuh"

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
    int heads, page_size, D, words, q_type, rule;
    RotArgs rot;
};

template <int TYPE, int L>
__global__ void __launch_bounds__(kApThreads) append_kernel(const AppendArgs a)
{
    using T = Elem<TYPE>;
    griddep_wait();
    const int part = threadIdx.x % L, per = 2 * a.heads;
    const int64_t rows = a.tokens * per, step = (int64_t)gridDim.x * (kApThreads / L);
    auto total = [&](float v) {
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    };
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
        float alpha;
        if (a.rule == ESB_SCALE_ABSMAX) {
            uint32_t mx = max(largest_of8(v[0], 1), largest_of8(v[1], 1));
#pragma unroll
            for (int o = L / 2; o > 0; o >>= 1) mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            alpha = absmax_scale(mx, s.f);
        } else {
            float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; i++) s1 += v[i / 8][i % 8];
            const float mean = total(s1) / (float)a.D;
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const float d = d0 + i < a.D ? v[i / 8][i % 8] - mean : 0.0f;
                s2 = fmaf(d, d, s2);
            }
            alpha = __fmul_rn(s.astar, __fadd_rn(__fsqrt_rn(total(s2) / (float)a.D), 1e-7f));
        }
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
template <int TYPE> ApKernel append_of(int L)
{
    switch (L) {
    case 4: return append_kernel<TYPE, 4>;
    case 8: return append_kernel<TYPE, 8>;
    default: return append_kernel<TYPE, 16>;
    }
}

}  // namespace

cudaError_t launch_cache_append(int64_t tokens, const esb_kv_cache& c, const esb_append& n, double alpha_star_k, double alpha_star_v,
                                cudaStream_t st)
{
    AppendArgs a = {};
    auto rows16 = [](const void* p, int64_t ld, int type) {
        return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld * type_bytes(type) % 16 == 0;
    };
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
    const int L = a.D <= 64 ? 4 : a.D <= 128 ? 8 : 16;
    const int64_t per = kApThreads / L, blocks = std::min<int64_t>((tokens * 2 * c.heads + per - 1) / per, 8ll * device_sm_count());
    static ApKernel (*const pick[3])(int) = {append_of<ESB_F32>, append_of<ESB_F16>, append_of<ESB_BF16>};
    return launch_pdl(pick[n.x_type](L), dim3((unsigned)blocks), dim3(kApThreads), 0, st, a);
}

}  // namespace esb
