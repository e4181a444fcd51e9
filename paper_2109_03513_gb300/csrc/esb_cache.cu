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
#include <type_traits>
#include <cuda_runtime.h>

#include "esb_internal.h"
#include "esb_heads.cuh"

namespace esb {

namespace {

constexpr int kApThreads = 256, kApBlocks = 2;     // on an SM
constexpr int kApAhead = 1;             // heads of a group that are loaded before they are needed

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
    int heads, page_size, page_shift, D, words, q_type, eights, tvec;
    RotArgs rot;
    HeadWork work;
};

// The spread's scale of a head whose 16 values a lane lie in a row (ROWS), or as
// the rotation pairs them.  Sums go in the order of the group projection's, so
// that the scale is the same number: over 16 values of a row and then over lanes,
// or, for sizes whose groups a warp takes (`eights`), over eight of each lane.
// 8192 tokens x 8 heads of 128 in bf16, rotated: 27.8 us (26 with the sums in the
// lanes' own order, whose scales differ in their last places).
template <int L, bool ROWS>
__device__ __forceinline__ float spread_scale(const AppendArgs& a, float astar, int half, const float (&u)[8], const float (&v)[8])
{
    const int part = threadIdx.x % L, left = a.D - 16 * part, turned = half >> 3;
    // which lane holds the eights that this one adds up, and in which of its two
    int lane[2];
    bool second[2];
#pragma unroll
    for (int h = 0; h < 2; h++) {
        const int e = 2 * part + h;
        lane[h] = e < turned ? e : (e < 2 * turned ? e - turned : part);
        second[h] = e < 2 * turned ? e >= turned : h;
    }
    auto value = [&](int h, int i) {
        if constexpr (ROWS) {
            return h ? v[i] : u[i];
        } else {
            const float x = __shfl_sync(0xffffffffu, u[i], lane[h], L), y = __shfl_sync(0xffffffffu, v[i], lane[h], L);
            return second[h] ? y : x;
        }
    };
    auto total = [&](float first, float last) {
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) last += __shfl_xor_sync(0xffffffffu, last, o);
        if (!a.eights) return last;
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) first += __shfl_xor_sync(0xffffffffu, first, o);
        return first + last;
    };
    const float n = (float)a.D;
    float first = 0.0f, last;
#pragma unroll
    for (int i = 0; i < 8; i++) first += value(0, i);
    last = a.eights ? 0.0f : first;
#pragma unroll
    for (int i = 0; i < 8; i++) last += value(1, i);
    const float mean = total(first, last) / n;
    first = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const float d = value(0, i) - mean;
        if (i < left) first = fmaf(d, d, first);
    }
    last = a.eights ? 0.0f : first;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const float d = value(1, i) - mean;
        if (8 + i < left) last = fmaf(d, d, last);
    }
    return __fmul_rn(astar, __fadd_rn(__fsqrt_rn(total(first, last) / n), 1e-7f));
}

// The scale of a head's 16 values in each of L lanes (those past its end 0), of
// its spread or its largest magnitude.
template <int L, bool SPREAD, bool ROWS>
__device__ __forceinline__ float scale_of(const AppendArgs& a, const AppendSide& s, int half, const float (&u)[8], const float (&v)[8])
{
    if constexpr (SPREAD) return spread_scale<L, ROWS>(a, s.astar, half, u, v);
    uint32_t mx = max(largest_of8(u, 1), largest_of8(v, 1));
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    return absmax_scale(mx, s.f);
}

// One token's head: its scale, then codes and values of the lane's two vectors
// of 8 from d0 and d1 on (there: the lane has them; ROWS: they lie in a row,
// else as a rotation by `half` pairs them).
template <int L, bool SPREAD, bool ROWS>
__device__ __forceinline__ void append_head(const AppendArgs& a, const AppendSide& s, bool on, int64_t slot, int64_t token, int head, int j0,
                                            bool there, int half, int d0, int d1, const float (&u)[8], const float (&v)[8])
{
    const float alpha = scale_of<L, SPREAD, ROWS>(a, s, half, u, v);
    if (!on) return;
    const int64_t page = a.page_shift >= 0 ? slot >> a.page_shift : slot / a.page_size;
    const int place = (int)(slot - page * a.page_size);
    const int row = head * a.page_size + place;
    if (j0 == 0) s.scales[page * a.page_lds + row] = alpha;
    uint32_t* codes = s.codes + page * a.page_ld + (int64_t)row * a.words;
    if (!there) {
        if (2 * j0 < a.words * 8) {                     // the words behind the values
            const uint32_t z = s.f.zero_code * 0x11111111u;
            *reinterpret_cast<uint2*>(codes + j0 / 4) = make_uint2(z, z);
        }
        return;
    }
    const GroupScale g = make_scale(alpha, s.f);
    uint32_t w0[1], w1[1];
    float q0[8], q1[8];
    quantise8<4, SPREAD>(u, g, s.f, w0, q0);            // absmax: no quotient is past the largest element
    quantise8<4, SPREAD>(v, g, s.f, w1, q1);
    if (d1 == d0 + 8) {
        *reinterpret_cast<uint2*>(codes + d0 / 8) = make_uint2(w0[0], w1[0]);
    } else {
        codes[d0 / 8] = w0[0];
        codes[d1 / 8] = w1[0];
    }
    if (s.q) {
        element_values(u, g, s.f, q0);
        element_values(v, g, s.f, q1);
        const int64_t at = token * s.ldq + head * a.D;
        store8_any(s.q, a.q_type, at + d0, 8, s.qvec, q0);
        store8_any(s.q, a.q_type, at + d1, 8, s.qvec, q1);
    }
}

// Heads of whole vectors: a lane holds 8 pairs of a key as the rotation pairs
// them, or 16 of a value's numbers, the next head's ahead; a warp keeps a
// token's cos and sin for several heads.  8192 tokens x 8 heads of 128 in bf16 to
// (4,2) with the values (80 MB): 27.2 us, bound by latency: four warps a scheduler,
// which issues in 54% of the cycles, wait for fixed latencies (1.9 cycles an
// instruction) and loads (1.2); no pipe is busier than 36%.  32 instructions a
// value: the exact rotation takes 8 of them, quotient, rounding, code and element
// some 20.  (41 us with rows in no order and a pair's other half read again.)
template <int TYPE, int L, int MODE, bool SPREAD>
__global__ void __launch_bounds__(kApThreads, kApBlocks) append_pairs_kernel(const AppendArgs a)
{
    using T = Elem<TYPE>;
    griddep_wait();
    const int j0 = (threadIdx.x % L) * 8;
#pragma unroll 1
    for (int k = 0; k < 2; k++) {
        HeadWalk<L, kApThreads / 32> to(a.work, k);
        if (!to.more()) continue;
        const AppendSide& s = a.side[k];
        const T* x = static_cast<const T*>(s.x);
        const int64_t ldx = s.ldx;
        // keys and values go the same way but for the rotation
        auto walk = [&](auto mode, const RotArgs& rot) {
            constexpr int M = decltype(mode)::value;
            const PairPlace p(j0, a.D / 2, rot);
            const bool turns = M == kPairHalves || (rot.dim && p.j0 < p.half);
            const int d0 = p.vec0<M>(), d1 = p.vec1<M>();
            float c[8], sn[8];
            RawPairs<T, M> next[kApAhead];
            HeadAt there[kApAhead];
            auto load = [&](int i) {
                there[i] = HeadAt(to);
                if (there[i].first && to.on) {
                    there[i].slot = __ldg(a.slots + to.token);
                    if (turns) there[i].pos = __ldg(a.positions + to.token);
                }
                next[i].load(x + (to.on ? to.token * ldx + to.head * a.D : 0), p, rot, to.on);
                to.next();
            };
#pragma unroll
            for (int i = 0; i < kApAhead; i++) load(i);
            int64_t slot = -1;
            while (there[0].more) {
                const RawPairs<T, M> raw = next[0];
                const HeadAt at = there[0];
#pragma unroll
                for (int i = 0; i + 1 < kApAhead; i++) {
                    next[i] = next[i + 1];
                    there[i] = there[i + 1];
                }
                load(kApAhead - 1);
                if (at.first) {
                    slot = at.slot;
                    if (turns) load_turn(rot, a.tvec, p, at.pos, c, sn);
                }
                float u[8], v[8];
                raw.u.values(u);
                raw.w.values(v);
                if (turns) {
                    float f[8], g[8];
                    if (p.in_rows<M>()) {
                        rows_to_pairs(u, v, f, g);
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; i++) { f[i] = u[i]; g[i] = v[i]; }
                    }
#pragma unroll
                    for (int i = 0; i < 8; i += 2) {
                        const Pair x0 = pair_of(f[i], f[i + 1]), x1 = pair_of(g[i], g[i + 1]), cc = pair_of(c[i], c[i + 1]);
                        const Pair sp = pair_of(sn[i], sn[i + 1]), sm = pair_of(-sn[i], -sn[i + 1]);
                        split(dot2_rn(x0, cc, x1, sm), f[i], f[i + 1]);
                        split(dot2_rn(x1, cc, x0, sp), g[i], g[i + 1]);
                    }
                    if (p.in_rows<M>()) {
                        pairs_to_rows(f, g, u, v);
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; i++) { u[i] = f[i]; v[i] = g[i]; }
                    }
                }
                append_head<L, SPREAD, M == kPairRows>(a, s, at.on && slot >= 0 && slot < a.places, slot, at.token, at.head, j0, p.count > 0, p.half, d0, d1, u, v);
            }
        };
        RotArgs none = {};
        if (k == 0) walk(std::integral_constant<int, MODE>(), a.rot);
        else walk(std::integral_constant<int, kPairRows>(), none);
    }
}
// Any heads: a lane holds 16 consecutive values, and reads a pair's other half again.
// Three blocks on an SM: left to itself the spread's kernel takes 117 registers, and
// 8192 x 8 heads of 128 that start anywhere 54 us, with three 43.
template <int TYPE, int L, bool SPREAD>
__global__ void __launch_bounds__(kApThreads, 3) append_kernel(const AppendArgs a)
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
        const float alpha = scale_of<L, SPREAD, true>(a, s, 0, v[0], v[1]);
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
template <int TYPE, int L, bool SPREAD> ApKernel append_of(int mode)
{
    switch (mode) {
    case kPairHalves: return append_pairs_kernel<TYPE, L, kPairHalves, SPREAD>;
    case kPairRows: return append_pairs_kernel<TYPE, L, kPairRows, SPREAD>;
    case kPairMixed: return append_pairs_kernel<TYPE, L, kPairMixed, SPREAD>;
    default: return append_kernel<TYPE, L, SPREAD>;
    }
}
template <int TYPE, bool SPREAD> ApKernel append_of(int L, int mode)
{
    return L == 4 ? append_of<TYPE, 4, SPREAD>(mode) : L == 8 ? append_of<TYPE, 8, SPREAD>(mode) : append_of<TYPE, 16, SPREAD>(mode);
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
    a.page_shift = -1;
    for (int i = 4; i < 31; i++)
        if (c.page_size == 1 << i) a.page_shift = i;
    const int padded = (c.head_dim + 31) / 32 * 32;
    a.eights = (padded & (padded - 1)) != 0;
    a.q_type = n.q_type; a.rot = make_rot(n.rotation, c.head_dim);
    a.tvec = table_vectors(a.rot);
    const int L = lanes_of(a.D);
    static ApKernel (*const pick[3][2])(int, int) = {{append_of<ESB_F32, false>, append_of<ESB_F32, true>},
                                                     {append_of<ESB_F16, false>, append_of<ESB_F16, true>},
                                                     {append_of<ESB_BF16, false>, append_of<ESB_BF16, true>}};
    const int mode = pair_mode(a.D, a.rot.dim, a.rot.inter, a.side[0].xvec && a.side[1].xvec);
    int64_t blocks;
    if (mode != kPairAny) {
        const int64_t most = (int64_t)device_sm_count() * (kApBlocks), warps = kApThreads / 32;
        a.work = split_heads(tokens, c.heads, c.heads, L, most * warps);
        blocks = std::min((a.work.part[0].items + a.work.part[1].items + warps - 1) / warps, most);
    } else {
        const int64_t per = kApThreads / L;
        blocks = std::min<int64_t>((tokens * 2 * c.heads + per - 1) / per, 8ll * device_sm_count());
    }
    return launch_pdl(pick[n.x_type][n.rule == ESB_SCALE_DDA](L, mode), dim3((unsigned)blocks), dim3(kApThreads), 0, st, a);
}

}  // namespace esb
