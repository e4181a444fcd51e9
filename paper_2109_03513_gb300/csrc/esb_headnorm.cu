// esb_headnorm.cu -- the root-mean-square norm of every head of queries and
// keys with the position rotation in the same pass, and its gradient.
//
// A lane holds 8 pairs of a head's values, as the rotation pairs them, so that
// a head (8 lanes for 128 values) needs only its sum of squares from other
// lanes.  A warp stays with a token for several heads: the token's cos and sin
// are in registers for all of them.
#include <algorithm>
#include <cstdint>
#include <cuda_runtime.h>

#include "esb_internal.h"
#include "esb_rotate.cuh"
#include "esb_rows.cuh"

namespace esb {

namespace {

constexpr int kHnThreads = 256, kHnWarps = kHnThreads / 32;
constexpr int kHnGradBlocks = 2;        // blocks on an SM of the gradient

struct HeadPart {
    const void *x, *dy, *weight;
    void* y;                            // forward: y; gradient: dx
    const float* rstd_in;
    float *rstd_out, *dweight;
    int64_t ldx, ldg, ldy;
    int heads;
};

struct HeadArgs {
    HeadPart part[2];
    const int64_t* positions;
    RotArgs rot;
    int64_t tokens;
    int D, heads;                       // heads of both parts
    int iter, chunks;                   // heads of a lane's group in one item; items of a token
    int w_type, tvec;
    float eps, inv_d;
    float* partial;                     // gradient: blocks x 2 x D
};

__device__ __forceinline__ float value_at(const void* p, int type, int i)
{
    if (type == ESB_F32) return static_cast<const float*>(p)[i];
    if (type == ESB_F16) return to_f32(static_cast<const __half*>(p)[i]);
    return to_f32(static_cast<const __nv_bfloat16*>(p)[i]);
}

// The pairs that a lane holds: (first, first + i) of `count`.
struct PairPlace {
    int j0, count;
    bool rows;                          // neighbours in memory: 16 values in a row
    int half;
    __device__ __forceinline__ PairPlace(int j, int pairs, const RotArgs& r)
    {
        j0 = j;
        count = min(8, max(0, pairs - j));
        half = r.dim >> 1;
        rows = r.inter || j0 >= half;
    }
    __device__ __forceinline__ int first(int i, const RotArgs& r) const { return r.inter || j0 + i >= half ? 2 * (j0 + i) : j0 + i; }
    __device__ __forceinline__ int second(int i, const RotArgs& r) const { return r.inter || j0 + i >= half ? 2 * (j0 + i) + 1 : j0 + i + half; }
};

// A lane's 16 values as they lie in memory.
template <class T, bool VEC>
struct RawPairs {
    Raw8<T> u, w;
    __device__ __forceinline__ void load(const T* x, const PairPlace& p, const RotArgs& r, bool on)
    {
        if constexpr (VEC) {
            const bool in = on && p.count > 0;
            const int at = p.rows ? 2 * p.j0 : p.j0;
            u.load(x + at, in ? 8 : 0, true);
            w.load(x + (p.rows ? at + 8 : at + p.half), in ? 8 : 0, true);
        } else {
            uint32_t a[8], b[8];
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const bool in = on && i < p.count;
                if constexpr (sizeof(T) == 4) {
                    a[i] = in ? __float_as_uint(x[p.first(i, r)]) : 0u;
                    b[i] = in ? __float_as_uint(x[p.second(i, r)]) : 0u;
                } else {
                    const uint16_t* h = reinterpret_cast<const uint16_t*>(x);
                    a[i] = in ? h[p.first(i, r)] : 0u;
                    b[i] = in ? h[p.second(i, r)] : 0u;
                }
            }
#pragma unroll
            for (int i = 0; i < (int)(2 * sizeof(T)); i++) {
                u.w[i] = sizeof(T) == 4 ? a[i] : a[(2 * i) & 7] | (a[(2 * i + 1) & 7] << 16);
                w.w[i] = sizeof(T) == 4 ? b[i] : b[(2 * i) & 7] | (b[(2 * i + 1) & 7] << 16);
            }
        }
    }
    __device__ __forceinline__ void values(const PairPlace& p, float (&a)[8], float (&b)[8]) const
    {
        float x[8], y[8];
        u.values(x);
        w.values(y);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const bool rows = VEC && p.rows;
            a[i] = rows ? (i < 4 ? x[(2 * i) & 7] : y[(2 * i) & 7]) : x[i];
            b[i] = rows ? (i < 4 ? x[(2 * i + 1) & 7] : y[(2 * i + 1) & 7]) : y[i];
        }
    }
};

template <class T, bool VEC>
__device__ __forceinline__ void store_pairs(T* y, const PairPlace& p, const RotArgs& r, const float (&a)[8], const float (&b)[8])
{
    if constexpr (VEC) {
        if (p.count <= 0) return;
        float u[8], w[8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            u[i] = p.rows ? ((i & 1) ? b[i / 2] : a[i / 2]) : a[i];
            w[i] = p.rows ? ((i & 1) ? b[4 + i / 2] : a[4 + i / 2]) : b[i];
        }
        const int at = p.rows ? 2 * p.j0 : p.j0;
        store8<T>(y + at, u);
        store8<T>(y + (p.rows ? at + 8 : at + p.half), w);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (i < p.count) {
                y[p.first(i, r)] = from_f32<T>(a[i]);
                y[p.second(i, r)] = from_f32<T>(b[i]);
            }
    }
}

// cos and sin of a lane's pairs; pairs past the rotated ones are left as they are.
__device__ __forceinline__ void load_turn(const HeadArgs& a, const PairPlace& p, int64_t pos, float (&c)[8], float (&s)[8])
{
    const RotArgs& r = a.rot;
    if (a.tvec && p.j0 + 8 <= p.half) {
        const bool in = pos >= 0 && pos < r.positions;
        const float* t = r.table + (in ? pos : 0) * r.ld + p.j0;
        const float4 c0 = __ldg(reinterpret_cast<const float4*>(t)), c1 = __ldg(reinterpret_cast<const float4*>(t + 4));
        const float4 s0 = __ldg(reinterpret_cast<const float4*>(t + p.half)), s1 = __ldg(reinterpret_cast<const float4*>(t + p.half + 4));
        c[0] = c0.x; c[1] = c0.y; c[2] = c0.z; c[3] = c0.w; c[4] = c1.x; c[5] = c1.y; c[6] = c1.z; c[7] = c1.w;
        s[0] = s0.x; s[1] = s0.y; s[2] = s0.z; s[3] = s0.w; s[4] = s1.x; s[5] = s1.y; s[6] = s1.z; s[7] = s1.w;
        if (!in) {
#pragma unroll
            for (int i = 0; i < 8; i++) c[i] = s[i] = __int_as_float(0x7fffffff);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; i++) {
        c[i] = 1.0f;
        s[i] = 0.0f;
        if (i < p.count && p.j0 + i < p.half) rot_at(r, pos, p.j0 + i, c[i], s[i]);
    }
}

template <int L>
__device__ __forceinline__ float group_sum(float v)
{
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Which heads a lane's group takes of an item, and of which part.
struct HeadPlace {
    int head, part;
    bool on;
    __device__ __forceinline__ HeadPlace(const HeadArgs& a, int h)
    {
        on = h < a.heads;
        part = h >= a.part[0].heads;
        head = part ? h - a.part[0].heads : h;
    }
};

template <int TYPE, int L, bool VEC>
__global__ void __launch_bounds__(kHnThreads) headnorm_kernel(const HeadArgs a)
{
    using T = Elem<TYPE>;
    constexpr int G = 32 / L;           // heads of a warp at a time
    griddep_wait();
    const int lane = threadIdx.x & 31, group = lane / L;
    const PairPlace p((lane % L) * 8, a.D / 2, a.rot);
    float wa[2][8], wb[2][8];
#pragma unroll
    for (int k = 0; k < 2; k++)
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const bool in = a.part[k].weight && i < p.count;
            wa[k][i] = in ? value_at(a.part[k].weight, a.w_type, p.first(i, a.rot)) : 1.0f;
            wb[k][i] = in ? value_at(a.part[k].weight, a.w_type, p.second(i, a.rot)) : 1.0f;
        }
    const int64_t items = a.tokens * a.chunks, step = (int64_t)gridDim.x * kHnWarps;
    for (int64_t item = (int64_t)blockIdx.x * kHnWarps + (threadIdx.x >> 5); item < items; item += step) {
        const int64_t token = item / a.chunks;
        const int h0 = (int)(item - token * a.chunks) * a.iter * G + group;
        float c[8], s[8];
        if (a.rot.dim) load_turn(a, p, __ldg(a.positions + token), c, s);
        RawPairs<T, VEC> next;
        auto load = [&](int it) {
            const HeadPlace hp(a, h0 + it * G);
            const bool on = hp.on && it < a.iter;
            const HeadPart& part = a.part[hp.part];
            next.load(static_cast<const T*>(part.x) + (on ? token * part.ldx + (int64_t)hp.head * a.D : 0), p, a.rot, on);
        };
        load(0);
        for (int it = 0; it < a.iter; it++) {
            const RawPairs<T, VEC> raw = next;
            const HeadPlace hp(a, h0 + it * G);
            load(it + 1);
            float u[8], v[8];
            raw.values(p, u, v);
            float ss = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; i++) ss = fmaf(u[i], u[i], fmaf(v[i], v[i], ss));
            const float rstd = __fdiv_rn(1.0f, __fsqrt_rn(fmaf(group_sum<L>(ss), a.inv_d, a.eps)));
            if (!hp.on) continue;
            const HeadPart& part = a.part[hp.part];
            if (part.rstd_out && p.j0 == 0) part.rstd_out[token * part.heads + hp.head] = rstd;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                u[i] *= rstd * (hp.part ? wa[1][i] : wa[0][i]);
                v[i] *= rstd * (hp.part ? wb[1][i] : wb[0][i]);
            }
            if (a.rot.dim && p.j0 < p.half) {
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const float x = u[i];
                    u[i] = fmaf(x, c[i], -(v[i] * s[i]));
                    v[i] = fmaf(v[i], c[i], x * s[i]);
                }
            }
            store_pairs<T, VEC>(static_cast<T*>(part.y) + token * part.ldy + (int64_t)hp.head * a.D, p, a.rot, u, v);
        }
    }
}

template <int TYPE, int L, bool VEC>
__global__ void __launch_bounds__(kHnThreads, kHnGradBlocks) headnorm_grad_kernel(const HeadArgs a)
{
    using T = Elem<TYPE>;
    constexpr int G = 32 / L;
    __shared__ float sums[kHnWarps][2][256];
    griddep_wait();
    const int lane = threadIdx.x & 31, group = lane / L, warp = threadIdx.x >> 5;
    const PairPlace p((lane % L) * 8, a.D / 2, a.rot);
    float da[2][8] = {}, db[2][8] = {};
    const int64_t items = a.tokens * a.chunks, step = (int64_t)gridDim.x * kHnWarps;
    for (int64_t item = (int64_t)blockIdx.x * kHnWarps + warp; item < items; item += step) {
        const int64_t token = item / a.chunks;
        const int h0 = (int)(item - token * a.chunks) * a.iter * G + group;
        float c[8], s[8];
        if (a.rot.dim) load_turn(a, p, __ldg(a.positions + token), c, s);
        RawPairs<T, VEC> next_x;
        RawPairs<T, VEC> next_g;
        float next_r = 0.0f;
        auto load = [&](int it) {
            const HeadPlace hp(a, h0 + it * G);
            const bool on = hp.on && it < a.iter;
            const HeadPart& part = a.part[hp.part];
            const int64_t at = on ? (int64_t)hp.head * a.D : 0, t = on ? token : 0;
            next_x.load(static_cast<const T*>(part.x) + t * part.ldx + at, p, a.rot, on);
            next_g.load(static_cast<const T*>(part.dy) + t * part.ldg + at, p, a.rot, on);
            next_r = on ? part.rstd_in[token * part.heads + hp.head] : 0.0f;
        };
        load(0);
        for (int it = 0; it < a.iter; it++) {
            const RawPairs<T, VEC> rx = next_x;
            const RawPairs<T, VEC> rg = next_g;
            const float rstd = next_r;
            const HeadPlace hp(a, h0 + it * G);
            load(it + 1);
            float u[8], v[8], g[8], h[8];
            rx.values(p, u, v);
            rg.values(p, g, h);
            if (a.rot.dim && p.j0 < p.half) {
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const float x = g[i];
                    g[i] = fmaf(x, c[i], h[i] * s[i]);
                    h[i] = fmaf(h[i], c[i], -(x * s[i]));
                }
            }
            const HeadPart& part = a.part[hp.part];
            float dot = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                u[i] *= rstd;           // n
                v[i] *= rstd;
                if (hp.on) {
                    const float x = g[i] * u[i], y = h[i] * v[i];
                    da[0][i] += hp.part ? 0.0f : x;
                    db[0][i] += hp.part ? 0.0f : y;
                    da[1][i] += hp.part ? x : 0.0f;
                    db[1][i] += hp.part ? y : 0.0f;
                }
                if (part.weight && i < p.count) {   // read again from the first-level cache: the sums have the registers
                    g[i] *= value_at(part.weight, a.w_type, p.first(i, a.rot));
                    h[i] *= value_at(part.weight, a.w_type, p.second(i, a.rot));
                }
                dot = fmaf(g[i], u[i], fmaf(h[i], v[i], dot));
            }
            dot = group_sum<L>(dot) * a.inv_d;
            if (!hp.on) continue;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                u[i] = rstd * fmaf(-u[i], dot, g[i]);
                v[i] = rstd * fmaf(-v[i], dot, h[i]);
            }
            store_pairs<T, VEC>(static_cast<T*>(part.y) + token * part.ldy + (int64_t)hp.head * a.D, p, a.rot, u, v);
        }
    }
    if (!a.partial) return;
#pragma unroll
    for (int k = 0; k < 2; k++)
#pragma unroll
        for (int i = 0; i < 8; i++) {
            float x = da[k][i], y = db[k][i];
#pragma unroll
            for (int o = L; o < 32; o <<= 1) {
                x += __shfl_xor_sync(0xffffffffu, x, o);
                y += __shfl_xor_sync(0xffffffffu, y, o);
            }
            if (group == 0 && i < p.count) {
                sums[warp][k][p.first(i, a.rot)] = x;
                sums[warp][k][p.second(i, a.rot)] = y;
            }
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * a.D; i += kHnThreads) {
        const int k = i >= a.D, e = i - k * a.D;
        float t = 0.0f;
        for (int w = 0; w < kHnWarps; w++) t += sums[w][k][e];
        a.partial[(int64_t)blockIdx.x * 2 * a.D + i] = t;
    }
}

// The blocks' sums in their order: 32 columns a block, 32 threads a column.
__global__ void __launch_bounds__(1024) headnorm_dweight_kernel(const float* partial, int blocks, int D, float* dq, float* dk)
{
    __shared__ float sums[32][33];
    griddep_wait();
    const int col = blockIdx.x * 32 + threadIdx.x % 32, part = threadIdx.x / 32;
    float t = 0.0f;
    if (col < 2 * D)
        for (int b = part; b < blocks; b += 32) t += partial[(int64_t)b * 2 * D + col];
    sums[part][threadIdx.x % 32] = t;
    __syncthreads();
    t = warp_sum(sums[threadIdx.x % 32][part]);
    const int out = blockIdx.x * 32 + part;
    if (threadIdx.x % 32 == 0 && out < 2 * D) {
        float* to = out < D ? dq : dk;
        if (to) to[out < D ? out : out - D] = t;
    }
}

int lanes_of(int D) { return D <= 64 ? 4 : D <= 128 ? 8 : 16; }

// Heads of a lane's group in an item: a token's, while that leaves 16 warps for every SM.
void split_heads(HeadArgs& a, int L)
{
    const int per = 32 / L, full = (a.heads + per - 1) / per;
    const int64_t items = 16ll * device_sm_count();
    const int64_t iter = a.tokens >= items ? full : full * a.tokens / items;
    a.iter = (int)std::clamp<int64_t>(iter, 1, full);
    a.chunks = (full + a.iter - 1) / a.iter;
}

int64_t blocks_of(const HeadArgs& a, int per_sm)
{
    return std::min<int64_t>((a.tokens * a.chunks + kHnWarps - 1) / kHnWarps, (int64_t)per_sm * device_sm_count());
}

bool rows16(const void* p, int64_t ld, int type)
{
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld * type_bytes(type) % 16 == 0;
}

using HnKernel = void (*)(const HeadArgs);
template <int TYPE, bool VEC> HnKernel norm_kernel(int L)
{
    switch (L) {
    case 4: return headnorm_kernel<TYPE, 4, VEC>;
    case 8: return headnorm_kernel<TYPE, 8, VEC>;
    default: return headnorm_kernel<TYPE, 16, VEC>;
    }
}
template <int TYPE, bool VEC> HnKernel grad_kernel(int L)
{
    switch (L) {
    case 4: return headnorm_grad_kernel<TYPE, 4, VEC>;
    case 8: return headnorm_grad_kernel<TYPE, 8, VEC>;
    default: return headnorm_grad_kernel<TYPE, 16, VEC>;
    }
}

// A lane's values are two vectors: whole eights of pairs on both sides of the rotation's end.
bool pairs_of_vectors(int D, const esb_rotation& r) { return D % 16 == 0 && (r.interleaved || r.dim % 16 == 0); }

}  // namespace

cudaError_t launch_headnorm(int64_t tokens, const esb_head_norm& n, cudaStream_t st)
{
    HeadArgs a = {};
    bool vec = pairs_of_vectors(n.head_dim, n.rotation);
    for (int k = 0; k < 2; k++) {
        const esb_heads& h = n.part[k];
        HeadPart& p = a.part[k];
        p.heads = h.heads;
        if (h.heads == 0) continue;
        p.x = h.x; p.ldx = h.ldx; p.y = h.y; p.ldy = h.ldy; p.weight = h.weight; p.rstd_out = h.rstd;
        vec = vec && rows16(h.x, h.ldx, n.x_type) && rows16(h.y, h.ldy, n.x_type);
    }
    a.positions = n.positions; a.rot = make_rot(&n.rotation, n.head_dim);
    a.tokens = tokens; a.D = n.head_dim; a.heads = n.part[0].heads + n.part[1].heads;
    a.w_type = n.w_type; a.tvec = a.rot.vec; a.eps = n.eps; a.inv_d = 1.0f / (float)n.head_dim;
    const int L = lanes_of(a.D);
    split_heads(a, L);
    static HnKernel (*const pick[3][2])(int) = {{norm_kernel<ESB_F32, false>, norm_kernel<ESB_F32, true>},
                                                {norm_kernel<ESB_F16, false>, norm_kernel<ESB_F16, true>},
                                                {norm_kernel<ESB_BF16, false>, norm_kernel<ESB_BF16, true>}};
    return launch_pdl(pick[n.x_type][vec](L), dim3((unsigned)blocks_of(a, 8)), dim3(kHnThreads), 0, st, a);
}

size_t headnorm_grad_workspace_bytes(int64_t tokens, int64_t heads, int head_dim)
{
    HeadArgs a = {};
    a.tokens = tokens; a.heads = (int)heads; a.D = head_dim;
    split_heads(a, lanes_of(head_dim));
    return sizeof(float) * 2 * (size_t)head_dim * (size_t)blocks_of(a, kHnGradBlocks);
}

cudaError_t launch_headnorm_grad(int64_t tokens, const esb_head_norm_grad& n, void* workspace, cudaStream_t st)
{
    HeadArgs a = {};
    bool vec = pairs_of_vectors(n.head_dim, n.rotation), sums = false;
    for (int k = 0; k < 2; k++) {
        const esb_heads_grad& h = n.part[k];
        HeadPart& p = a.part[k];
        p.heads = h.heads;
        sums = sums || h.dweight;
        p.dweight = h.dweight;
        if (h.heads == 0) continue;
        p.x = h.x; p.ldx = h.ldx; p.dy = h.dy; p.ldg = h.ldg; p.y = h.dx; p.ldy = h.lddx; p.weight = h.weight; p.rstd_in = h.rstd;
        vec = vec && rows16(h.x, h.ldx, n.x_type) && rows16(h.dy, h.ldg, n.x_type) && rows16(h.dx, h.lddx, n.x_type);
    }
    a.positions = n.positions; a.rot = make_rot(&n.rotation, n.head_dim);
    a.tokens = tokens; a.D = n.head_dim; a.heads = n.part[0].heads + n.part[1].heads;
    a.w_type = n.w_type; a.tvec = a.rot.vec; a.inv_d = 1.0f / (float)n.head_dim;
    a.partial = sums ? static_cast<float*>(workspace) : nullptr;
    const int L = lanes_of(a.D);
    split_heads(a, L);
    const int blocks = (int)blocks_of(a, kHnGradBlocks);
    static HnKernel (*const pick[3][2])(int) = {{grad_kernel<ESB_F32, false>, grad_kernel<ESB_F32, true>},
                                                {grad_kernel<ESB_F16, false>, grad_kernel<ESB_F16, true>},
                                                {grad_kernel<ESB_BF16, false>, grad_kernel<ESB_BF16, true>}};
    cudaError_t e = launch_pdl(pick[n.x_type][vec](L), dim3((unsigned)blocks), dim3(kHnThreads), 0, st, a);
    if (e != cudaSuccess || !sums) return e;
    return launch_pdl(headnorm_dweight_kernel, dim3((unsigned)((2 * a.D + 31) / 32)), dim3(1024), 0, st,
                      static_cast<const float*>(a.partial), blocks, a.D, a.part[0].dweight, a.part[1].dweight);
}

}  // namespace esb
