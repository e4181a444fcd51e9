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
#include "esb_heads.cuh"

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
    HeadWork work;
    const int64_t* positions;
    RotArgs rot;
    int D, w_type, tvec;
    float eps, inv_d;
    float* partial;                     // gradient: blocks x 2 x D
};

__device__ __forceinline__ float value_at(const void* p, int type, int i)
{
    if (type == ESB_F32) return static_cast<const float*>(p)[i];
    if (type == ESB_F16) return to_f32(static_cast<const __half*>(p)[i]);
    return to_f32(static_cast<const __nv_bfloat16*>(p)[i]);
}

template <int L>
__device__ __forceinline__ float group_sum(float v)
{
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

__device__ __forceinline__ void load_weights(const HeadArgs& a, int part, const PairPlace& p, float (&wa)[8], float (&wb)[8])
{
    const void* w = a.part[part].weight;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        wa[i] = w && i < p.count ? value_at(w, a.w_type, p.first(i, a.rot)) : 1.0f;
        wb[i] = w && i < p.count ? value_at(w, a.w_type, p.second(i, a.rot)) : 1.0f;
    }
}

// Bound by HBM and by the latency of few values in flight: 24 warps on an SM
// with one head of a lane's group ahead.
template <int TYPE, int L, bool VEC>
__global__ void __launch_bounds__(kHnThreads, TYPE == ESB_F32 ? 2 : 3) headnorm_kernel(const HeadArgs a)
{
    using T = Elem<TYPE>;
    griddep_wait();
    const PairPlace p((threadIdx.x % L) * 8, a.D / 2, a.rot);
    float wa[8], wb[8], c[8], s[8];
    int weights = -1;
    HeadWalk<L, kHnWarps> at = {}, to = {};   // where the work is, where the loads are
    RawPairs<T, VEC> next;
    int64_t next_pos = 0, at_pos;
    auto load = [&]() {
        const HeadPart& part = a.part[to.part];
        if (to.it == 0) next_pos = a.rot.dim && to.on ? __ldg(a.positions + to.token) : 0;
        next.load(static_cast<const T*>(part.x) + (to.on ? to.token * part.ldx + (int64_t)to.head * a.D : 0), p, a.rot, to.on);
    };
    to.start(a.work);
    load();
    at = to;
    while (at.more(a.work)) {
        const RawPairs<T, VEC> raw = next;
        at_pos = next_pos;
        to.next(a.work);
        load();
        if (at.it == 0) {
            if (a.rot.dim && at.token < a.work.tokens) load_turn(a.rot, a.tvec, p, at_pos, c, s);
            if (at.part != weights) load_weights(a, weights = at.part, p, wa, wb);
        }
        float u[8], v[8];
        raw.values(p, u, v);
        float ss = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; i++) ss = fmaf(u[i], u[i], fmaf(v[i], v[i], ss));
        const float rstd = __fdiv_rn(1.0f, __fsqrt_rn(fmaf(group_sum<L>(ss), a.inv_d, a.eps)));
        if (at.on) {
            const HeadPart& part = a.part[at.part];
            if (part.rstd_out && p.j0 == 0) part.rstd_out[at.token * part.heads + at.head] = rstd;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                u[i] *= rstd * wa[i];
                v[i] *= rstd * wb[i];
            }
            if (a.rot.dim && p.j0 < p.half) {
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const float x = u[i];
                    u[i] = fmaf(x, c[i], -(v[i] * s[i]));
                    v[i] = fmaf(v[i], c[i], x * s[i]);
                }
            }
            store_pairs<T, VEC>(static_cast<T*>(part.y) + at.token * part.ldy + (int64_t)at.head * a.D, p, a.rot, u, v);
        }
        at = to;
    }
}

template <int TYPE, int L, bool VEC>
__global__ void __launch_bounds__(kHnThreads, kHnGradBlocks) headnorm_grad_kernel(const HeadArgs a)
{
    using T = Elem<TYPE>;
    __shared__ float sums[kHnWarps][2][256];
    griddep_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const PairPlace p((lane % L) * 8, a.D / 2, a.rot);
    for (int i = threadIdx.x; i < kHnWarps * 2 * 256; i += kHnThreads) (&sums[0][0][0])[i] = 0.0f;
    __syncthreads();
    float wa[8], wb[8], c[8], s[8], da[8], db[8];
#pragma unroll
    for (int i = 0; i < 8; i++) da[i] = db[i] = 0.0f;
    int weights = -1;
    auto flush = [&]() {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            float x = da[i], y = db[i];
#pragma unroll
            for (int o = L; o < 32; o <<= 1) {
                x += __shfl_xor_sync(0xffffffffu, x, o);
                y += __shfl_xor_sync(0xffffffffu, y, o);
            }
            if (lane < L && i < p.count) {
                sums[warp][weights][p.first(i, a.rot)] = x;
                sums[warp][weights][p.second(i, a.rot)] = y;
            }
            da[i] = db[i] = 0.0f;
        }
    };
    HeadWalk<L, kHnWarps> at = {}, to = {};
    RawPairs<T, VEC> next_x, next_g;
    float next_r;
    int64_t next_pos = 0, at_pos;
    auto load = [&]() {
        const HeadPart& part = a.part[to.part];
        if (to.it == 0) next_pos = a.rot.dim && to.on ? __ldg(a.positions + to.token) : 0;
        const int64_t h = to.on ? (int64_t)to.head * a.D : 0, t = to.on ? to.token : 0;
        next_x.load(static_cast<const T*>(part.x) + t * part.ldx + h, p, a.rot, to.on);
        next_g.load(static_cast<const T*>(part.dy) + t * part.ldg + h, p, a.rot, to.on);
        next_r = to.on ? part.rstd_in[to.token * part.heads + to.head] : 0.0f;
    };
    to.start(a.work);
    load();
    at = to;
    while (at.more(a.work)) {
        const RawPairs<T, VEC> rx = next_x, rg = next_g;
        const float rstd = next_r;
        at_pos = next_pos;
        to.next(a.work);
        load();
        if (at.it == 0) {
            if (a.rot.dim && at.token < a.work.tokens) load_turn(a.rot, a.tvec, p, at_pos, c, s);
            if (at.part != weights) {
                if (weights >= 0) flush();
                load_weights(a, weights = at.part, p, wa, wb);
            }
        }
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
        float dot = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            u[i] *= rstd;               // n
            v[i] *= rstd;
            if (at.on) {
                da[i] = fmaf(g[i], u[i], da[i]);
                db[i] = fmaf(h[i], v[i], db[i]);
            }
            g[i] *= wa[i];
            h[i] *= wb[i];
            dot = fmaf(g[i], u[i], fmaf(h[i], v[i], dot));
        }
        dot = group_sum<L>(dot) * a.inv_d;
        if (at.on) {
            const HeadPart& part = a.part[at.part];
#pragma unroll
            for (int i = 0; i < 8; i++) {
                u[i] = rstd * fmaf(-u[i], dot, g[i]);
                v[i] = rstd * fmaf(-v[i], dot, h[i]);
            }
            store_pairs<T, VEC>(static_cast<T*>(part.y) + at.token * part.ldy + (int64_t)at.head * a.D, p, a.rot, u, v);
        }
        at = to;
    }
    if (!a.partial) return;
    if (weights >= 0) flush();
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

int64_t blocks_of(const HeadArgs& a, int64_t most)
{
    return std::min((a.work.part[0].items + a.work.part[1].items + kHnWarps - 1) / kHnWarps, most);
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

}  // namespace

cudaError_t launch_headnorm(int64_t tokens, const esb_head_norm& n, cudaStream_t st)
{
    HeadArgs a = {};
    bool vec = pairs_of_vectors(n.head_dim, n.rotation.dim, n.rotation.interleaved);
    for (int k = 0; k < 2; k++) {
        const esb_heads& h = n.part[k];
        HeadPart& p = a.part[k];
        p.heads = h.heads;
        if (h.heads == 0) continue;
        p.x = h.x; p.ldx = h.ldx; p.y = h.y; p.ldy = h.ldy; p.weight = h.weight; p.rstd_out = h.rstd;
        vec = vec && rows16(h.x, h.ldx, n.x_type) && rows16(h.y, h.ldy, n.x_type);
    }
    a.positions = n.positions; a.rot = make_rot(&n.rotation, n.head_dim);
    a.D = n.head_dim;
    a.w_type = n.w_type; a.tvec = a.rot.vec; a.eps = n.eps; a.inv_d = 1.0f / (float)n.head_dim;
    const int L = lanes_of(a.D);
    const int64_t most = (int64_t)device_sm_count() * (n.x_type == ESB_F32 ? 2 : 3);
    a.work = split_heads(tokens, a.part[0].heads, a.part[1].heads, L, most * kHnWarps);
    static HnKernel (*const pick[3][2])(int) = {{norm_kernel<ESB_F32, false>, norm_kernel<ESB_F32, true>},
                                                {norm_kernel<ESB_F16, false>, norm_kernel<ESB_F16, true>},
                                                {norm_kernel<ESB_BF16, false>, norm_kernel<ESB_BF16, true>}};
    return launch_pdl(pick[n.x_type][vec](L), dim3((unsigned)blocks_of(a, most)), dim3(kHnThreads), 0, st, a);
}

// A part of the sums for every block that there may be.
size_t headnorm_grad_workspace_bytes(int64_t tokens, int64_t heads, int head_dim)
{
    const int64_t rows = (tokens * heads + kHnWarps - 1) / kHnWarps + 1;
    return sizeof(float) * 2 * (size_t)head_dim * (size_t)std::min<int64_t>(rows, (int64_t)kHnGradBlocks * device_sm_count());
}

cudaError_t launch_headnorm_grad(int64_t tokens, const esb_head_norm_grad& n, void* workspace, cudaStream_t st)
{
    HeadArgs a = {};
    bool vec = pairs_of_vectors(n.head_dim, n.rotation.dim, n.rotation.interleaved), sums = false;
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
    a.D = n.head_dim;
    a.w_type = n.w_type; a.tvec = a.rot.vec; a.inv_d = 1.0f / (float)n.head_dim;
    a.partial = sums ? static_cast<float*>(workspace) : nullptr;
    const int L = lanes_of(a.D);
    const int64_t most = (int64_t)kHnGradBlocks * device_sm_count();
    a.work = split_heads(tokens, a.part[0].heads, a.part[1].heads, L, most * kHnWarps);
    const int blocks = (int)blocks_of(a, most);
    static HnKernel (*const pick[3][2])(int) = {{grad_kernel<ESB_F32, false>, grad_kernel<ESB_F32, true>},
                                                {grad_kernel<ESB_F16, false>, grad_kernel<ESB_F16, true>},
                                                {grad_kernel<ESB_BF16, false>, grad_kernel<ESB_BF16, true>}};
    cudaError_t e = launch_pdl(pick[n.x_type][vec](L), dim3((unsigned)blocks), dim3(kHnThreads), 0, st, a);
    if (e != cudaSuccess || !sums) return e;
    return launch_pdl(headnorm_dweight_kernel, dim3((unsigned)((2 * a.D + 31) / 32)), dim3(1024), 0, st,
                      static_cast<const float*>(a.partial), blocks, a.D, a.part[0].dweight, a.part[1].dweight);
}

}  // namespace esb
