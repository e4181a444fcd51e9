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
constexpr int kHnBlocks = 2;            // on an SM
constexpr int kHnAhead = 2;             // heads of a group loaded before they are needed (the gradient: one, x and dy)

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

// 8192 x (32 + 8) heads of 128 in bf16 (172 MB): 39.5 us, 4.4 TB/s, 64% of the
// copy rate.  16 warps on an SM, each with kHnAhead heads of a lane's group
// loaded ahead, wait for loads and for the chain of a head (its squares, their
// sum over lanes, the root, the rotation); 15 instructions a value.  24 warps of
// 80 registers spill (47 us), three heads ahead are no faster (40.4).
template <int TYPE, int L, int MODE>
__global__ void __launch_bounds__(kHnThreads, kHnBlocks) headnorm_kernel(const HeadArgs a)
{
    using T = Elem<TYPE>;
    griddep_wait();
    const PairPlace p((threadIdx.x % L) * 8, a.D / 2, a.rot);
    const bool turns = MODE == kPairHalves || (a.rot.dim && p.j0 < p.half);
#pragma unroll 1
    for (int k = 0; k < 2; k++) {
        HeadWalk<L, kHnWarps> to(a.work, k);
        if (!to.more()) continue;
        const T* x = static_cast<const T*>(a.part[k].x);
        T* y = static_cast<T*>(a.part[k].y);
        float* rstds = a.part[k].rstd_out;
        const int64_t ldx = a.part[k].ldx, ldy = a.part[k].ldy;
        float wa[8], wb[8], c[8], s[8];
        load_weights(a, k, p, wa, wb);
        RawPairs<T, MODE> next[kHnAhead];
        HeadAt there[kHnAhead];
        auto load = [&](int i) {
            there[i] = HeadAt(to);
            there[i].pos = there[i].first && a.rot.dim && to.on ? __ldg(a.positions + to.token) : 0;
            next[i].load(x + (to.on ? to.token * ldx + to.head * a.D : 0), p, a.rot, to.on);
            to.next();
        };
#pragma unroll
        for (int i = 0; i < kHnAhead; i++) load(i);
        while (there[0].more) {
            const RawPairs<T, MODE> raw = next[0];
            const HeadAt at = there[0];
            const int64_t pos = at.pos;
#pragma unroll
            for (int i = 0; i + 1 < kHnAhead; i++) {
                next[i] = next[i + 1];
                there[i] = there[i + 1];
            }
            load(kHnAhead - 1);
            if (at.first && turns) load_turn(a.rot, a.tvec, p, pos, c, s);
            float u[8], v[8];
            raw.values(p, u, v);
            Pair ss = pair_of(0.0f, 0.0f);
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const Pair q = pair_of(u[i], u[i + 1]), r = pair_of(v[i], v[i + 1]);
                ss = fma2(q, q, fma2(r, r, ss));
            }
            float s0, s1;
            split(ss, s0, s1);
            const float rstd = rsqrt_of(fmaf(group_sum<L>(s0 + s1), a.inv_d, a.eps));
            if (at.on) {
                if (rstds && p.j0 == 0) rstds[(int64_t)at.token * to.heads + at.head] = rstd;
                const Pair rr = pair_of(rstd, rstd);
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    split(mul2(mul2(rr, pair_of(wa[i], wa[i + 1])), pair_of(u[i], u[i + 1])), u[i], u[i + 1]);
                    split(mul2(mul2(rr, pair_of(wb[i], wb[i + 1])), pair_of(v[i], v[i + 1])), v[i], v[i + 1]);
                }
                if (turns) turn_pairs<false>(u, v, c, s);
                store_pairs<T, MODE>(y + at.token * ldy + at.head * a.D, p, a.rot, u, v);
            }
        }
    }
}

// The same with x and dy, and sums of the weights' gradients in registers: 8192 x
// (16 + 4) heads of 128 in bf16 (126 MB) 35 us, with the forward pass 59.
template <int TYPE, int L, int MODE>
__global__ void __launch_bounds__(kHnThreads, kHnBlocks) headnorm_grad_kernel(const HeadArgs a)
{
    using T = Elem<TYPE>;
    __shared__ float sums[kHnWarps][2][256];
    griddep_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const PairPlace p((lane % L) * 8, a.D / 2, a.rot);
    const bool turns = MODE == kPairHalves || (a.rot.dim && p.j0 < p.half);
#pragma unroll 1
    for (int k = 0; k < 2; k++) {
        HeadWalk<L, kHnWarps> to(a.work, k);
        const T *x = static_cast<const T*>(a.part[k].x), *dy = static_cast<const T*>(a.part[k].dy);
        T* dx = static_cast<T*>(a.part[k].y);
        const float* rstds = a.part[k].rstd_in;
        const int64_t ldx = a.part[k].ldx, ldg = a.part[k].ldg, lddx = a.part[k].ldy;
        float wa[8], wb[8], c[8], s[8];
        Pair da[4], db[4];
        load_weights(a, k, p, wa, wb);
#pragma unroll
        for (int i = 0; i < 4; i++) da[i] = db[i] = pair_of(0.0f, 0.0f);
        RawPairs<T, MODE> next_x, next_g;
        float next_r = 0.0f;
        HeadAt there;
        auto load = [&]() {
            there = HeadAt(to);
            there.pos = there.first && a.rot.dim && to.on ? __ldg(a.positions + to.token) : 0;
            const int h = to.head * a.D;
            next_x.load(x + (to.on ? to.token * ldx + h : 0), p, a.rot, to.on);
            next_g.load(dy + (to.on ? to.token * ldg + h : 0), p, a.rot, to.on);
            next_r = to.on ? rstds[(int64_t)to.token * to.heads + to.head] : 0.0f;   // a head that is not there adds nothing
            to.next();
        };
        there = HeadAt(to);
        if (there.more) load();
        while (there.more) {
            const RawPairs<T, MODE> rx = next_x, rg = next_g;
            const float rstd = next_r;
            const HeadAt at = there;
            load();
            if (at.first && turns) load_turn(a.rot, a.tvec, p, at.pos, c, s);
            float u[8], v[8], g[8], h[8];
            rx.values(p, u, v);
            rg.values(p, g, h);
            if (turns && at.on) turn_pairs<true>(g, h, c, s);
            const Pair rr = pair_of(rstd, rstd);
            Pair dots = pair_of(0.0f, 0.0f);
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                // n, the weights' sums, g weight
                const Pair n0 = mul2(pair_of(u[i], u[i + 1]), rr), n1 = mul2(pair_of(v[i], v[i + 1]), rr);
                const Pair g0 = pair_of(g[i], g[i + 1]), g1 = pair_of(h[i], h[i + 1]);
                da[i / 2] = fma2(g0, n0, da[i / 2]);
                db[i / 2] = fma2(g1, n1, db[i / 2]);
                const Pair e0 = mul2(g0, pair_of(wa[i], wa[i + 1])), e1 = mul2(g1, pair_of(wb[i], wb[i + 1]));
                dots = fma2(e0, n0, fma2(e1, n1, dots));
                split(n0, u[i], u[i + 1]);
                split(n1, v[i], v[i + 1]);
                split(e0, g[i], g[i + 1]);
                split(e1, h[i], h[i + 1]);
            }
            float d0, d1;
            split(dots, d0, d1);
            const float dot = group_sum<L>(d0 + d1) * a.inv_d;
            if (at.on) {
                const Pair minus = pair_of(-dot, -dot);
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    split(mul2(rr, fma2(pair_of(u[i], u[i + 1]), minus, pair_of(g[i], g[i + 1]))), u[i], u[i + 1]);
                    split(mul2(rr, fma2(pair_of(v[i], v[i + 1]), minus, pair_of(h[i], h[i + 1]))), v[i], v[i + 1]);
                }
                store_pairs<T, MODE>(dx + at.token * lddx + at.head * a.D, p, a.rot, u, v);
            }
        }
        // this warp's sums: its lanes' groups joined
#pragma unroll
        for (int i = 0; i < 8; i++) {
            float x0, x1, y0, y1;
            split(da[i / 2], x0, x1);
            split(db[i / 2], y0, y1);
            float xs = i & 1 ? x1 : x0, ys = i & 1 ? y1 : y0;
#pragma unroll
            for (int o = L; o < 32; o <<= 1) {
                xs += __shfl_xor_sync(0xffffffffu, xs, o);
                ys += __shfl_xor_sync(0xffffffffu, ys, o);
            }
            if (lane < L && i < p.count) {
                sums[warp][k][p.first(i, a.rot)] = xs;
                sums[warp][k][p.second(i, a.rot)] = ys;
            }
        }
    }
    if (!a.partial) return;
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
template <int TYPE, int L> HnKernel kernel_of(int mode, bool grad)
{
    switch (mode) {
    case kPairHalves: return grad ? headnorm_grad_kernel<TYPE, L, kPairHalves> : headnorm_kernel<TYPE, L, kPairHalves>;
    case kPairRows: return grad ? headnorm_grad_kernel<TYPE, L, kPairRows> : headnorm_kernel<TYPE, L, kPairRows>;
    case kPairMixed: return grad ? headnorm_grad_kernel<TYPE, L, kPairMixed> : headnorm_kernel<TYPE, L, kPairMixed>;
    default: return grad ? headnorm_grad_kernel<TYPE, L, kPairAny> : headnorm_kernel<TYPE, L, kPairAny>;
    }
}
template <int TYPE> HnKernel kernel_of(int L, int mode, bool grad)
{
    return L == 4 ? kernel_of<TYPE, 4>(mode, grad) : L == 8 ? kernel_of<TYPE, 8>(mode, grad) : kernel_of<TYPE, 16>(mode, grad);
}
HnKernel kernel_of(int type, int L, int mode, bool grad)
{
    return type == ESB_F32 ? kernel_of<ESB_F32>(L, mode, grad) : type == ESB_F16 ? kernel_of<ESB_F16>(L, mode, grad) : kernel_of<ESB_BF16>(L, mode, grad);
}

}  // namespace

cudaError_t launch_headnorm(int64_t tokens, const esb_head_norm& n, cudaStream_t st)
{
    HeadArgs a = {};
    bool vec = true;
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
    a.w_type = n.w_type; a.tvec = table_vectors(a.rot); a.eps = n.eps; a.inv_d = 1.0f / (float)n.head_dim;
    const int L = lanes_of(a.D);
    const int64_t most = (int64_t)device_sm_count() * kHnBlocks;
    a.work = split_heads(tokens, a.part[0].heads, a.part[1].heads, L, most * kHnWarps);
    const int mode = pair_mode(a.D, a.rot.dim, a.rot.inter, vec);
    return launch_pdl(kernel_of(n.x_type, L, mode, false), dim3((unsigned)blocks_of(a, most)), dim3(kHnThreads), 0, st, a);
}

// A part of the sums for every block that there may be.
size_t headnorm_grad_workspace_bytes(int64_t tokens, int64_t heads, int head_dim)
{
    const int64_t rows = (tokens * heads + kHnWarps - 1) / kHnWarps + 1;
    return sizeof(float) * 2 * (size_t)head_dim * (size_t)std::min<int64_t>(rows, (int64_t)device_sm_count() * kHnBlocks);
}

cudaError_t launch_headnorm_grad(int64_t tokens, const esb_head_norm_grad& n, void* workspace, cudaStream_t st)
{
    HeadArgs a = {};
    bool vec = true, sums = false;
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
    a.w_type = n.w_type; a.tvec = table_vectors(a.rot); a.inv_d = 1.0f / (float)n.head_dim;
    a.partial = sums ? static_cast<float*>(workspace) : nullptr;
    const int L = lanes_of(a.D);
    const int64_t most = (int64_t)device_sm_count() * kHnBlocks;
    a.work = split_heads(tokens, a.part[0].heads, a.part[1].heads, L, most * kHnWarps);
    const int blocks = (int)blocks_of(a, most);
    const int mode = pair_mode(a.D, a.rot.dim, a.rot.inter, vec);
    cudaError_t e = launch_pdl(kernel_of(n.x_type, L, mode, true), dim3((unsigned)blocks), dim3(kHnThreads), 0, st, a);
    if (e != cudaSuccess || !sums) return e;
    return launch_pdl(headnorm_dweight_kernel, dim3((unsigned)((2 * a.D + 31) / 32)), dim3(1024), 0, st,
                      static_cast<const float*>(a.partial), blocks, a.D, a.part[0].dweight, a.part[1].dweight);
}

}  // namespace esb
