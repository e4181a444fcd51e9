// esb_norm.cu -- root-mean-square norm with the residual's addition, its
// output plain or in ESB codes with scales, and its gradient.
#include <cstdint>
#include <type_traits>
#include <cuda_runtime.h>

#include "esb_internal.h"
#include "esb_rows.cuh"

namespace esb {

namespace {

constexpr int kNormThreads = 256;

struct NormArgs {
    int64_t rows, cols;
    esb_norm n;
    int64_t group, ngroups;     // columns of a group (a multiple of 32) and groups of a row; 0 without codes
    int xvec, rvec, hvec, yvec, qvec, wvec, cvec;
    QuantFmt f;
};

template <int NW>
__device__ __forceinline__ float block_sum(float v, float* sh)
{
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < NW; i++) t += sh[i];
    return t;
}

template <int NW>
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t* sh)
{
    v = __reduce_max_sync(0xffffffffu, v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    uint32_t t = 0u;
#pragma unroll
    for (int i = 0; i < NW; i++) t = max(t, sh[i]);
    return t;
}

// Codes (and values) of the eight values y at column e of a row.
__device__ __forceinline__ void put_codes8(const NormArgs& a, int64_t row, int64_t e, const float (&y)[8], const GroupScale& s)
{
    uint32_t w[2];
    float q[8];
    const int n = left_of(a.cols, e);
    quantise8<8, false>(y, s, a.f, w, q);
    if (n < 8) zero_past<8>(w, n, a.f);
    uint32_t* p = a.n.codes + row * a.n.ldc + e / 4;
    if (a.cvec && e / 4 + 1 < a.n.ldc) {
        *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    } else {
        p[0] = w[0];
        if (e / 4 + 1 < a.n.ldc) p[1] = w[1];
    }
    if (!a.n.yq || n <= 0) return;
    element_values(y, s, a.f, q);
    store8_any(a.n.yq, a.n.y_type, row * a.n.ldq + e, n, a.qvec, q);
}

// A block for each row, of any length: every pass reads the row again, and
// only the last one writes, each value by the thread that has read it (so h
// may lie on x or on the residual).
template <int TYPE>
__global__ void __launch_bounds__(kNormThreads) rmsnorm_kernel(const NormArgs a)
{
    using T = Elem<TYPE>;
    constexpr int NW = kNormThreads / 32;
    __shared__ float shf[NW];
    __shared__ uint32_t shu[NW];
    griddep_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(a.n.x) + row * a.n.ldx;
        const T* r = a.n.residual ? static_cast<const T*>(a.n.residual) + row * a.n.ldr : nullptr;
        auto sum8 = [&](int64_t e, float (&z)[8]) {
            load8_to(x + e, left_of(a.cols, e), a.xvec, z);
            if (r) {
                float t[8];
                load8_to(r + e, left_of(a.cols, e), a.rvec, t);
#pragma unroll
                for (int i = 0; i < 8; i++) z[i] = __fadd_rn(z[i], t[i]);
            }
        };
        float z[8], w[8], y[8];
        float ss = 0.0f;
        for (int64_t e = threadIdx.x * 8; e < a.cols; e += kNormThreads * 8) {
            sum8(e, z);
#pragma unroll
            for (int i = 0; i < 8; i++) ss = fmaf(z[i], z[i], ss);
        }
        ss = block_sum<NW>(ss, shf);
        const float rstd = __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(__fdiv_rn(ss, (float)a.cols), a.n.eps)));
        if (a.n.rstd && threadIdx.x == 0) a.n.rstd[row] = rstd;
        auto norm8 = [&](int64_t e) {
            sum8(e, z);
            if (a.n.weight) load8_any(a.n.weight, a.n.w_type, e, left_of(a.cols, e), a.wvec, w);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                y[i] = __fmul_rn(z[i], rstd);
                if (a.n.weight) y[i] = __fmul_rn(y[i], w[i]);
            }
        };
        auto put8 = [&](int64_t e) {
            if (a.n.h) store8_to(static_cast<T*>(a.n.h) + row * a.n.ldh + e, left_of(a.cols, e), a.hvec, z);
            if (a.n.y) store8_any(a.n.y, a.n.y_type, row * a.n.ldy + e, left_of(a.cols, e), a.yvec, y);
        };
        if (!a.ngroups) {
            for (int64_t e = threadIdx.x * 8; e < a.cols; e += kNormThreads * 8) {
                norm8(e);
                put8(e);
            }
            continue;
        }
        // one group for the row: all threads; else a warp for each group
        const bool whole = a.ngroups == 1;
        for (int64_t g = whole ? 0 : warp; g < a.ngroups; g += NW) {
            const int64_t e0 = g * a.group, e1 = min(e0 + a.group, a.cols);
            const int64_t first = e0 + (whole ? (int)threadIdx.x : lane) * 8, step = whole ? kNormThreads * 8 : 256;
            uint32_t mx = 0u;
            for (int64_t e = first; e < e1; e += step) {
                norm8(e);
#pragma unroll
                for (int i = 0; i < 8; i++) mx = max(mx, magnitude_bits(y[i], a.f.is_signed));
            }
            mx = whole ? block_max<NW>(mx, shu) : __reduce_max_sync(0xffffffffu, mx);
            const float alpha = absmax_scale(mx, a.f);
            if (first == e0) a.n.scales[row * a.n.lds + g] = alpha;
            const GroupScale s = make_scale(alpha, a.f);
            const int64_t end = g == a.ngroups - 1 ? a.n.ldc * 4 : e0 + a.group;
            for (int64_t e = first; e < end; e += step) {
                norm8(e);
                if (e < a.cols) put8(e);
                put_codes8(a, row, e, y, s);
            }
        }
    }
}

// ------------------------------------------------------- rows in registers

// A row of up to 16 TPR values by TPR threads, 16 a thread, held in registers
// from its one read to its last write; the next row is on its way meanwhile.
// A group of codes is 2 to 16 lanes (32 to 256 values), or the row.  Many rows
// are bound by instructions and HBM alike: 8192 x 4096 bf16 with residual,
// codes and values (9 bytes for a value of x, 302 MB, 45 us at the copy rate)
// 58 us with two blocks of 256 on an SM, 66 with three; 62 with a branch at every
// eight's kind and stores.  Few rows are bound by latency: one row of 4096
// takes 3.2 us.
template <int TYPE, int TPR>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR, TPR >= 512 ? 1 : (TPR < 256 ? 4 : 2)) rmsnorm_rows_kernel(const NormArgs a)
{
    using T = Elem<TYPE>;
    constexpr int THREADS = TPR < 128 ? 128 : TPR, PER = THREADS / TPR, NW = TPR / 32;
    constexpr bool AHEAD = TPR <= 512;                  // 1024 threads have 64 registers each: no next row, no weights
    __shared__ float shf[2][NW];
    __shared__ uint32_t shu[2][NW];
    griddep_wait();
    const int t = threadIdx.x % TPR, lanes = (int)a.group / 16, e = t * 16;
    const int n = left_of(a.cols, e);
    const float inv_cols = 1.0f / (float)a.cols;
    int64_t row = (int64_t)blockIdx.x * PER + threadIdx.x / TPR;
    const int64_t step = (int64_t)gridDim.x * PER;
    const T* px = static_cast<const T*>(a.n.x) + row * a.n.ldx + e;
    const T* pr = static_cast<const T*>(a.n.residual) + row * a.n.ldr + e;
    Raw8<T> rx[2], rr[2];
    auto load = [&](bool on) {
        const int k = on ? n : 0;
        rx[0].load(px, k, a.xvec);
        rx[1].load(px + 8, k - 8, a.xvec);
        if (a.n.residual) {
            rr[0].load(pr, k, a.rvec);
            rr[1].load(pr + 8, k - 8, a.rvec);
        }
        px += step * a.n.ldx;
        pr += step * a.n.ldr;
    };
    float w[2][8];
    auto weights = [&]() {
#pragma unroll
        for (int v = 0; v < 2; v++) {
            if (a.n.weight) {
                load8_any(a.n.weight, a.n.w_type, e + 8 * v, n - 8 * v, a.wvec, w[v]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; i++) w[v][i] = 1.0f;
            }
        }
    };
    if (AHEAD) {
        load(row < a.rows);
        weights();
    }
    // whole sixteens of a signed set, written by vectors and with values of x's
    // type, take few branches
    const bool straight = n >= 16 && a.f.plain && a.cvec && (!a.n.yq || (a.n.y_type == TYPE && a.qvec));
    int flip = 0;
    // a block's rows go on together, so that every thread meets every barrier
    for (int64_t first = (int64_t)blockIdx.x * PER; first < a.rows; first += step, row += step, flip ^= 1) {
        const bool on = PER == 1 || row < a.rows;
        if (!AHEAD) load(on);
        float z[2][8];
#pragma unroll
        for (int v = 0; v < 2; v++) {
            rx[v].values(z[v]);
            if (a.n.residual) {
                float u[8];
                rr[v].values(u);
#pragma unroll
                for (int i = 0; i < 8; i += 2) split(add2(pair_of(z[v][i], z[v][i + 1]), pair_of(u[i], u[i + 1])), z[v][i], z[v][i + 1]);
            }
        }
        if (AHEAD) load(row + step < a.rows);
        Pair sq = pair_of(0.0f, 0.0f);
#pragma unroll
        for (int v = 0; v < 2; v++)
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const Pair p = pair_of(z[v][i], z[v][i + 1]);
                sq = fma2(p, p, sq);
            }
        float s0, s1;
        split(sq, s0, s1);
        float ss = warp_sum(s0 + s1);
        if constexpr (NW > 1) {
            if ((threadIdx.x & 31) == 0) shf[flip][threadIdx.x >> 5] = ss;
            __syncthreads();
            ss = 0.0f;
#pragma unroll
            for (int i = 0; i < NW; i++) ss += shf[flip][i];
        }
        const float rstd = __frsqrt_rn(fmaf(ss, inv_cols, a.n.eps));
        if (!on) continue;                              // only where a row is a warp: no barrier below
        if (a.n.rstd && t == 0) a.n.rstd[row] = rstd;
        if (a.n.h) {
            T* h = static_cast<T*>(a.n.h) + row * a.n.ldh + e;
            store8_to(h, n, a.hvec, z[0]);
            store8_to(h + 8, n - 8, a.hvec, z[1]);
        }
        if (!AHEAD) weights();
#pragma unroll
        for (int v = 0; v < 2; v++)
#pragma unroll
            for (int i = 0; i < 8; i += 2)
                split(mul2(mul2(pair_of(z[v][i], z[v][i + 1]), pair_of(rstd, rstd)), pair_of(w[v][i], w[v][i + 1])), z[v][i], z[v][i + 1]);
        if (a.n.y) {
            store8_any(a.n.y, a.n.y_type, row * a.n.ldy + e, n, a.yvec, z[0]);
            store8_any(a.n.y, a.n.y_type, row * a.n.ldy + e + 8, n - 8, a.yvec, z[1]);
        }
        if (!a.ngroups) continue;
        // what lies past the row is 0 times rstd: 0, or NaN as the whole row
        uint32_t mx = 0u;
#pragma unroll
        for (int v = 0; v < 2; v++) mx = max(mx, largest_of8(z[v], a.f.is_signed));
        if (a.ngroups > 1) {
            for (int o = lanes / 2; o > 0; o >>= 1) mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        } else {
            mx = __reduce_max_sync(0xffffffffu, mx);
            if constexpr (NW > 1) {
                if ((threadIdx.x & 31) == 0) shu[flip][threadIdx.x >> 5] = mx;
                __syncthreads();
#pragma unroll
                for (int i = 0; i < NW; i++) mx = max(mx, shu[flip][i]);
            }
        }
        const float alpha = absmax_scale(mx, a.f);
        const int64_t left = a.n.ldc - (int64_t)t * 4;  // words of the row from this thread's first one on
        if (left > 0) {
            if (a.ngroups == 1) {
                if (t == 0) a.n.scales[row * a.n.lds] = alpha;
            } else if (t % lanes == 0 && n > 0) {
                a.n.scales[row * a.n.lds + t / lanes] = alpha;
            }
            const GroupScale s = make_scale(alpha, a.f);
            uint32_t c[2][2];
            uint32_t* p = a.n.codes + row * a.n.ldc + t * 4;
            if (straight && s.fast) {
                T* yq = static_cast<T*>(a.n.yq) + row * a.n.ldq + e;
                auto sixteen = [&](auto linear) {
#pragma unroll
                    for (int v = 0; v < 2; v++) {
                        float q[8];
                        places8<8, decltype(linear)::value, false>(z[v], s, a.f, c[v], q);
                        codes8<8>(z[v], a.f, c[v]);
                        if (a.n.yq) {
                            element_values(z[v], s, a.f, q);
                            store8<T>(yq + 8 * v, q);
                        }
                    }
                };
                if (a.f.linear) sixteen(std::true_type());
                else sixteen(std::false_type());
                *reinterpret_cast<uint4*>(p) = make_uint4(c[0][0], c[0][1], c[1][0], c[1][1]);
            } else {
#pragma unroll
                for (int v = 0; v < 2; v++) {
                    float q[8];
                    quantise8<8, false>(z[v], s, a.f, c[v], q);
                    if (n - 8 * v < 8) zero_past<8>(c[v], n - 8 * v, a.f);
                    if (a.n.yq) {
                        element_values(z[v], s, a.f, q);
                        store8_any(a.n.yq, a.n.y_type, row * a.n.ldq + e + 8 * v, n - 8 * v, a.qvec, q);
                    }
                }
                if (a.cvec && left >= 4) {
                    *reinterpret_cast<uint4*>(p) = make_uint4(c[0][0], c[0][1], c[1][0], c[1][1]);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        if (i < left) p[i] = c[i / 2][i % 2];
                }
            }
        }
        // words past those that the threads' values reach (a long row stride)
        for (int64_t i = (int64_t)TPR * 4 + t; i < a.n.ldc; i += TPR) a.n.codes[row * a.n.ldc + i] = a.f.zero_code * 0x01010101u;
    }
}

// ------------------------------------------------------------- backward

struct NormGradArgs {
    int64_t rows, cols;
    esb_norm_grad n;
    int gvec, hvec, dhvec, dxvec, wvec;
    float* part;                // parts x cols partial sums of dweight
    int parts;
};

// dx = rstd (d - n mean(d n)) + dh with n = h rstd, d = dy w: a block for
// each row of any length, which it reads twice.
template <int TYPE>
__global__ void __launch_bounds__(kNormThreads) rmsnorm_dx_kernel(const NormGradArgs a)
{
    using T = Elem<TYPE>;
    constexpr int NW = kNormThreads / 32;
    __shared__ float shf[NW];
    griddep_wait();
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* h = static_cast<const T*>(a.n.h) + row * a.n.ldh;
        const float rstd = a.n.rstd[row];
        float n[8], d[8], t[8];
        auto both8 = [&](int64_t e) {
            load8_to(h + e, left_of(a.cols, e), a.hvec, n);
            load8_any(a.n.dy, a.n.g_type, row * a.n.ldg + e, left_of(a.cols, e), a.gvec, d);
            if (a.n.weight) load8_any(a.n.weight, a.n.w_type, e, left_of(a.cols, e), a.wvec, t);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                n[i] *= rstd;
                if (a.n.weight) d[i] *= t[i];
            }
        };
        float s = 0.0f;
        for (int64_t e = threadIdx.x * 8; e < a.cols; e += kNormThreads * 8) {
            both8(e);
#pragma unroll
            for (int i = 0; i < 8; i++) s = fmaf(d[i], n[i], s);
        }
        const float m = block_sum<NW>(s, shf) / (float)a.cols;
        for (int64_t e = threadIdx.x * 8; e < a.cols; e += kNormThreads * 8) {
            both8(e);
            if (a.n.dh) load8_to(static_cast<const T*>(a.n.dh) + row * a.n.lddh + e, left_of(a.cols, e), a.dhvec, t);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                d[i] = rstd * fmaf(-n[i], m, d[i]);
                if (a.n.dh) d[i] += t[i];
            }
            store8_to(static_cast<T*>(a.n.dx) + row * a.n.lddx + e, left_of(a.cols, e), a.dxvec, d);
        }
    }
}

// dweight of such rows: block (x, y) adds dy n over rows y, y + parts, ... of
// its columns.
template <int TYPE>
__global__ void __launch_bounds__(kNormThreads) rmsnorm_dw_kernel(const NormGradArgs a)
{
    using T = Elem<TYPE>;
    griddep_wait();
    const int64_t e = ((int64_t)blockIdx.x * kNormThreads + threadIdx.x) * 8;
    if (e >= a.cols) return;
    float s[8] = {}, n[8], d[8];
    for (int64_t row = blockIdx.y; row < a.rows; row += a.parts) {
        const float rstd = a.n.rstd[row];
        load8_to(static_cast<const T*>(a.n.h) + row * a.n.ldh + e, left_of(a.cols, e), a.hvec, n);
        load8_any(a.n.dy, a.n.g_type, row * a.n.ldg + e, left_of(a.cols, e), a.gvec, d);
#pragma unroll
        for (int i = 0; i < 8; i++) s[i] = fmaf(d[i], n[i] * rstd, s[i]);
    }
    store8_to(a.part + (int64_t)blockIdx.y * a.cols + e, left_of(a.cols, e), false, s);
}

// Both for rows in registers: a thread keeps its columns of every row of its
// block, their weights and their part of dweight, and loads the next row while
// it works on this one.  8192 x 4096 bf16, 268 MB of reads and writes (the
// kernels above read the gradient and h twice): forward and backward together
// 100 us with two blocks of 512 on an SM, 117 with one; 79 at the copy rate.
template <int TYPE, int GTYPE, int TPR, int NV>
__global__ void __launch_bounds__(TPR, TPR >= 1024 ? 1 : (TPR < 128 ? 8 : (TYPE == ESB_F32 ? 512 : 1024) / TPR)) rmsnorm_grad_rows_kernel(const NormGradArgs a)
{
    using T = Elem<TYPE>;
    using G = Elem<GTYPE>;
    constexpr int NW = TPR / 32;
    __shared__ float shf[2][NW];
    griddep_wait();
    float w[NV][8], dw[NV][8];
    int64_t e[NV];
#pragma unroll
    for (int v = 0; v < NV; v++) {
        e[v] = (int64_t)(v * TPR + threadIdx.x) * 8;
#pragma unroll
        for (int i = 0; i < 8; i++) { w[v][i] = 1.0f; dw[v][i] = 0.0f; }
        if (NV == 1 && a.n.weight) load8_any(a.n.weight, a.n.w_type, e[v], left_of(a.cols, e[v]), a.wvec, w[v]);
    }
    float rstd = 0.0f;
    Raw8<T> rh[NV], rt[NV];                             // the next row, on its way
    Raw8<G> rg[NV];
    auto load = [&](int64_t row) {
        const bool on = row < a.rows;
        if (on) rstd = a.n.rstd[row];
#pragma unroll
        for (int v = 0; v < NV; v++) {
            const int left = on ? left_of(a.cols, e[v]) : 0;
            rh[v].load(static_cast<const T*>(a.n.h) + row * a.n.ldh + e[v], left, a.hvec);
            rg[v].load(static_cast<const G*>(a.n.dy) + row * a.n.ldg + e[v], left, a.gvec);
            if (NV == 1 && a.n.dh) rt[v].load(static_cast<const T*>(a.n.dh) + row * a.n.lddh + e[v], left, a.dhvec);
        }
    };
    load(blockIdx.x);
    int flip = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, flip ^= 1) {
        const float rs = rstd;
        float n[NV][8], d[NV][8], t[8];
#pragma unroll
        for (int v = 0; v < NV; v++) {
            rh[v].values(n[v]);
            rg[v].values(d[v]);
        }
        if (NV == 1 && a.n.dh) rt[0].values(t);
        load(row + gridDim.x);
        float s = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; v++) {
            // of two vectors the weights (and dh below) are not kept: 64 registers a thread
            if (NV > 1 && a.n.weight) load8_any(a.n.weight, a.n.w_type, e[v], left_of(a.cols, e[v]), a.wvec, t);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                n[v][i] *= rs;
                dw[v][i] = fmaf(d[v][i], n[v][i], dw[v][i]);
                if (NV == 1) d[v][i] *= w[v][i];
                else if (a.n.weight) d[v][i] *= t[i];
                s = fmaf(d[v][i], n[v][i], s);
            }
        }
        s = warp_sum(s);
        if ((threadIdx.x & 31) == 0) shf[flip][threadIdx.x >> 5] = s;
        __syncthreads();
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < NW; i++) s += shf[flip][i];
        const float m = s / (float)a.cols;
#pragma unroll
        for (int v = 0; v < NV; v++) {
            if (NV > 1 && a.n.dh) load8_to(static_cast<const T*>(a.n.dh) + row * a.n.lddh + e[v], left_of(a.cols, e[v]), a.dhvec, t);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                d[v][i] = rs * fmaf(-n[v][i], m, d[v][i]);
                if (a.n.dh) d[v][i] += t[i];
            }
            store8_to(static_cast<T*>(a.n.dx) + row * a.n.lddx + e[v], left_of(a.cols, e[v]), a.dxvec, d[v]);
        }
    }
    if (a.part) {
#pragma unroll
        for (int v = 0; v < NV; v++) store8_to(a.part + blockIdx.x * a.cols + e[v], left_of(a.cols, e[v]), (a.cols & 3) == 0, dw[v]);
    }
}

// The parts' sums, in a fixed order: a warp's lanes take 32 columns, the
// warps every 8th part, then the warps' sums in turn.
__global__ void __launch_bounds__(kNormThreads) rmsnorm_dw_join_kernel(const float* part, int parts, int64_t cols, float* dw)
{
    __shared__ float sh[kNormThreads / 32][32];
    griddep_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (c < cols)
        for (int p = warp; p < parts; p += kNormThreads / 32) s += part[p * cols + c];
    sh[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && c < cols) {
#pragma unroll
        for (int i = 1; i < kNormThreads / 32; i++) s += sh[i][lane];
        dw[c] = s;
    }
}

using NormKernel = void (*)(const NormArgs);
struct NormPlan {
    NormKernel kernel;
    int tpr;
};
template <int TYPE> NormPlan norm_plan(int64_t cols)
{
    if (cols <= 512) return {rmsnorm_rows_kernel<TYPE, 32>, 32};
    if (cols <= 2048) return {rmsnorm_rows_kernel<TYPE, 128>, 128};
    if (cols <= 4096) return {rmsnorm_rows_kernel<TYPE, 256>, 256};
    if (cols <= 8192) return {rmsnorm_rows_kernel<TYPE, 512>, 512};
    if (cols <= 16384) return {rmsnorm_rows_kernel<TYPE, 1024>, 1024};
    return {rmsnorm_kernel<TYPE>, 0};
}

bool rows16(const void* p, int64_t ld, int type)
{
    return p && (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld * type_bytes(type) % 16 == 0;
}

using GradKernel = void (*)(const NormGradArgs);
struct GradPlan {
    GradKernel kernel;
    int tpr;
};
template <int TYPE, int GTYPE> GradPlan grad_plan(int64_t cols)
{
    if (cols <= 256) return {rmsnorm_grad_rows_kernel<TYPE, GTYPE, 32, 1>, 32};
    if (cols <= 1024) return {rmsnorm_grad_rows_kernel<TYPE, GTYPE, 128, 1>, 128};
    if (cols <= 2048) return {rmsnorm_grad_rows_kernel<TYPE, GTYPE, 256, 1>, 256};
    if (cols <= 4096) return {rmsnorm_grad_rows_kernel<TYPE, GTYPE, 512, 1>, 512};
    if (cols <= 8192) return {rmsnorm_grad_rows_kernel<TYPE, GTYPE, 1024, 1>, 1024};
    if (cols <= 16384) return {rmsnorm_grad_rows_kernel<TYPE, GTYPE, 1024, 2>, 1024};
    return {nullptr, 0};
}

// Parts of dweight, one for each block: as many as the SMs hold (fewer where
// a part would get less than 4 rows).
int dw_parts(int64_t rows, int64_t cols)
{
    const GradPlan p = grad_plan<ESB_BF16, ESB_BF16>(cols);
    int64_t n = p.tpr ? (int64_t)device_sm_count() * (p.tpr >= 1024 ? 1 : 1024 / p.tpr) : 64;
    if (n > (rows + 3) / 4) n = (rows + 3) / 4;
    return (int)(n < 1 ? 1 : n);
}

}  // namespace

cudaError_t launch_rmsnorm(int64_t rows, int64_t cols, const esb_norm& n, cudaStream_t st)
{
    NormArgs a;
    a.rows = rows; a.cols = cols; a.n = n;
    a.group = a.ngroups = 0;
    a.f = make_quant_fmt(n.codes ? n.fmt : esb_format{8, 6, 1}, n.rounding);
    if (n.codes) {
        a.group = n.group > 0 && n.group < cols ? n.group : (cols + 31) / 32 * 32;
        a.ngroups = (cols + a.group - 1) / a.group;
    }
    a.xvec = rows16(n.x, n.ldx, n.x_type);
    a.rvec = rows16(n.residual, n.ldr, n.x_type);
    a.hvec = rows16(n.h, n.ldh, n.x_type);
    a.yvec = rows16(n.y, n.ldy, n.y_type);
    a.qvec = rows16(n.yq, n.ldq, n.y_type);
    a.wvec = rows16(n.weight, 0, n.w_type);
    a.cvec = rows16(n.codes, n.ldc, ESB_F32);
    const int64_t sms = device_sm_count();
    static NormPlan (*const plans[3])(int64_t) = {norm_plan<ESB_F32>, norm_plan<ESB_F16>, norm_plan<ESB_BF16>};
    static const NormKernel any[3] = {rmsnorm_kernel<ESB_F32>, rmsnorm_kernel<ESB_F16>, rmsnorm_kernel<ESB_BF16>};
    const NormPlan p = plans[n.x_type](cols);
    const bool lanes = a.ngroups <= 1 || a.group == 32 || a.group == 64 || a.group == 128 || a.group == 256;
    if (!p.tpr || !lanes) {
        const int64_t cap = sms * 8;
        return launch_pdl(any[n.x_type], dim3((unsigned)(rows < cap ? rows : cap)), dim3(kNormThreads), 0, st, a);
    }
    const int threads = p.tpr < 128 ? 128 : p.tpr;
    int64_t blocks = (rows + threads / p.tpr - 1) / (threads / p.tpr);
    const int64_t cap = sms * (threads >= 1024 ? 1 : 512 / threads);   // what the SMs hold at once: each block keeps its weights
    if (blocks > cap) blocks = cap;
    return launch_pdl(p.kernel, dim3((unsigned)blocks), dim3((unsigned)threads), 0, st, a);
}

size_t rmsnorm_grad_workspace_bytes(int64_t rows, int64_t cols) { return sizeof(float) * (size_t)dw_parts(rows, cols) * (size_t)cols; }

cudaError_t launch_rmsnorm_grad(int64_t rows, int64_t cols, const esb_norm_grad& n, void* workspace, cudaStream_t st)
{
    NormGradArgs a;
    a.rows = rows; a.cols = cols; a.n = n;
    a.gvec = rows16(n.dy, n.ldg, n.g_type);
    a.hvec = rows16(n.h, n.ldh, n.x_type);
    a.dhvec = rows16(n.dh, n.lddh, n.x_type);
    a.dxvec = rows16(n.dx, n.lddx, n.x_type);
    a.wvec = rows16(n.weight, 0, n.w_type);
    a.part = n.dweight ? static_cast<float*>(workspace) : nullptr;
    a.parts = dw_parts(rows, cols);
    GradPlan p{nullptr, 0};
    if (n.g_type == n.x_type) {
        static GradPlan (*const same[3])(int64_t) = {grad_plan<ESB_F32, ESB_F32>, grad_plan<ESB_F16, ESB_F16>, grad_plan<ESB_BF16, ESB_BF16>};
        p = same[n.x_type](cols);
    }
    cudaError_t e = cudaSuccess;
    if (p.kernel) {
        e = launch_pdl(p.kernel, dim3((unsigned)a.parts), dim3((unsigned)p.tpr), 0, st, a);
    } else {
        static const GradKernel dxs[3] = {rmsnorm_dx_kernel<ESB_F32>, rmsnorm_dx_kernel<ESB_F16>, rmsnorm_dx_kernel<ESB_BF16>};
        static const GradKernel dws[3] = {rmsnorm_dw_kernel<ESB_F32>, rmsnorm_dw_kernel<ESB_F16>, rmsnorm_dw_kernel<ESB_BF16>};
        if (n.dweight) {
            // before dx, which may lie on the gradient or on h
            const unsigned bx = (unsigned)((cols + kNormThreads * 8 - 1) / (kNormThreads * 8));
            e = launch_pdl(dws[n.x_type], dim3(bx, (unsigned)a.parts), dim3(kNormThreads), 0, st, a);
            if (e != cudaSuccess) return e;
        }
        const int64_t cap = (int64_t)device_sm_count() * 8;
        e = launch_pdl(dxs[n.x_type], dim3((unsigned)(rows < cap ? rows : cap)), dim3(kNormThreads), 0, st, a);
    }
    if (e != cudaSuccess || !n.dweight) return e;
    return launch_pdl(rmsnorm_dw_join_kernel, dim3((unsigned)((cols + 31) / 32)), dim3(kNormThreads), 0, st, (const float*)a.part, a.parts,
                      cols, n.dweight);
}

}  // namespace esb
