// esb_norm.cu -- root-mean-square norm with the residual's addition, its
// output plain or in ESB codes with scales, and its gradient.
#include <cstdint>
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
    int xvec, rvec, hvec, yvec, qvec, wvec;
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
            load8_to(x + e, a.cols - e, a.xvec, z);
            if (r) {
                float t[8];
                load8_to(r + e, a.cols - e, a.rvec, t);
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
            if (a.n.weight) load8_any(a.n.weight, a.n.w_type, e, a.cols - e, a.wvec, w);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                y[i] = __fmul_rn(z[i], rstd);
                if (a.n.weight) y[i] = __fmul_rn(y[i], w[i]);
            }
        };
        auto put8 = [&](int64_t e) {
            if (a.n.h) store8_to(static_cast<T*>(a.n.h) + row * a.n.ldh + e, a.cols - e, a.hvec, z);
            if (a.n.y) store8_any(a.n.y, a.n.y_type, row * a.n.ldy + e, a.cols - e, a.yvec, y);
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
            const float alpha = __fdiv_rn(__uint_as_float(mx), a.f.C);
            if (first == e0) a.n.scales[row * a.n.lds + g] = alpha;
            const GroupScale s = make_scale(alpha);
            const int64_t end = g == a.ngroups - 1 ? a.n.ldc * 4 : e0 + a.group;
            for (int64_t e = first; e < end; e += step) {
                const int64_t n = a.cols - e;
                norm8(e);
                if (n > 0) put8(e);
                uint32_t c[8];
                float q[8];
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    c[i] = quantise(y[i], s, a.f, q[i]);
                    q[i] = __fmul_rn(alpha, q[i]);
                    if (i >= n) c[i] = a.f.zero_code;
                }
                uint32_t* cw = a.n.codes + row * a.n.ldc + e / 4;
                cw[0] = c[0] | (c[1] << 8) | (c[2] << 16) | (c[3] << 24);
                if (e / 4 + 1 < a.n.ldc) cw[1] = c[4] | (c[5] << 8) | (c[6] << 16) | (c[7] << 24);
                if (a.n.yq && n > 0) store8_any(a.n.yq, a.n.y_type, row * a.n.ldq + e, n, a.qvec, q);
            }
        }
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
// each row, which it reads twice.
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
            load8_to(h + e, a.cols - e, a.hvec, n);
            load8_any(a.n.dy, a.n.g_type, row * a.n.ldg + e, a.cols - e, a.gvec, d);
            if (a.n.weight) load8_any(a.n.weight, a.n.w_type, e, a.cols - e, a.wvec, t);
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
            if (a.n.dh) load8_to(static_cast<const T*>(a.n.dh) + row * a.n.lddh + e, a.cols - e, a.dhvec, t);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                d[i] = rstd * fmaf(-n[i], m, d[i]);
                if (a.n.dh) d[i] += t[i];
            }
            store8_to(static_cast<T*>(a.n.dx) + row * a.n.lddx + e, a.cols - e, a.dxvec, d);
        }
    }
}

// dweight: block (x, y) adds dy n over rows y, y + parts, ... of its columns.
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
        load8_to(static_cast<const T*>(a.n.h) + row * a.n.ldh + e, a.cols - e, a.hvec, n);
        load8_any(a.n.dy, a.n.g_type, row * a.n.ldg + e, a.cols - e, a.gvec, d);
#pragma unroll
        for (int i = 0; i < 8; i++) s[i] = fmaf(d[i], n[i] * rstd, s[i]);
    }
    store8_to(a.part + (int64_t)blockIdx.y * a.cols + e, a.cols - e, false, s);
}

// The parts' sums, in their order.
__global__ void __launch_bounds__(kNormThreads) rmsnorm_dw_join_kernel(const float* part, int parts, int64_t cols, float* dw)
{
    griddep_wait();
    const int64_t c = (int64_t)blockIdx.x * kNormThreads + threadIdx.x;
    if (c >= cols) return;
    float s = 0.0f;
    for (int p = 0; p < parts; p++) s += part[p * cols + c];
    dw[c] = s;
}

bool rows16(const void* p, int64_t ld, int type)
{
    return p && (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld * type_bytes(type) % 16 == 0;
}

int dw_parts(int64_t rows) { return (int)(rows < 64 ? 1 : (rows < 64 * 64 ? rows / 64 : 64)); }

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
    const int64_t cap = (int64_t)device_sm_count() * 8;
    const unsigned blocks = (unsigned)(rows < cap ? rows : cap);
    using Kernel = void (*)(const NormArgs);
    static const Kernel kernels[3] = {rmsnorm_kernel<ESB_F32>, rmsnorm_kernel<ESB_F16>, rmsnorm_kernel<ESB_BF16>};
    return launch_pdl(kernels[n.x_type], dim3(blocks), dim3(kNormThreads), 0, st, a);
}

size_t rmsnorm_grad_workspace_bytes(int64_t rows, int64_t cols) { return sizeof(float) * (size_t)dw_parts(rows) * (size_t)cols; }

cudaError_t launch_rmsnorm_grad(int64_t rows, int64_t cols, const esb_norm_grad& n, void* workspace, cudaStream_t st)
{
    NormGradArgs a;
    a.rows = rows; a.cols = cols; a.n = n;
    a.gvec = rows16(n.dy, n.ldg, n.g_type);
    a.hvec = rows16(n.h, n.ldh, n.x_type);
    a.dhvec = rows16(n.dh, n.lddh, n.x_type);
    a.dxvec = rows16(n.dx, n.lddx, n.x_type);
    a.wvec = rows16(n.weight, 0, n.w_type);
    a.part = static_cast<float*>(workspace);
    a.parts = dw_parts(rows);
    using Kernel = void (*)(const NormGradArgs);
    static const Kernel dxs[3] = {rmsnorm_dx_kernel<ESB_F32>, rmsnorm_dx_kernel<ESB_F16>, rmsnorm_dx_kernel<ESB_BF16>};
    static const Kernel dws[3] = {rmsnorm_dw_kernel<ESB_F32>, rmsnorm_dw_kernel<ESB_F16>, rmsnorm_dw_kernel<ESB_BF16>};
    cudaError_t e = cudaSuccess;
    if (n.dweight) {
        const unsigned bx = (unsigned)((cols + kNormThreads * 8 - 1) / (kNormThreads * 8));
        e = launch_pdl(dws[n.x_type], dim3(bx, (unsigned)a.parts), dim3(kNormThreads), 0, st, a);
        if (e != cudaSuccess) return e;
        e = launch_pdl(rmsnorm_dw_join_kernel, dim3((unsigned)((cols + kNormThreads - 1) / kNormThreads)), dim3(kNormThreads), 0, st,
                       (const float*)a.part, a.parts, cols, n.dweight);
        if (e != cudaSuccess) return e;
    }
    const int64_t cap = (int64_t)device_sm_count() * 8;
    return launch_pdl(dxs[n.x_type], dim3((unsigned)(rows < cap ? rows : cap)), dim3(kNormThreads), 0, st, a);
}

}  // namespace esb
