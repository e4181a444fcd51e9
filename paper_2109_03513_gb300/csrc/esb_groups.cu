// esb_groups.cu -- projection onto ESB codes with a scale for every group of
// values of a row: alpha = max|x| / C, or the DDA scale of the group
// (Sec. III-D with the group as the tensor), then Eq. cheap_projection.
#include <cstdint>
#include <cuda_runtime.h>

#include "esb_internal.h"
#include "esb_rows.cuh"

namespace esb {

namespace {

constexpr int kGroupThreads = 256;

struct GroupArgs {
    const void* x;
    int64_t rows, cols, ldx, group, ngroups;
    uint32_t* codes;
    int64_t ldc;
    float* scales;
    int64_t lds;
    void* xq;
    int xq_type;
    int64_t ldq;
    int rule, xvec, qvec;
    float astar;
    QuantFmt f;
};

template <int B>
__device__ __forceinline__ void put_codes(const GroupArgs& a, int64_t row, int64_t vec, const uint32_t (&c)[8])
{
    uint32_t* p = a.codes + row * a.ldc;
    if (B == 4) {
        if (vec < a.ldc)
            p[vec] = c[0] | (c[1] << 4) | (c[2] << 8) | (c[3] << 12) | (c[4] << 16) | (c[5] << 20) | (c[6] << 24) | (c[7] << 28);
    } else {
        const int64_t w = 2 * vec;
        if (w < a.ldc) p[w] = c[0] | (c[1] << 8) | (c[2] << 16) | (c[3] << 24);
        if (w + 1 < a.ldc) p[w + 1] = c[4] | (c[5] << 8) | (c[6] << 16) | (c[7] << 24);
    }
}

template <int B>
__device__ __forceinline__ void project8(const GroupArgs& a, int64_t row, int64_t vec, const float (&v)[8], const GroupScale& s)
{
    uint32_t c[8];
    float q[8];
    const int64_t n = a.cols - vec * 8;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        c[i] = quantise(v[i], s, a.f, q[i]);
        q[i] = __fmul_rn(s.alpha, q[i]);
        if (i >= n) c[i] = a.f.zero_code;
    }
    put_codes<B>(a, row, vec, c);
    if (a.xq && n > 0) store8_any(a.xq, a.xq_type, row * a.ldq + vec * 8, n, a.qvec, q);
}

// alpha of a group of n values from its sums: the largest magnitude over C,
// or alpha* (spread + 1e-7) in fp32, spread the standard deviation about the
// group's own mean (signed) or the root mean square (unsigned).
__device__ __forceinline__ float absmax_scale(uint32_t mx, const QuantFmt& f) { return __fdiv_rn(__uint_as_float(mx), f.C); }

// A warp for each group, of any length: the values are read twice.
template <int TYPE, int B>
__global__ void __launch_bounds__(kGroupThreads) project_groups_kernel(const GroupArgs a)
{
    using T = Elem<TYPE>;
    griddep_wait();
    const int lane = threadIdx.x & 31;
    const int64_t warp = (int64_t)blockIdx.x * (kGroupThreads / 32) + (threadIdx.x >> 5);
    const int64_t nwarps = (int64_t)gridDim.x * (kGroupThreads / 32);
    const int64_t total = a.rows * a.ngroups;
    for (int64_t g = warp; g < total; g += nwarps) {
        const int64_t row = g / a.ngroups, gi = g - row * a.ngroups;
        const T* x = static_cast<const T*>(a.x) + row * a.ldx;
        const int64_t e0 = gi * a.group, e1 = min(e0 + a.group, a.cols);
        float v[8];
        float alpha;
        if (a.rule == ESB_SCALE_ABSMAX) {
            uint32_t mx = 0u;
            for (int64_t e = e0 + lane * 8; e < e1; e += 256) {
                load8_to(x + e, e1 - e, a.xvec, v);
#pragma unroll
                for (int i = 0; i < 8; i++) mx = max(mx, magnitude_bits(v[i], a.f.is_signed));
            }
            alpha = absmax_scale(__reduce_max_sync(0xffffffffu, mx), a.f);
        } else {
            float s1 = 0.0f, s2 = 0.0f;
            const float n = (float)(e1 - e0);
            float mean = 0.0f;
            if (a.f.is_signed) {
                for (int64_t e = e0 + lane * 8; e < e1; e += 256) {
                    load8_to(x + e, e1 - e, a.xvec, v);
#pragma unroll
                    for (int i = 0; i < 8; i++) s1 += v[i];
                }
                mean = warp_sum(s1) / n;
            }
            for (int64_t e = e0 + lane * 8; e < e1; e += 256) {
                load8_to(x + e, e1 - e, a.xvec, v);
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const float d = e + i < e1 ? v[i] - mean : 0.0f;
                    s2 = fmaf(d, d, s2);
                }
            }
            alpha = __fmul_rn(a.astar, __fadd_rn(__fsqrt_rn(warp_sum(s2) / n), 1e-7f));
        }
        if (lane == 0) a.scales[row * a.lds + gi] = alpha;
        const GroupScale s = make_scale(alpha);
        // the last group's warp also writes the words past the columns
        const int64_t end = gi == a.ngroups - 1 ? a.ldc * (32 / B) : e0 + a.group;
        for (int64_t e = e0 + lane * 8; e < end; e += 256) {
            load8_to(x + e, e1 - e, a.xvec, v);
            project8<B>(a, row, e / 8, v, s);
        }
    }
}

}  // namespace

cudaError_t launch_project_groups(const void* x, int x_type, int64_t rows, int64_t cols, int64_t ldx, const esb_format& f,
                                  int rounding, int rule, int64_t group, double alpha_star, uint32_t* codes, int64_t ldc,
                                  float* scales, int64_t lds, void* xq, int xq_type, int64_t ldq, cudaStream_t st)
{
    GroupArgs a;
    auto rows16 = [](const void* p, int64_t ld, int type) {
        return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld * type_bytes(type) % 16 == 0;
    };
    a.x = x; a.rows = rows; a.cols = cols; a.ldx = ldx;
    a.group = group > 0 && group < cols ? group : (cols + 31) / 32 * 32;
    a.ngroups = (cols + a.group - 1) / a.group;
    a.codes = codes; a.ldc = ldc; a.scales = scales; a.lds = lds;
    a.xq = xq; a.xq_type = xq_type; a.ldq = ldq;
    a.rule = rule; a.astar = (float)alpha_star;
    a.xvec = rows16(x, ldx, x_type);
    a.qvec = xq && rows16(xq, ldq, xq_type);
    a.f = make_quant_fmt(f, rounding);
    const int64_t total = rows * a.ngroups;
    const int64_t per = kGroupThreads / 32;
    int64_t blocks = (total + per - 1) / per;
    const int64_t cap = (int64_t)device_sm_count() * 8;
    if (blocks > cap) blocks = cap;
    using Kernel = void (*)(const GroupArgs);
    static const Kernel kernels[3][2] = {{project_groups_kernel<ESB_F32, 4>, project_groups_kernel<ESB_F32, 8>},
                                         {project_groups_kernel<ESB_F16, 4>, project_groups_kernel<ESB_F16, 8>},
                                         {project_groups_kernel<ESB_BF16, 4>, project_groups_kernel<ESB_BF16, 8>}};
    return launch_pdl(kernels[x_type][f.b == 8], dim3((unsigned)blocks), dim3(kGroupThreads), 0, st, a);
}

}  // namespace esb
