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
    int rule, xvec, qvec, cvec;
    float astar;
    QuantFmt f;
};

// Codes (and values) of the eight values v at place 8 vec of a row.
template <int B>
__device__ __forceinline__ void project8(const GroupArgs& a, int64_t row, int64_t vec, const float (&v)[8], const GroupScale& s)
{
    uint32_t w[B / 4];
    float q[8];
    const int64_t n = a.cols - vec * 8;
    quantise8<B>(v, s, a.f, w, q);
    if (n < 8) zero_past<B>(w, n, a.f);
    uint32_t* p = a.codes + row * a.ldc + vec * (B / 4);
    if (B == 8 && a.cvec && vec * 2 + 1 < a.ldc) {
        *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[B / 4 - 1]);
    } else {
#pragma unroll
        for (int i = 0; i < B / 4; i++)
            if (vec * (B / 4) + i < a.ldc) p[i] = w[i];
    }
    if (a.xq && n > 0) store8_any(a.xq, a.xq_type, row * a.ldq + vec * 8, n, a.qvec, q);
}

// alpha of a group of n values from its sums: the largest magnitude over C,
// or alpha* (spread + 1e-7) in fp32, spread the standard deviation about the
// group's own mean (signed) or the root mean square (unsigned).
__device__ __forceinline__ float absmax_scale(uint32_t mx, const QuantFmt& f) { return __fdiv_rn(__uint_as_float(mx), f.C); }

// A warp for each group, of any length: the values are read twice or, for
// the DDA scale, three times.
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
        const GroupScale s = make_scale(alpha, a.f);
        // the last group's warp also writes the words past the columns
        const int64_t end = gi == a.ngroups - 1 ? a.ldc * (32 / B) : e0 + a.group;
        for (int64_t e = e0 + lane * 8; e < end; e += 256) {
            load8_to(x + e, e1 - e, a.xvec, v);
            project8<B>(a, row, e / 8, v, s);
        }
    }
}

// Groups of 32, 64, 128 or 256 values: 8 a lane, LANES lanes to a group, the
// values in registers from the scale to the codes, kVecs vectors of 8 in
// flight.  Rows are padded to whole groups (`vecs` vectors); a thread goes on
// by dr rows and dv vectors.  16384 x 4096 bf16 with values: 302 MB of reads
// and writes; two passes by a warp for each group took 422 us.
constexpr int kVecs = 4;
template <int TYPE, int B, int LANES>
__global__ void __launch_bounds__(kGroupThreads) project_small_groups_kernel(const GroupArgs a, int64_t vecs, int64_t dr, int64_t dv)
{
    using T = Elem<TYPE>;
    griddep_wait();
    const int64_t at = (int64_t)blockIdx.x * kGroupThreads + threadIdx.x;
    int64_t row = at / vecs, vec = at - row * vecs;
    const int part = threadIdx.x % LANES;               // vecs and a block are whole groups
    auto total = [&](float v) {
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    };
    while (__any_sync(0xffffffffu, row < a.rows)) {
        float v[kVecs][8];
        int64_t rows[kVecs], at_vec[kVecs];
#pragma unroll
        for (int u = 0; u < kVecs; u++) {
            rows[u] = row;
            at_vec[u] = vec;
            const int64_t n = row < a.rows ? a.cols - vec * 8 : 0;
            load8_to(static_cast<const T*>(a.x) + row * a.ldx + vec * 8, n, a.xvec, v[u]);
            row += dr;
            vec += dv;
            if (vec >= vecs) { vec -= vecs; row++; }
        }
#pragma unroll
        for (int u = 0; u < kVecs; u++) {
            float alpha;
            if (a.rule == ESB_SCALE_ABSMAX) {
                uint32_t mx = 0u;
#pragma unroll
                for (int i = 0; i < 8; i++) mx = max(mx, magnitude_bits(v[u][i], a.f.is_signed));
#pragma unroll
                for (int o = LANES / 2; o > 0; o >>= 1) mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, o));
                alpha = absmax_scale(mx, a.f);
            } else {
                const int64_t left = a.cols - (at_vec[u] - part) * 8;
                const float n = (float)(left < 8 * LANES ? left : 8 * LANES);
                float mean = 0.0f, s2 = 0.0f;
                if (a.f.is_signed) {
#pragma unroll
                    for (int i = 0; i < 8; i++) mean += v[u][i];
                    mean = total(mean) / n;
                }
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const float d = at_vec[u] * 8 + i < a.cols ? v[u][i] - mean : 0.0f;
                    s2 = fmaf(d, d, s2);
                }
                alpha = __fmul_rn(a.astar, __fadd_rn(__fsqrt_rn(total(s2) / n), 1e-7f));
            }
            if (rows[u] >= a.rows) continue;
            const int64_t gi = at_vec[u] / LANES;
            if (part == 0 && gi < a.ngroups) a.scales[rows[u] * a.lds + gi] = alpha;
            project8<B>(a, rows[u], at_vec[u], v[u], make_scale(alpha, a.f));
        }
    }
}

using GroupKernel = void (*)(const GroupArgs);
using SmallKernel = void (*)(const GroupArgs, int64_t, int64_t, int64_t);
template <int TYPE, int B> SmallKernel small_kernel(int lanes)
{
    switch (lanes) {
    case 4: return project_small_groups_kernel<TYPE, B, 4>;
    case 8: return project_small_groups_kernel<TYPE, B, 8>;
    case 16: return project_small_groups_kernel<TYPE, B, 16>;
    default: return project_small_groups_kernel<TYPE, B, 32>;
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
    a.cvec = (reinterpret_cast<uintptr_t>(codes) & 7u) == 0 && ldc % 2 == 0;
    const int64_t sms = device_sm_count();
    if (a.group == 32 || a.group == 64 || a.group == 128 || a.group == 256) {
        const int lanes = (int)a.group / 8;
        static SmallKernel (*const pick[3][2])(int) = {{small_kernel<ESB_F32, 4>, small_kernel<ESB_F32, 8>},
                                                       {small_kernel<ESB_F16, 4>, small_kernel<ESB_F16, 8>},
                                                       {small_kernel<ESB_BF16, 4>, small_kernel<ESB_BF16, 8>}};
        // vectors of a row up to its last code word, in whole groups
        const int64_t vecs0 = f.b == 4 ? ldc : (ldc + 1) / 2;
        const int64_t vecs = (vecs0 + lanes - 1) / lanes * lanes, total = rows * vecs;
        int64_t blocks = (total + kGroupThreads - 1) / kGroupThreads;
        const int64_t cap = sms * 6;
        if (blocks > cap) blocks = cap;
        const int64_t threads = blocks * kGroupThreads;
        return launch_pdl(pick[x_type][f.b == 8](lanes), dim3((unsigned)blocks), dim3(kGroupThreads), 0, st, a, vecs, threads / vecs,
                          threads % vecs);
    }
    const int64_t total = rows * a.ngroups;
    const int64_t per = kGroupThreads / 32;
    int64_t blocks = (total + per - 1) / per;
    const int64_t cap = sms * 8;
    if (blocks > cap) blocks = cap;
    static const GroupKernel kernels[3][2] = {{project_groups_kernel<ESB_F32, 4>, project_groups_kernel<ESB_F32, 8>},
                                              {project_groups_kernel<ESB_F16, 4>, project_groups_kernel<ESB_F16, 8>},
                                              {project_groups_kernel<ESB_BF16, 4>, project_groups_kernel<ESB_BF16, 8>}};
    return launch_pdl(kernels[x_type][f.b == 8], dim3((unsigned)blocks), dim3(kGroupThreads), 0, st, a);
}

}  // namespace esb
