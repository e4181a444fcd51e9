// esb_matvec.cu -- few rows times a matrix of 4-bit ESB codes with group
// scales: y[m][n] = bias[n] + sum_g s[n][g] sum_{k in g} q(W[n][k]) x[m][k].
#include <cstdint>
#include <cuda_runtime.h>

#include "esb_internal.h"
#include "esb_rows.cuh"

namespace esb {

namespace {

constexpr int kMvThreads = 256;
constexpr int kMvRows = 4;

struct MvArgs {
    int64_t M, N, K;
    const void* x;
    int64_t ldx;
    esb_coded xc;               // for x_type ESB_CODES
    esb_coded w;
    int64_t xgroup;
    const float* bias;
    void* y;
    int y_type;
    int64_t ldy;
    int xvec;
};

__device__ __forceinline__ void put_y(const MvArgs& a, int64_t m, int64_t n, float v)
{
    if (a.bias) v += a.bias[n];
    const int64_t at = m * a.ldy + n;
    if (a.y_type == ESB_F32) static_cast<float*>(a.y)[at] = v;
    else if (a.y_type == ESB_F16) static_cast<__half*>(a.y)[at] = __float2half_rn(v);
    else static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v);
}

// A warp for each column n, kMvRows rows at a time.
template <int XT>
__global__ void __launch_bounds__(kMvThreads) matvec_kernel(const MvArgs a)
{
    __shared__ float tab[16], xtab[256];
    griddep_wait();
    if (threadIdx.x < 16) tab[threadIdx.x] = code_value(threadIdx.x, 4, a.w.fmt.k);
    if (XT == ESB_CODES) xtab[threadIdx.x] = code_value(threadIdx.x, 8, a.xc.fmt.k);
    __syncthreads();
    const int lane = threadIdx.x & 31;
    const int64_t n = (int64_t)blockIdx.x * (kMvThreads / 32) + (threadIdx.x >> 5);
    if (n >= a.N) return;
    const uint32_t* w = a.w.codes + n * a.w.ld;
    const float* ws = a.w.scales + n * a.w.lds;
    for (int64_t m0 = (int64_t)blockIdx.y * kMvRows; m0 < a.M; m0 += (int64_t)gridDim.y * kMvRows) {
        float acc[kMvRows] = {};
        for (int64_t k = lane * 8; k < a.K; k += 256) {
            const uint32_t word = w[k / 8];
            const float s = ws[k / a.w.group];
#pragma unroll
            for (int j = 0; j < kMvRows; j++) {
                if (m0 + j >= a.M) break;
                float v[8], d = 0.0f, sx = 1.0f;
                if constexpr (XT == ESB_CODES) {
                    const uint32_t* xw = a.xc.codes + (m0 + j) * a.xc.ld + k / 4;
                    const uint32_t w0 = xw[0], w1 = k + 4 < a.K ? xw[1] : 0u;
#pragma unroll
                    for (int i = 0; i < 8; i++) v[i] = k + i < a.K ? xtab[((i < 4 ? w0 : w1) >> (8 * (i & 3))) & 255u] : 0.0f;
                    sx = a.xc.scales[(m0 + j) * a.xc.lds + k / a.xgroup];
                } else {
                    load8_to(static_cast<const Elem<XT>*>(a.x) + (m0 + j) * a.ldx + k, a.K - k, a.xvec, v);
                }
#pragma unroll
                for (int i = 0; i < 8; i++)
                    if (k + i < a.K) d = fmaf(tab[(word >> (4 * i)) & 15u] * s, v[i], d);
                acc[j] = fmaf(d, sx, acc[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < kMvRows; j++) {
            const float t = warp_sum(acc[j]);
            if (lane == 0 && m0 + j < a.M) put_y(a, m0 + j, n, t);
        }
    }
}

}  // namespace

cudaError_t launch_matvec_groups(int64_t M, int64_t N, int64_t K, const void* x, int x_type, int64_t ldx, const esb_coded* xc,
                                 const esb_coded& w, const float* bias, void* y, int y_type, int64_t ldy, cudaStream_t st)
{
    MvArgs a;
    a.M = M; a.N = N; a.K = K;
    a.x = x; a.ldx = ldx;
    a.xc = xc ? *xc : esb_coded{};
    a.w = w;
    const int64_t whole = (K + 31) / 32 * 32;
    if (a.w.group <= 0 || a.w.group > K) a.w.group = whole;
    a.xgroup = xc && xc->group > 0 && xc->group < K ? xc->group : whole;
    a.bias = bias; a.y = y; a.y_type = y_type; a.ldy = ldy;
    a.xvec = x && (reinterpret_cast<uintptr_t>(x) & 15u) == 0 && ldx * type_bytes(x_type) % 16 == 0;
    const int64_t tiles = (M + kMvRows - 1) / kMvRows;
    const dim3 grid((unsigned)((N + kMvThreads / 32 - 1) / (kMvThreads / 32)), (unsigned)(tiles < 65535 ? tiles : 65535));
    using Kernel = void (*)(const MvArgs);
    static const Kernel kernels[4] = {matvec_kernel<ESB_F32>, matvec_kernel<ESB_F16>, matvec_kernel<ESB_BF16>, matvec_kernel<ESB_CODES>};
    return launch_pdl(kernels[x_type], grid, dim3(kMvThreads), 0, st, a);
}

}  // namespace esb
