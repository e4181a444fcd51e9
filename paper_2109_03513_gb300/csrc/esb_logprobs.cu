// esb_logprobs.cu -- log probabilities of given tokens, entropy and the most
// likely alternatives of rows of logits, and the gradient.
#include <cstdint>
#include <cuda_runtime.h>

#include "esb_internal.h"
#include "esb_rows.cuh"

namespace esb {

namespace {

constexpr int kLpThreads = 256;

struct LpArgs {
    const void* x;
    int64_t rows, cols, ldx;
    const int64_t* ids;
    int top;
    float *logp, *entropy, *lse, *top_logp;
    int64_t* top_ids;
    int vec;
};

// Order of the alternatives: the larger logit first, the lower place among
// equals.  Key 0 is below every number; NaN and -inf have it.
__device__ __forceinline__ unsigned long long top_key(float v, uint32_t at)
{
    if (!(v > __int_as_float(0xff800000))) return 0ull;
    const uint32_t u = __float_as_uint(v == 0.0f ? 0.0f : v);   // -0 counts as 0
    return ((unsigned long long)((u >> 31) ? ~u : u | 0x80000000u) << 32) | (0xffffffffu - at);
}

template <int NW>
__device__ __forceinline__ float lp_block(float v, float* sh, bool is_max)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float t = __shfl_xor_sync(0xffffffffu, v, o);
        v = is_max ? fmaxf(v, t) : v + t;
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    v = sh[0];
#pragma unroll
    for (int i = 1; i < NW; i++) v = is_max ? fmaxf(v, sh[i]) : v + sh[i];
    return v;
}

template <int TYPE>
__global__ void __launch_bounds__(kLpThreads) logprobs_kernel(const LpArgs a)
{
    using T = Elem<TYPE>;
    constexpr int NW = kLpThreads / 32;
    __shared__ float shf[NW];
    __shared__ unsigned long long shk[NW];
    griddep_wait();
    const float ninf = __int_as_float(0xff800000);
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + row * a.ldx;
        float v[8];
        float m = ninf;
        for (int64_t e = threadIdx.x * 8; e < a.cols; e += kLpThreads * 8) {
            load8_to(x + e, a.cols - e, a.vec, v);
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (e + i < a.cols) m = fmaxf(m, v[i]);
        }
        m = lp_block<NW>(m, shf, true);
        const bool empty = m == ninf;            // or every value NaN
        float s = 0.0f, sx = 0.0f;
        for (int64_t e = threadIdx.x * 8; e < a.cols; e += kLpThreads * 8) {
            load8_to(x + e, a.cols - e, a.vec, v);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                if (e + i >= a.cols || v[i] == ninf) continue;
                const float d = v[i] - m, p = __expf(d);
                s += p;
                sx = fmaf(p, p > 0.0f ? d : 0.0f, sx);
            }
        }
        s = lp_block<NW>(s, shf, false);
        sx = lp_block<NW>(sx, shf, false);
        const float lz = logf(s);
        const float lse = m + lz;
        if (threadIdx.x == 0) {
            const bool none = empty && s == 0.0f;   // every logit is -inf
            if (a.lse) a.lse[row] = none ? ninf : lse;
            if (a.entropy) a.entropy[row] = none ? 0.0f : lz - sx / s;
            if (a.logp) {
                const int64_t t = a.ids[row];
                a.logp[row] = t < 0 || t >= a.cols ? 0.0f : (none ? ninf : (to_f32(x[t]) - m) - lz);
            }
        }
        unsigned long long last = ~0ull;
        for (int j = 0; j < a.top; j++) {
            unsigned long long best = 0ull;
            for (int64_t e = threadIdx.x; e < a.cols; e += kLpThreads) {
                const unsigned long long k = top_key(to_f32(x[e]), (uint32_t)e);
                if (k < last && k > best) best = k;
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                const unsigned long long t = __shfl_xor_sync(0xffffffffu, best, o);
                best = t > best ? t : best;
            }
            __syncthreads();
            if ((threadIdx.x & 31) == 0) shk[threadIdx.x >> 5] = best;
            __syncthreads();
            best = shk[0];
#pragma unroll
            for (int i = 1; i < NW; i++) best = shk[i] > best ? shk[i] : best;
            last = best;
            if (threadIdx.x == 0) {
                const int64_t at = best ? (int64_t)(0xffffffffu - (uint32_t)best) : -1;
                a.top_ids[row * a.top + j] = at;
                a.top_logp[row * a.top + j] = best ? (to_f32(x[at]) - m) - lz : ninf;
            }
        }
    }
}

struct LpGradArgs {
    const void* x;
    int64_t rows, cols, ldx;
    const int64_t* ids;
    const float *lse, *entropy, *dlogp, *dentropy;
    void* dx;
    int64_t lddx;
    int vec, dvec;
};

// dx = g (1_t - p) - gH p (log p + H), p = e^(x - lse).
template <int TYPE>
__global__ void __launch_bounds__(kLpThreads) logprobs_grad_kernel(const LpGradArgs a)
{
    using T = Elem<TYPE>;
    griddep_wait();
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + row * a.ldx;
        T* dx = static_cast<T*>(a.dx) + row * a.lddx;
        const int64_t t = a.ids ? a.ids[row] : -1;
        const float g = a.dlogp && t >= 0 && t < a.cols ? a.dlogp[row] : 0.0f;
        const float gh = a.dentropy ? a.dentropy[row] : 0.0f, H = a.dentropy ? a.entropy[row] : 0.0f;
        const float lse = a.lse[row];
        for (int64_t e = threadIdx.x * 8; e < a.cols; e += kLpThreads * 8) {
            float v[8];
            load8_to(x + e, a.cols - e, a.vec, v);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float lp = v[i] - lse;
                const float p = __expf(lp);
                // a masked logit has no gradient (a row of them lse = -inf)
                const bool zero = v[i] == __int_as_float(0xff800000) || p == 0.0f;
                v[i] = zero ? 0.0f : -p * fmaf(gh, lp + H, g);
                if (e + i == t) v[i] += g;
            }
            store8_to(dx + e, a.cols - e, a.dvec, v);
        }
    }
}

}  // namespace

cudaError_t launch_logprobs(const void* x, int type, int64_t rows, int64_t cols, int64_t ldx, const int64_t* ids, int top,
                            float* logp, float* entropy, float* lse, float* top_logp, int64_t* top_ids, cudaStream_t st)
{
    LpArgs a{x, rows, cols, ldx, ids, top, logp, entropy, lse, top_logp, top_ids, 0};
    a.vec = (reinterpret_cast<uintptr_t>(x) & 15u) == 0 && ldx * type_bytes(type) % 16 == 0;
    const int64_t cap = (int64_t)device_sm_count() * 8;
    using Kernel = void (*)(const LpArgs);
    static const Kernel kernels[3] = {logprobs_kernel<ESB_F32>, logprobs_kernel<ESB_F16>, logprobs_kernel<ESB_BF16>};
    return launch_pdl(kernels[type], dim3((unsigned)(rows < cap ? rows : cap)), dim3(kLpThreads), 0, st, a);
}

cudaError_t launch_logprobs_grad(const void* x, int type, int64_t rows, int64_t cols, int64_t ldx, const int64_t* ids,
                                 const float* lse, const float* entropy, const float* dlogp, const float* dentropy, void* dx,
                                 int64_t lddx, cudaStream_t st)
{
    LpGradArgs a{x, rows, cols, ldx, ids, lse, entropy, dlogp, dentropy, dx, lddx, 0, 0};
    a.vec = (reinterpret_cast<uintptr_t>(x) & 15u) == 0 && ldx * type_bytes(type) % 16 == 0;
    a.dvec = (reinterpret_cast<uintptr_t>(dx) & 15u) == 0 && lddx * type_bytes(type) % 16 == 0;
    const int64_t cap = (int64_t)device_sm_count() * 8;
    using Kernel = void (*)(const LpGradArgs);
    static const Kernel kernels[3] = {logprobs_grad_kernel<ESB_F32>, logprobs_grad_kernel<ESB_F16>, logprobs_grad_kernel<ESB_BF16>};
    return launch_pdl(kernels[type], dim3((unsigned)(rows < cap ? rows : cap)), dim3(kLpThreads), 0, st, a);
}

}  // namespace esb
