// esb_groups.cu -- projection onto ESB codes with a scale for every group of
// values of a row: alpha = max|x| / C, or the DDA scale of the group
// (Sec. III-D with the group as the tensor), then Eq. cheap_projection.
#include <cstdint>
#include <type_traits>
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
    const int n = left_of(a.cols, vec * 8);
    quantise8<B, true>(v, s, a.f, w, q);
    if (n < 8) zero_past<B>(w, n, a.f);
    uint32_t* p = a.codes + row * a.ldc + vec * (B / 4);
    if (B == 8 && a.cvec && vec * 2 + 1 < a.ldc) {
        *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[B / 4 - 1]);
    } else {
#pragma unroll
        for (int i = 0; i < B / 4; i++)
            if (vec * (B / 4) + i < a.ldc) p[i] = w[i];
    }
    if (!a.xq || n <= 0) return;
    element_values(v, s, a.f, q);
    store8_any(a.xq, a.xq_type, row * a.ldq + vec * 8, n, a.qvec, q);
}

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
                load8_to(x + e, left_of(e1, e), a.xvec, v);
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
                    load8_to(x + e, left_of(e1, e), a.xvec, v);
#pragma unroll
                    for (int i = 0; i < 8; i++) s1 += v[i];
                }
                mean = warp_sum(s1) / n;
            }
            for (int64_t e = e0 + lane * 8; e < e1; e += 256) {
                load8_to(x + e, left_of(e1, e), a.xvec, v);
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
            load8_to(x + e, left_of(e1, e), a.xvec, v);
            project8<B>(a, row, e / 8, v, s);
        }
    }
}

// Groups of 32, 64, 128 or 256 values: 16 a lane, LANES lanes to a group, the
// values in registers from the scale to the codes.  Rows are padded to whole
// groups (`chunks` sixteens); a thread goes on by dr rows and dc sixteens.
// Instructions and HBM bound it alike: a value may cost 24 at the copy rate, and
// the quotient, its rounding and sign, the element's value and a sixteenth of
// the group's scale take about as many.  16384 x 4096 bf16 to (4,2) with values
// (304 MB of reads and writes, 45 us at the copy rate): 55 us with the next
// sixteen loaded ahead, one eight after the other from there to its stores, few
// branches for whole sixteens, and four blocks on an SM.  62 with a branch at
// every eight's kind and stores; with those, 73 without the load ahead, 66 with
// three blocks and 73 with five, whose registers spill, 72 with blocks of a
// single sixteen a thread.
template <int TYPE, int B, int LANES>
__global__ void __launch_bounds__(kGroupThreads, 4) project_small_groups_kernel(const GroupArgs a, int chunks, int dr, int dc)
{
    using T = Elem<TYPE>;
    griddep_wait();
    const int at = (int)blockIdx.x * kGroupThreads + (int)threadIdx.x;
    int row = at / chunks, chunk = at - row * chunks;
    const int part = threadIdx.x % LANES;               // chunks and a block are whole groups
    const int rows = (int)a.rows;
    auto total = [&](float v) {
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    };
    // whole sixteens of a signed set under absmax scales, written by vectors and
    // with values of x's type, take few branches
    const bool straight = a.f.plain && a.rule == ESB_SCALE_ABSMAX && a.cvec && (!a.xq || (a.xq_type == TYPE && a.qvec));
    Raw8<T> next[2];
    auto load = [&]() {
        const int64_t e = (int64_t)chunk * 16;
        const int n = row < rows ? left_of(a.cols, e) : 0;
        const T* x = static_cast<const T*>(a.x) + row * a.ldx + e;
        next[0].load(x, n, a.xvec);
        next[1].load(x + 8, n - 8, a.xvec);
    };
    load();
    while (__any_sync(0xffffffffu, row < rows)) {
        const Raw8<T> raw[2] = {next[0], next[1]};
        const int in_row = row, in_chunk = chunk;
        row += dr;
        chunk += dc;
        if (chunk >= chunks) { chunk -= chunks; row++; }
        load();
        const int64_t e = (int64_t)in_chunk * 16;
        float v[8];
        float alpha;
        if (a.rule == ESB_SCALE_ABSMAX) {
            uint32_t mx = 0u;
            if (TYPE != ESB_F32 && a.f.is_signed) {
                // magnitudes in pairs of 16 bits, which order as the numbers do
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int i = 0; i < 4; i++) mx = __vmaxu2(mx, raw[h].w[i] & 0x7fff7fffu);
                mx = max(mx & 0xffffu, mx >> 16);
                const uint16_t m16 = (uint16_t)mx;
                mx = __float_as_uint(to_f32(*reinterpret_cast<const T*>(&m16)));
            } else {
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    raw[h].values(v);
                    mx = max(mx, largest_of8(v, a.f.is_signed));
                }
            }
#pragma unroll
            for (int o = LANES / 2; o > 0; o >>= 1) mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            alpha = absmax_scale(mx, a.f);
        } else {
            const int64_t left = a.cols - (e - part * 16);
            const float n = (float)(left < 16 * LANES ? left : 16 * LANES);
            float mean = 0.0f, s2 = 0.0f;
            if (a.f.is_signed) {
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    raw[h].values(v);
#pragma unroll
                    for (int i = 0; i < 8; i++) mean += v[i];
                }
                mean = total(mean) / n;
            }
#pragma unroll
            for (int h = 0; h < 2; h++) {
                raw[h].values(v);
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const float d = e + 8 * h + i < a.cols ? v[i] - mean : 0.0f;
                    s2 = fmaf(d, d, s2);
                }
            }
            alpha = __fmul_rn(a.astar, __fadd_rn(__fsqrt_rn(total(s2) / n), 1e-7f));
        }
        if (in_row >= rows) continue;
        const int64_t gi = in_chunk / LANES;
        if (part == 0 && gi < a.ngroups) a.scales[in_row * a.lds + gi] = alpha;
        const GroupScale s = make_scale(alpha, a.f);
        const int left = left_of(a.cols, e);
        uint32_t w[2][B / 4];
        constexpr int WORDS = B / 2;                    // of 16 codes
        uint32_t* p = a.codes + in_row * a.ldc + (int64_t)in_chunk * WORDS;
        auto put_words = [&]() {
            if constexpr (B == 4) *reinterpret_cast<uint2*>(p) = make_uint2(w[0][0], w[1][0]);
            else *reinterpret_cast<uint4*>(p) = make_uint4(w[0][0], w[0][B / 4 - 1], w[1][0], w[1][B / 4 - 1]);
        };
        if (straight && left >= 16 && s.fast) {
            T* q = static_cast<T*>(a.xq) + in_row * a.ldq + e;
            auto sixteen = [&](auto linear) {
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    float r[8];
                    if constexpr (TYPE == ESB_F32) {
                        raw[h].values(v);
                        places8<B, decltype(linear)::value, false>(v, s, a.f, w[h], r);
                        codes8<B>(v, a.f, w[h]);
                        if (a.xq) {
                            element_values(v, s, a.f, r);
                            store8<T>(q + 8 * h, r);
                        }
                    } else {
                        // signs in pairs of 16 bits, off and on again
#pragma unroll
                        for (int i = 0; i < 4; i++) unpack2<T>(raw[h].w[i] & 0x7fff7fffu, v[2 * i], v[2 * i + 1]);
                        places8<B, decltype(linear)::value, false, true>(v, s, a.f, w[h], r);
                        codes8<B>(raw[h].w, a.f, w[h]);
                        if (a.xq) {
                            uint32_t y[4];
#pragma unroll
                            for (int i = 0; i < 4; i++) {
                                split(mul2(pair_of(s.step, s.step), pair_of(r[2 * i], r[2 * i + 1])), r[2 * i], r[2 * i + 1]);
                                y[i] = pack2<T>(r[2 * i], r[2 * i + 1]) | (raw[h].w[i] & 0x80008000u);
                            }
                            *reinterpret_cast<uint4*>(q + 8 * h) = make_uint4(y[0], y[1], y[2], y[3]);
                        }
                    }
                }
            };
            if (a.f.linear) sixteen(std::true_type());
            else sixteen(std::false_type());
            put_words();
            continue;
        }
#pragma unroll
        for (int h = 0; h < 2; h++) {
            float r[8];
            const int n = left - 8 * h;
            raw[h].values(v);
            if (a.rule == ESB_SCALE_ABSMAX) quantise8<B, false>(v, s, a.f, w[h], r);
            else quantise8<B, true>(v, s, a.f, w[h], r);
            if (n < 8) zero_past<B>(w[h], n, a.f);
            if (a.xq && n > 0) {
                element_values(v, s, a.f, r);
                store8_any(a.xq, a.xq_type, in_row * a.ldq + e + 8 * h, n, a.qvec, r);
            }
        }
        if (a.cvec && (int64_t)(in_chunk + 1) * WORDS <= a.ldc) {
            put_words();
        } else {
#pragma unroll
            for (int i = 0; i < WORDS; i++)
                if ((int64_t)in_chunk * WORDS + i < a.ldc) p[i] = w[i / (B / 4)][i % (B / 4)];
        }
    }
}

using GroupKernel = void (*)(const GroupArgs);
using SmallKernel = void (*)(const GroupArgs, int, int, int);
template <int TYPE, int B> SmallKernel small_kernel(int lanes)
{
    switch (lanes) {
    case 2: return project_small_groups_kernel<TYPE, B, 2>;
    case 4: return project_small_groups_kernel<TYPE, B, 4>;
    case 8: return project_small_groups_kernel<TYPE, B, 8>;
    default: return project_small_groups_kernel<TYPE, B, 16>;
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
    const int words = f.b / 2;                          // of 16 codes
    a.cvec = (reinterpret_cast<uintptr_t>(codes) & (4u * words - 1u)) == 0 && ldc % words == 0;
    const int64_t sms = device_sm_count();
    const int lanes = (int)(a.group / 16);
    // sixteens of a row up to its last code word, in whole groups
    const int64_t chunks = lanes ? ((ldc + words - 1) / words + lanes - 1) / lanes * lanes : 0;
    if ((a.group == 32 || a.group == 64 || a.group == 128 || a.group == 256) && rows < (1 << 30) && chunks < (1 << 30)) {
        static SmallKernel (*const pick[3][2])(int) = {{small_kernel<ESB_F32, 4>, small_kernel<ESB_F32, 8>},
                                                       {small_kernel<ESB_F16, 4>, small_kernel<ESB_F16, 8>},
                                                       {small_kernel<ESB_BF16, 4>, small_kernel<ESB_BF16, 8>}};
        int64_t blocks = (rows * chunks + kGroupThreads - 1) / kGroupThreads;
        const int64_t cap = sms * 16;
        if (blocks > cap) blocks = cap;
        const int64_t threads = blocks * kGroupThreads;
        return launch_pdl(pick[x_type][f.b == 8](lanes), dim3((unsigned)blocks), dim3(kGroupThreads), 0, st, a, (int)chunks,
                          (int)(threads / chunks), (int)(threads % chunks));
    }
    a.cvec = (reinterpret_cast<uintptr_t>(codes) & 7u) == 0 && ldc % 2 == 0;
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
