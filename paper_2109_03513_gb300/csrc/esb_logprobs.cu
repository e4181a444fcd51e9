// esb_logprobs.cu -- log probabilities of given tokens, entropy and the most
// likely alternatives of rows of logits, and the gradient.
//
// One pass over the row: every thread keeps the largest logit m that it has
// met, sum e^(x-m) and sum e^(x-m) (x-m), rescaled when m grows; they are
// joined over the block, and over the blocks of a cluster where a few rows
// would leave SMs idle.  With M, S and D those of the row,
//   lse = M + log S,  entropy = log S - D / S.
// 2 or 4 bytes a logit from HBM; at the measured copy rate a bf16 logit has
// about 11 issue slots.  Differences, products and sums go in pairs (two fp32
// numbers an instruction), the largest of 16 logits in pairs of 16 bits.
// 4096 x 49999 bf16: 87 us without alternatives (60 at the copy rate), bound by
// instructions; 159 with 8 and 238 with 32 of them, which add barriers and
// sorts.  A row of 131072 with 8: 8.5 us, all latency.
//
// The alternatives come out of the same pass.  A key orders logits by value,
// then by place.  After a row's first block of logits the best keys of the 32
// lanes, each over all warps, are 32 logits of the row, so the top-th best of
// them is a bound that no alternative lies below; from then on a thread puts
// logits at or above the bound into a list, which is sorted and cut to the best
// 32 now and then, raising the bound.  Where it overflows all the same (rows
// that ascend), the row is taken again in steps that it holds.
#include <cstdint>
#include <cuda_runtime.h>

#include "esb_internal.h"
#include "esb_rows.cuh"

namespace esb {

namespace {

constexpr int kLpMaxWarps = 16;
constexpr int kLpValues = 16;           // logits of a thread in a block of them; half a warp takes them one each
constexpr int kLpList = 2048;
constexpr int kLpFull = 128;            // keys in the list that are worth a cut
constexpr int kLpMaxCluster = 8;

using Key = unsigned long long;

struct LpArgs {
    const void* x;
    int64_t rows, cols, ldx;
    const int64_t* ids;
    int top, split;                     // split: blocks of a row, a cluster
    float *logp, *entropy, *lse, *top_logp;
    int64_t* top_ids;
};

// Key 0 is below every number; NaN and -inf have it.
__device__ __forceinline__ Key top_key(float v, uint32_t at)
{
    if (!(v > __int_as_float(0xff800000))) return 0ull;
    const uint32_t u = __float_as_uint(v == 0.0f ? 0.0f : v);   // -0 counts as 0
    return ((Key)((u >> 31) ? ~u : u | 0x80000000u) << 32) | (0xffffffffu - at);
}
__device__ __forceinline__ uint32_t key_place(Key k) { return 0xffffffffu - (uint32_t)k; }
__device__ __forceinline__ float key_value(Key k)
{
    const uint32_t u = (uint32_t)(k >> 32);
    return __uint_as_float((u >> 31) ? u & 0x7fffffffu : ~u);
}

// e^x for x <= 0 (and NaN): the hardware's 2^y with results below 2^-126 as 0.
// y is rounded, so the result is off by some 2 + 1.2 |x| units in the last
// place: far terms, whose share of a sum is e^x, have the large errors.  A
// more exact e^x would take several more of the instructions that bound the
// pass.
__device__ __forceinline__ float exp_of(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x * 1.44269504f));
    return r;
}

__device__ __forceinline__ float ex2_of(float y)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(y));
    return r;
}

struct LpSums {
    float m, s, d;
};
// The sums of two parts of a row.  A part without a logit has m = lowest and
// s = 0; a factor of 0 drops a part whose difference is not finite.
__device__ __forceinline__ LpSums join(const LpSums& a, const LpSums& b)
{
    LpSums r;
    r.m = fmaxf(a.m, b.m);
    const float da = a.m - r.m, db = b.m - r.m, fa = exp_of(da), fb = exp_of(db);
    r.s = a.s * fa + b.s * fb;
    r.d = (fa == 0.0f ? 0.0f : fa * fmaf(da, a.s, a.d)) + (fb == 0.0f ? 0.0f : fb * fmaf(db, b.s, b.d));
    if (!(a.s == a.s) || !(b.s == b.s)) r.s = r.d = __int_as_float(0x7fffffff);
    return r;
}

// Descending bitonic sort of one key a lane; merge keeps the best 32 of two
// descending lists.
__device__ __forceinline__ Key shfl_key(Key k, int o)
{
    return ((Key)__shfl_xor_sync(0xffffffffu, (uint32_t)(k >> 32), o) << 32) | __shfl_xor_sync(0xffffffffu, (uint32_t)k, o);
}
__device__ __forceinline__ Key pick(Key k, int o, bool larger)
{
    const Key t = shfl_key(k, o);
    return (t > k) == larger ? t : k;
}
__device__ __forceinline__ Key sort32(Key k, int lane)
{
#pragma unroll
    for (int n = 2; n <= 32; n *= 2)
#pragma unroll
        for (int o = n / 2; o > 0; o /= 2) k = pick(k, o, ((lane & o) == 0) == ((lane & n) == 0 || n == 32));
    return k;
}
__device__ __forceinline__ Key merge32(Key best, Key more, int lane)
{
    const Key r = ((Key)__shfl_sync(0xffffffffu, (uint32_t)(more >> 32), 31 - lane) << 32) | __shfl_sync(0xffffffffu, (uint32_t)more, 31 - lane);
    Key k = best > r ? best : r;                        // a bitonic sequence
#pragma unroll
    for (int o = 16; o > 0; o /= 2) k = pick(k, o, (lane & o) == 0);
    return k;
}

struct LpShared {
    LpSums sums[kLpMaxWarps], total;
    Key lanes[kLpMaxWarps][32];
    Key best[32];                       // the best keys so far, descending
    Key bound;                          // no alternative is below it
    int count, overflow;
    LpSums parts[kLpMaxCluster];        // of the cluster's blocks, in block 0
    Key part_keys[kLpMaxCluster][32];
    Key list[kLpList];
};

// The list's keys into the best 32, by the whole block (the list is complete,
// and a barrier follows): every warp sorts its part, warp 0 takes them
// together.  The bound is the top-th of them.
template <int WARPS>
__device__ __forceinline__ void cut_list(LpShared& sh, int top, int warp, int lane)
{
    const int n = min(sh.count, kLpList);
    Key mine = 0ull;
    for (int i = warp * 32; i < n; i += WARPS * 32) {
        const Key k = sort32(i + lane < n ? sh.list[i + lane] : 0ull, lane);
        mine = i < WARPS * 32 ? k : merge32(mine, k, lane);
    }
    if (warp * 32 < n) sh.lanes[warp][lane] = mine;
    __syncthreads();
    if (warp == 0) {
        Key best = sh.best[lane];
        for (int w = 0; w < WARPS && w * 32 < n; w++) best = merge32(best, sh.lanes[w][lane], lane);
        sh.best[lane] = best;
        const Key b = ((Key)__shfl_sync(0xffffffffu, (uint32_t)(best >> 32), top - 1) << 32) | __shfl_sync(0xffffffffu, (uint32_t)best, top - 1);
        if (lane == 0) {
            if (b > sh.bound) sh.bound = b;
            sh.count = 0;
        }
    }
}

template <class T>
__device__ __forceinline__ void remote_store(T* p, int rank, const T& v)
{
    static_assert(sizeof(T) % 4 == 0, "words");
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    const uint32_t* w = reinterpret_cast<const uint32_t*>(&v);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 4); i++)
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(a + 4 * i), "r"(w[i]) : "memory");
}
__device__ __forceinline__ void lp_cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}

// A row as 16-byte vectors: `head` values before the first 16-byte boundary,
// then `vecs` vectors, then what is left.
template <class T>
struct RowParts {
    int head, tail_at;                  // values before the vectors; the first value after them
    int64_t vecs;
    __device__ __forceinline__ RowParts(const T* x, int64_t cols)
    {
        constexpr int V = 16 / sizeof(T);
        const int mis = (int)((reinterpret_cast<uintptr_t>(x) & 15u) / sizeof(T));
        const int64_t h = mis ? V - mis : 0;
        head = (int)(h < cols ? h : cols);
        vecs = (cols - head) / V;
        tail_at = (int)(head + vecs * V);
    }
};

// Larger and smaller halves of two pairs of 16-bit numbers (the number of a
// number and NaN).
template <class T> __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b);
template <class T> __device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b);
template <> __device__ __forceinline__ uint32_t max2<__nv_bfloat16>(uint32_t a, uint32_t b)
{
    const __nv_bfloat162 r = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
}
template <> __device__ __forceinline__ uint32_t min2<__nv_bfloat16>(uint32_t a, uint32_t b)
{
    const __nv_bfloat162 r = __hmin2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
}
template <> __device__ __forceinline__ uint32_t max2<__half>(uint32_t a, uint32_t b)
{
    const __half2 r = __hmax2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
}
template <> __device__ __forceinline__ uint32_t min2<__half>(uint32_t a, uint32_t b)
{
    const __half2 r = __hmin2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
}

// Registers: 64 a thread; for fp32 and up to 8 warps a block more, with 24 warps
// on an SM (2048 x 65536: 89 us, 99 with 32, whose loads run less far ahead;
// blocks of 16 are slower that way, 28 us for 256 x 65537 and not 24).
template <int TYPE, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, (TYPE == ESB_F32 && WARPS < 16 ? 24 : 32) / WARPS) logprobs_kernel(const LpArgs a)
{
    constexpr int kLpThreads = WARPS * 32, kLpWarps = WARPS;
    using T = Elem<TYPE>;
    constexpr int V = 16 / sizeof(T), U = kLpValues / V;   // values of a vector, vectors of a thread in a block of logits
    extern __shared__ __align__(16) unsigned char lp_smem[];
    LpShared& sh = *reinterpret_cast<LpShared*>(lp_smem);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rank = a.split > 1 ? (int)(blockIdx.x % a.split) : 0;
    const float ninf = __int_as_float(0xff800000), lowest = -__int_as_float(0x7f7fffff);
    griddep_wait();
    if (a.split > 1) lp_cluster_barrier();              // every block of the cluster runs before its memory is written
    for (int64_t row = blockIdx.x / a.split; row < a.rows; row += gridDim.x / a.split) {
        const T* x = static_cast<const T*>(a.x) + row * a.ldx;
        const RowParts<T> rp(x, a.cols);
        const T* xv = x + rp.head;
        if (a.top) {
            if (threadIdx.x < 32) sh.best[threadIdx.x] = 0ull;
            if (threadIdx.x == 0) { sh.bound = 0ull; sh.count = 0; sh.overflow = 0; }
            __syncthreads();
        }
        // two halves of the thread's sums, added up at the end
        float m = lowest;
        Pair s2 = pair_of(0.0f, 0.0f), d2 = s2;
        const Pair log2e = pair_of(1.44269504f, 1.44269504f);
        auto add = [&](float x0, float x1, const Pair& minus_m, bool clamp) {
            Pair d = add2(pair_of(x0, x1), minus_m);
            float y0, y1;
            split(mul2(d, log2e), y0, y1);
            const Pair p = pair_of(ex2_of(y0), ex2_of(y1));
            s2 = add2(s2, p);
            if (clamp) {
                // x - m = -inf as a number; p is 0 there
                split(d, y0, y1);
                d = pair_of(fmaxf(y0, -200.0f), fmaxf(y1, -200.0f));
            }
            d2 = fma2(p, d, d2);
        };
        auto raise = [&](float to) {
            if (to > m) {
                const float d = m - to, f = exp_of(d);
                const Pair f2 = pair_of(f, f);
                // d may be -inf where f is 0; s2 never is, and keeps NaN
                d2 = f == 0.0f ? pair_of(0.0f, 0.0f) : mul2(f2, fma2(pair_of(d, d), s2, d2));
                s2 = mul2(f2, s2);
                m = to;
            }
        };
        Key bound = 0ull;
        bool full = false;              // this thread has met a list that is worth a cut
        auto offer = [&](float v, uint32_t at) {
            const Key k = top_key(v, at);
            if (k < bound || !k) return;
            const int i = atomicAdd(&sh.count, 1);
            if (i < kLpList) sh.list[i] = k;
            else sh.overflow = 1;
            full |= i >= kLpFull;
        };
        constexpr int64_t step = (int64_t)kLpThreads * U;   // vectors of a block of logits
        bool first = true;
        int blocks = 0;
        uint4 next[U];
        auto load = [&](int64_t v0) {
            const uint4* from = reinterpret_cast<const uint4*>(xv) + v0 + threadIdx.x;
            if (v0 + step <= rp.vecs) {
#pragma unroll
                for (int u = 0; u < U; u++) next[u] = __ldg(from + u * kLpThreads);
            } else {
                // -inf past the row
                constexpr uint32_t F = TYPE == ESB_F32 ? 0xff800000u : (TYPE == ESB_F16 ? 0xfc00fc00u : 0xff80ff80u);
#pragma unroll
                for (int u = 0; u < U; u++) {
                    next[u] = make_uint4(F, F, F, F);
                    if (v0 + u * kLpThreads + threadIdx.x < rp.vecs) next[u] = __ldg(from + u * kLpThreads);
                }
            }
        };
        load(rank * step);
        for (int64_t v0 = rank * step; v0 < rp.vecs || first; v0 += a.split * step) {
            uint4 raw[U];
#pragma unroll
            for (int u = 0; u < U; u++) raw[u] = next[u];
            load(v0 + a.split * step);
            // a few values before and after the vectors: the first block of
            // the row has them, one a thread
            float edge = ninf;
            uint32_t edge_at = 0u;
            if (first && rank == 0) {
                const int64_t e = threadIdx.x < (unsigned)rp.head ? threadIdx.x : (int64_t)rp.tail_at + threadIdx.x - rp.head;
                if (e < a.cols && threadIdx.x < 32) { edge = to_f32(x[e]); edge_at = (uint32_t)e; }
            }
            float v[U][V];
            float big = fmaxf(lowest, edge);                // the thread's largest
            float least_of = ninf;                          // its smallest (fp32: not looked for)
#pragma unroll
            for (int u = 0; u < U; u++) {
                if constexpr (V == 8) {
                    unpack2<T>(raw[u].x, v[u][0], v[u][1]);
                    unpack2<T>(raw[u].y, v[u][2], v[u][3]);
                    unpack2<T>(raw[u].z, v[u][4], v[u][5]);
                    unpack2<T>(raw[u].w, v[u][6], v[u][7]);
                } else {
                    v[u][0] = __uint_as_float(raw[u].x); v[u][1] = __uint_as_float(raw[u].y);
                    v[u][2] = __uint_as_float(raw[u].z); v[u][3] = __uint_as_float(raw[u].w);
                }
            }
            if constexpr (V == 8) {
                // in pairs of 16 bits: the largest and the smallest
                uint32_t hi = raw[0].x, lo = raw[0].x;
#pragma unroll
                for (int u = 0; u < U; u++) {
                    const uint32_t w[4] = {raw[u].x, raw[u].y, raw[u].z, raw[u].w};
#pragma unroll
                    for (int j = u ? 0 : 1; j < 4; j++) {
                        hi = max2<T>(hi, w[j]);
                        lo = min2<T>(lo, w[j]);
                    }
                }
                float a0, a1;
                unpack2<T>(hi, a0, a1);
                big = fmaxf(big, fmaxf(a0, a1));
                unpack2<T>(lo, a0, a1);
                least_of = fminf(a0, a1);
            } else {
#pragma unroll
                for (int u = 0; u < U; u++)
#pragma unroll
                    for (int j = 0; j < V; j++) big = fmaxf(big, v[u][j]);
            }
            raise(big);
            const Pair minus_m = pair_of(-m, -m);
            if (edge != ninf) add(edge, ninf, minus_m, true);
            // a difference of -inf: a masked logit, or bf16's lowest from its largest
            if (V == 8 && least_of - m > ninf) {
#pragma unroll
                for (int u = 0; u < U; u++)
#pragma unroll
                    for (int j = 0; j < V; j += 2) add(v[u][j], v[u][j + 1], minus_m, false);
            } else {
#pragma unroll
                for (int u = 0; u < U; u++)
#pragma unroll
                    for (int j = 0; j < V; j += 2) add(v[u][j], v[u][j + 1], minus_m, true);
            }
            if (a.top) {
                // of value n of the thread t
                auto place = [&](int t, int n) { return (uint32_t)(rp.head + (v0 + n / V * kLpThreads + t) * V + n % V); };
                if (bound == 0ull) {                    // the same for every thread
                    // the best key of every lane over the warps
                    Key k = top_key(edge, edge_at);
                    int n = -1;                         // the thread's largest is met first at its lowest place
#pragma unroll
                    for (int i = kLpValues - 1; i >= 0; i--) n = v[i / V][i % V] == big ? i : n;
                    if (n >= 0) {
                        const Key c = top_key(big, place(threadIdx.x, n));
                        k = c > k ? c : k;
                    }
                    sh.lanes[warp][lane] = k;
                    __syncthreads();
                    if (warp == 0) {
#pragma unroll
                        for (int w = 1; w < kLpWarps; w++) k = sh.lanes[w][lane] > k ? sh.lanes[w][lane] : k;
                        k = sort32(k, lane);
                        if (lane == a.top - 1) sh.bound = k;
                    }
                    __syncthreads();
                    bound = sh.bound;
                }
                if (edge > ninf) offer(edge, edge_at);
                // Most threads have nothing at or above the bound.  The warp
                // takes those that do two at a time, 16 lanes for the values
                // of each, read again: few instructions, and in one place.
                const float least = bound ? key_value(bound) : lowest;
                for (unsigned hits = __ballot_sync(0xffffffffu, big >= least); hits; hits &= hits - 1) {
                    const unsigned more = hits & (hits - 1);
                    const unsigned mine = lane < kLpValues ? hits : more;
                    if (mine) {
                        const int t = warp * 32 + __ffs(mine) - 1, n = lane % kLpValues;
                        if (v0 + n / V * kLpThreads + t < rp.vecs) {
                            const uint32_t at = place(t, n);
                            const float w = to_f32(x[at]);
                            if (w >= least) offer(w, at);
                        }
                    }
                    if (more) hits = more;
                }
                // Every fourth block of logits, and for many alternatives the
                // first, whose bound is far below them: a cut?  The list holds
                // more than four blocks usually add.
                if (((++blocks & 3) == 0 || (blocks == 1 && a.top > 12)) && __syncthreads_or(full)) {
                    cut_list<WARPS>(sh, a.top, warp, lane);
                    __syncthreads();
                    bound = sh.bound;
                    full = false;
                }
            }
            first = false;
        }
        // the block's sums
        float sa, sb, da, db;
        split(s2, sa, sb);
        split(d2, da, db);
        LpSums t = {m, sa + sb, da + db};
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const LpSums b = {__shfl_xor_sync(0xffffffffu, t.m, o), __shfl_xor_sync(0xffffffffu, t.s, o), __shfl_xor_sync(0xffffffffu, t.d, o)};
            t = join(t, b);
        }
        if (lane == 0) sh.sums[warp] = t;
        __syncthreads();
        if (warp == (a.top ? kLpWarps - 1 : 0)) {       // while warp 0 sorts
            if (lane < kLpWarps) t = sh.sums[lane];
            else t = {lowest, 0.0f, 0.0f};
#pragma unroll
            for (int o = kLpWarps / 2; o > 0; o >>= 1) {
                const LpSums b = {__shfl_xor_sync(0xffffffffu, t.m, o), __shfl_xor_sync(0xffffffffu, t.s, o), __shfl_xor_sync(0xffffffffu, t.d, o)};
                t = join(t, b);
            }
            if (lane == 0) sh.total = t;
        }
        if (a.top) {
            if (sh.overflow) {
                // uniform after the barrier above; rare: this block's part of
                // the row again, a value a thread between barriers
                if (threadIdx.x < 32) sh.best[threadIdx.x] = 0ull;
                if (threadIdx.x == 0) sh.count = 0;
                bound = sh.bound;
                full = false;
                __syncthreads();
                for (int64_t e0 = 0; e0 < a.cols; e0 += kLpThreads) {
                    const int64_t e = e0 + threadIdx.x;
                    if (e < a.cols) {
                        const uint32_t block = (uint32_t)((uint64_t)(e - rp.head) / (uint64_t)(V * step));
                        const bool in = e < rp.head || e >= rp.tail_at ? rank == 0 : (int)(block % (uint32_t)a.split) == rank;
                        if (in) offer(to_f32(x[e]), (uint32_t)e);
                    }
                    if (__syncthreads_or(full)) {
                        cut_list<WARPS>(sh, a.top, warp, lane);
                        __syncthreads();
                        bound = sh.bound;
                        full = false;
                    }
                }
            }
            cut_list<WARPS>(sh, a.top, warp, lane);
            t = sh.total;
        }
        // the cluster's sums and keys, in block 0
        Key best = 0ull;
        if (warp == 0 && a.top) best = sh.best[lane];
        if (a.split > 1) {
            if (warp == 0 && rank) {
                if (lane == 0) remote_store(&sh.parts[rank], 0, t);
                if (a.top) remote_store(&sh.part_keys[rank][lane], 0, best);
            }
            lp_cluster_barrier();
            if (warp == 0 && rank == 0)
                for (int r = 1; r < a.split; r++) {
                    t = join(t, sh.parts[r]);       // in every lane, of which lane 0 counts
                    if (a.top) best = merge32(best, sh.part_keys[r][lane], lane);
                }
        }
        if (warp == 0 && rank == 0) {
            // lane 0 has the sums in their order
            t = {__shfl_sync(0xffffffffu, t.m, 0), __shfl_sync(0xffffffffu, t.s, 0), __shfl_sync(0xffffffffu, t.d, 0)};
            const bool none = t.m == lowest && t.s == 0.0f;     // every logit is -inf
            const float lz = logf(t.s);
            if (lane == 0) {
                if (a.lse) a.lse[row] = none ? ninf : t.m + lz;
                if (a.entropy) a.entropy[row] = none ? 0.0f : lz - t.d / t.s;
                if (a.logp) {
                    const int64_t id = a.ids[row];
                    a.logp[row] = id < 0 || id >= a.cols ? 0.0f : (none ? ninf : (to_f32(x[id]) - t.m) - lz);
                }
            }
            if (lane < a.top) {
                a.top_ids[row * a.top + lane] = best ? (int64_t)key_place(best) : -1;
                a.top_logp[row * a.top + lane] = best ? (to_f32(x[key_place(best)]) - t.m) - lz : ninf;
            }
        }
        if (a.split > 1) lp_cluster_barrier();          // the parts are written again
        else __syncthreads();                           // and so are the block's own numbers
    }
}

struct LpGradArgs {
    const void* x;
    int64_t rows, cols, ldx;
    const int64_t* ids;
    const float *lse, *entropy, *dlogp, *dentropy;
    void* dx;
    int64_t lddx;
    int split;                          // blocks of a row
};

// dx = g (1_t - p) - gH p (log p + H), p = e^(x - lse): a read and a write of
// every logit, HBM-bound.  A row's values before and after its 16-byte vectors
// go one a thread; where x and dx lie differently within 16 bytes, all do.
template <int TYPE>
__global__ void __launch_bounds__(256) logprobs_grad_kernel(const LpGradArgs a)
{
    using T = Elem<TYPE>;
    constexpr int V = 16 / sizeof(T), U = 4, THREADS = 256;
    griddep_wait();
    const int64_t total = a.rows * a.split;
    for (int64_t w = blockIdx.x; w < total; w += gridDim.x) {
        const int64_t row = w / a.split;
        const int part = (int)(w - row * a.split);
        const T* x = static_cast<const T*>(a.x) + row * a.ldx;
        T* dx = static_cast<T*>(a.dx) + row * a.lddx;
        const int64_t t = a.ids ? a.ids[row] : -1;
        const float lse = a.lse[row];
        float g = a.dlogp && t >= 0 && t < a.cols ? a.dlogp[row] : 0.0f;
        const float at_id = g;
        const float gh = a.dentropy ? a.dentropy[row] : 0.0f;
        // p (gH log p + gH H + g); a row whose lse is NaN has NaN gradients
        g = a.dentropy ? fmaf(gh, a.entropy[row], g) : g;
        if (lse != lse) g = lse;
        auto grad = [&](float v) {
            const float lp = fmaxf(v - lse, -200.0f);   // p is 0 there
            return -exp_of(lp) * fmaf(gh, lp, g);
        };
        RowParts<T> rp(x, a.cols);
        if (((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(dx)) & 15u) != 0) {
            rp.head = 0;
            rp.vecs = 0;
            rp.tail_at = 0;
        }
        const T* xv = x + rp.head;
        T* dv = dx + rp.head;
        const int64_t at_vec = t >= rp.head && t < rp.tail_at ? (t - rp.head) / V : -1;
        const int at_j = (int)((t - rp.head) % V);
        for (int64_t i0 = (int64_t)part * THREADS * U + threadIdx.x; i0 < rp.vecs; i0 += (int64_t)a.split * THREADS * U) {
            uint4 raw[U];
#pragma unroll
            for (int u = 0; u < U; u++)
                if (i0 + u * THREADS < rp.vecs) raw[u] = reinterpret_cast<const uint4*>(xv)[i0 + u * THREADS];
#pragma unroll
            for (int u = 0; u < U; u++) {
                const int64_t i = i0 + u * THREADS;
                if (i >= rp.vecs) break;
                float v[V];
                if constexpr (V == 8) {
                    unpack2<T>(raw[u].x, v[0], v[1]);
                    unpack2<T>(raw[u].y, v[2], v[3]);
                    unpack2<T>(raw[u].z, v[4], v[5]);
                    unpack2<T>(raw[u].w, v[6], v[7]);
                } else {
                    v[0] = __uint_as_float(raw[u].x); v[1] = __uint_as_float(raw[u].y);
                    v[2] = __uint_as_float(raw[u].z); v[3] = __uint_as_float(raw[u].w);
                }
#pragma unroll
                for (int j = 0; j < V; j++) v[j] = grad(v[j]);
                if (i == at_vec) {
#pragma unroll
                    for (int j = 0; j < V; j++)
                        if (j == at_j) v[j] += at_id;
                }
                if constexpr (V == 8) {
                    reinterpret_cast<uint4*>(dv)[i] =
                        make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
                } else {
                    reinterpret_cast<float4*>(dv)[i] = make_float4(v[0], v[1], v[2], v[3]);
                }
            }
        }
        // the rest, one by one
        const int64_t rest = rp.head + (a.cols - rp.tail_at);
        for (int64_t k = (int64_t)part * THREADS + threadIdx.x; k < rest; k += (int64_t)a.split * THREADS) {
            const int64_t e = k < rp.head ? k : rp.tail_at + (k - rp.head);
            float v = grad(to_f32(x[e]));
            if (e == t) v += at_id;
            dx[e] = from_f32<T>(v);
        }
    }
}

}  // namespace

cudaError_t launch_logprobs(const void* x, int type, int64_t rows, int64_t cols, int64_t ldx, const int64_t* ids, int top,
                            float* logp, float* entropy, float* lse, float* top_logp, int64_t* top_ids, cudaStream_t st)
{
    LpArgs a{x, rows, cols, ldx, ids, top, 1, logp, entropy, lse, top_logp, top_ids};
    // Rows that do not fill the SMs are split over clusters of 2, 4 or 8
    // blocks, as long as each has a block of logits.
    const int64_t sms = device_sm_count();
    // Warps of a row: 16 where there are few rows (256 x 65537 fp32, 5
    // alternatives: 24 us, 31 with 8); where many rows' barriers and joins
    // overlap, 8 with alternatives, whose list is a block's (4096 x 49999 bf16, 8
    // of them: 163 us, 185 with 4), and 4 without (87 us, 92 with 8, 122 with 16)
    // or for short rows.
    const bool small = cols <= 4 * 32 * kLpValues * 2, many = rows >= 4 * sms;
    const int size = small || (many && !top) ? 2 : (many ? 1 : 0);
    const int threads = 512 >> size;
    while (a.split < kLpMaxCluster && rows * a.split * 2 <= 2 * sms && cols > (int64_t)a.split * threads * kLpValues) a.split *= 2;
    const int64_t cap = 2 * (2048 / threads) * sms / a.split;
    const unsigned blocks = (unsigned)((rows < cap ? rows : cap) * a.split);
    using Kernel = void (*)(const LpArgs);
    static const Kernel kernels[3][3] = {{logprobs_kernel<ESB_F32, 16>, logprobs_kernel<ESB_F16, 16>, logprobs_kernel<ESB_BF16, 16>},
                                         {logprobs_kernel<ESB_F32, 8>, logprobs_kernel<ESB_F16, 8>, logprobs_kernel<ESB_BF16, 8>},
                                         {logprobs_kernel<ESB_F32, 4>, logprobs_kernel<ESB_F16, 4>, logprobs_kernel<ESB_BF16, 4>}};
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = sizeof(LpShared);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)a.split;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = a.split > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernels[size][type], a);
}

cudaError_t launch_logprobs_grad(const void* x, int type, int64_t rows, int64_t cols, int64_t ldx, const int64_t* ids,
                                 const float* lse, const float* entropy, const float* dlogp, const float* dentropy, void* dx,
                                 int64_t lddx, cudaStream_t st)
{
    LpGradArgs a{x, rows, cols, ldx, ids, lse, entropy, dlogp, dentropy, dx, lddx, 1};
    const int64_t sms = device_sm_count(), per = 256 * 4 * (type == ESB_F32 ? 4 : 8);
    // blocks of a row: enough of them for the SMs, none without values
    while (rows * a.split < 16 * sms && (int64_t)a.split * 2 * per <= cols + per) a.split *= 2;
    const int64_t total = rows * a.split, cap = 8 * sms;
    using Kernel = void (*)(const LpGradArgs);
    static const Kernel kernels[3] = {logprobs_grad_kernel<ESB_F32>, logprobs_grad_kernel<ESB_F16>, logprobs_grad_kernel<ESB_BF16>};
    return launch_pdl(kernels[type], dim3((unsigned)(total < cap ? total : cap)), dim3(256), 0, st, a);
}

}  // namespace esb
