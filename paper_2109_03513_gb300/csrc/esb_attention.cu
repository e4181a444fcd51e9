// esb_attention.cu -- attention of queries over a paged cache of keys and
// values in 4-bit ESB codes.
//
// One pass over the cache with the running maximum and sum of the softmax.  A
// tile is the queries of a sequence that share a head of the cache, up to R =
// 8 NT rows (row = query * group + head in the group).  Places go in stages of
// 16: a warp copies a stage's codes and scales to shared memory some stages
// ahead, decodes them to fp16 (exact: at most 3 significant bits) straight into
// operands of the matrix instruction,
//   S' (16 places x 8 rows)  = K Q'        over the head's values,
//   O' (values x 8 rows)    += V' P'       over the 16 places,
// so that a place's scale is a factor of a row of S' and of a row of P', and
// the rows of a tile are columns everywhere: 8 rows fill an instruction, which
// a single query's group of heads often just does.
//
// Weights carry v's scale: with u = score + log2(v's scale) and M the largest u
// so far (up to 2^8; it is raised when a u passes that), the weight 2^(score -
// M) v_scale is of order 1 whatever the scales are, and is rounded to fp16.
//
// The work, blocks of 64 places of all tiles in a row, is cut into equal parts,
// one for each thread block, wherever that cuts a tile; parts of tiles go to
// the workspace, and a second kernel joins them in their order.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cuda_runtime.h>

#include "esb_internal.h"
#include "esb_rotate.cuh"
#include "esb_rows.cuh"

namespace esb {

namespace {

constexpr int kAtWarps = 4, kAtThreads = 32 * kAtWarps;
constexpr int kAtPlaces = 16;                           // of a stage
constexpr int kAtBlock = kAtPlaces * kAtWarps;          // places of a block of work
constexpr int kAtMinBlocks = 2;                         // of a thread block, while there is enough work

struct AttnArgs {
    const void* q;
    int64_t ldq;
    void* out;
    int64_t ldo;
    float* lse;
    const int32_t *starts, *lens, *pages;
    int64_t ld_pages, tokens;
    const uint32_t *kc, *vc;
    const float *ks, *vs;
    int64_t npages, page_ld, page_lds;
    uint2 klut, vlut;                                   // high bytes of the fp16 numbers of codes 0..7
    int seqs, max_pages, heads, group, D, chunks, page_size, page_shift, window;
    int q_type, out_type, qvec, ovec;
    float scale2;                                       // scale log2(e)
    RotArgs rot;
    float* partial;                                     // slots of R x (DP + 2) floats
    int4* head;                                         // slots
};

// ------------------------------------------------------------ instructions

__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t s)
{
    uint32_t r;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(s));
    return r;
}
__device__ __forceinline__ void mma16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t a)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(a));
    return r;
}
__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float lg2(float x)
{
    float r;
    asm("lg2.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ void copy16(uint32_t to, const void* from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t to, const void* from)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_end_stage() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Eight codes to four pairs of fp16 numbers in their order.  A number of a 4-bit
// set is its high byte (the low one is 0): a permute finds four magnitudes by
// their codes, another spreads the sign bits (it repeats the top bit of a chosen
// byte of 0x80 where the code's top bit is set).
__device__ __forceinline__ void decode8(uint32_t w, const uint2& lut, uint32_t (&r)[4])
{
    const uint32_t m = w & 0x77777777u, wh = w >> 16;
    uint32_t a = prmt(lut.x, lut.y, m), b = prmt(lut.x, lut.y, m >> 16);
    a |= (prmt(0x80808080u, 0x80808080u, w) << 1) & 0x80808080u;
    b |= (prmt(0x80808080u, 0x80808080u, wh) << 1) & 0x80808080u;
    r[0] = prmt(a, 0u, 0x1404u);
    r[1] = prmt(a, 0u, 0x3424u);
    r[2] = prmt(b, 0u, 0x1404u);
    r[3] = prmt(b, 0u, 0x3424u);
}

// ----------------------------------------------------------- shared memory

// A stage: 16 rows of K's codes, 16 of V's, their scales.  Rows are spread so
// that neither the reads of K (a row a quad, all its words) nor those of V (every
// second row, two of a row's words a lane) meet a bank twice.
template <int DP> struct Stage {
    static constexpr int kRow = DP / 2;                 // bytes of a row of codes
    static constexpr int kBytes = 2 * kAtPlaces * kRow + 2 * kAtPlaces * 4;
    static constexpr int kV = kAtPlaces * kRow, kKs = 2 * kV;
    __device__ __forceinline__ static uint32_t at(int row, int chunk)
    {
        if constexpr (DP == 64) return (row >> 2) * 128 + (((row & 3) ^ ((row >> 2) & 1)) * 32) + chunk * 16;
        else if constexpr (DP == 128)
            return (row >> 1) * 128 + ((row ^ (row >> 1)) & 1) * 64 + ((chunk ^ (((row >> 2) & 1) << 1)) * 16);
        else return row * 128 + ((chunk ^ ((row & 1) << 2) ^ (((row >> 1) & 3) << 1)) * 16);
    }
};

template <int DP, int NT, int NP> struct Shape {
    static constexpr int R = 8 * NT, kSteps = DP / 16;
    static constexpr int kStages = DP == 256 ? 4 : 6;
    static constexpr bool kQueryRegs = NT * NP * kSteps <= 16;   // else queries are read from shared memory for every stage
    static constexpr int kSm = NT == 1 ? (DP == 256 ? 3 : 4) : (NT == 2 && DP <= 128 && NP == 1 ? 3 : 2);
    static constexpr int kQueryBytes = NT * NP * kSteps * 32 * 8;
    static constexpr int kRing = kAtWarps * kStages * Stage<DP>::kBytes, kMerge = kAtWarps * R * DP * 4;
    static constexpr int kSums = kAtWarps * R * 8;      // maxima and sums of the warps
    static constexpr int kBytes = (kRing > kMerge ? kRing : kMerge) + kQueryBytes + kSums + 4 * R;
    static constexpr int kSlot = R * (DP + 2);          // floats of a part of a tile
};

// -------------------------------------------------------------------- work

struct Seq {
    int64_t row0;                       // of q
    int nq, len, seen;                  // queries, places in use, places that the page table holds
};
__device__ __forceinline__ Seq sequence(const AttnArgs& a, int b)
{
    Seq s;
    int64_t r0 = b, r1 = b + 1;
    if (a.starts) { r0 = a.starts[b]; r1 = a.starts[b + 1]; }
    r0 = r0 < 0 ? 0 : (r0 > a.tokens ? a.tokens : r0);
    r1 = r1 < r0 ? r0 : (r1 > a.tokens ? a.tokens : r1);
    s.row0 = r0;
    s.nq = (int)(r1 - r0);
    s.len = max(a.lens[b], 0);
    const int64_t held = (int64_t)a.max_pages * a.page_size;
    s.seen = s.len < held ? s.len : (int)held;
    return s;
}
template <int R> __device__ __forceinline__ int tiles_of(const AttnArgs& a, const Seq& s) { return (int)(((int64_t)s.nq * a.group + R - 1) / R); }

struct Tile {
    int lo, hi, blocks;                 // places lo .. hi - 1, lo a multiple of 16; blocks of work (one where there are none)
};
template <int R> __device__ __forceinline__ Tile tile_of(const AttnArgs& a, const Seq& s, int i)
{
    Tile t;
    const int64_t rows = (int64_t)s.nq * a.group, first = (int64_t)i * R, last = min(first + R, rows) - 1;
    const int64_t p0 = (int64_t)s.len - s.nq + first / a.group, p1 = (int64_t)s.len - s.nq + last / a.group;
    t.hi = (int)max((int64_t)0, min(p1 + 1, (int64_t)s.seen));
    t.lo = a.window > 0 ? (int)max((int64_t)0, p0 - a.window + 1) & ~(kAtPlaces - 1) : 0;
    t.blocks = t.hi > t.lo ? (t.hi - t.lo + kAtBlock - 1) / kAtBlock : 1;
    return t;
}

__device__ __forceinline__ int64_t block_sum(int64_t v, int64_t* sh)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < kAtWarps; w++) v += sh[w];
    return v;
}

// Work of sequences b0 + thread (0 past the end), long ones by the whole block.
template <int R>
__device__ __forceinline__ int64_t work_of(const AttnArgs& a, int b0, int64_t* sh)
{
    const int b = b0 + threadIdx.x;
    int64_t w = 0;
    bool many = false;
    if (b < a.seqs) {
        const Seq s = sequence(a, b);
        const int n = tiles_of<R>(a, s);
        many = n > 8;
        if (!many)
            for (int i = 0; i < n; i++) w += tile_of<R>(a, s, i).blocks;
    }
    if (a.starts && __syncthreads_or(many)) {
        __shared__ unsigned list[kAtWarps];
        const unsigned m = __ballot_sync(0xffffffffu, many);
        if ((threadIdx.x & 31) == 0) list[threadIdx.x >> 5] = m;
        __syncthreads();
        for (int k = 0; k < kAtThreads; k++) {
            if (!(list[k >> 5] >> (k & 31) & 1u)) continue;
            const Seq s = sequence(a, b0 + k);
            const int n = tiles_of<R>(a, s);
            int64_t part = 0;
            for (int i = threadIdx.x; i < n; i += kAtThreads) part += tile_of<R>(a, s, i).blocks;
            part = block_sum(part, sh);
            if (threadIdx.x == k) w = part;
        }
        __syncthreads();
    }
    return w * a.heads;
}

// Which of the block's threads holds place `at` of their works in a row, and
// what of `at` is left there.
struct Found {
    int who;
    int64_t rest;
};
__device__ __forceinline__ Found find(int64_t w, int64_t at, int64_t* sh, int64_t& total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t p = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t t = __shfl_up_sync(0xffffffffu, p, o);
        if (lane >= o) p += t;
    }
    __syncthreads();
    if (lane == 31) sh[warp] = p;
    if (threadIdx.x == 0) sh[kAtWarps] = -1;
    __syncthreads();
    total = 0;
    int64_t before = 0;
#pragma unroll
    for (int k = 0; k < kAtWarps; k++) {
        if (k < warp) before += sh[k];
        total += sh[k];
    }
    p += before;                                        // works up to this thread's end
    if (at < p && at >= p - w) {
        sh[kAtWarps] = threadIdx.x;
        sh[kAtWarps + 1] = at - (p - w);
    }
    __syncthreads();
    Found f;
    f.who = (int)sh[kAtWarps];
    f.rest = sh[kAtWarps + 1];
    return f;
}

// ------------------------------------------------------------------ kernel

template <int DP, int NT, int NP>
__global__ void __launch_bounds__(kAtThreads, Shape<DP, NT, NP>::kSm) attention_kernel(const AttnArgs a)
{
    using Sh = Shape<DP, NT, NP>;
    using St = Stage<DP>;
    constexpr int R = Sh::R, STEPS = Sh::kSteps, W = DP / 8, WK = W / 4, WV = W / 8, ST = Sh::kStages;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ int64_t sh[kAtWarps + 2];
    unsigned char* ring = smem;
    float* merge = reinterpret_cast<float*>(smem);
    uint2* qf = reinterpret_cast<uint2*>(smem + (Sh::kRing > Sh::kMerge ? Sh::kRing : Sh::kMerge));
    float2* sums = reinterpret_cast<float2*>(reinterpret_cast<unsigned char*>(qf) + Sh::kQueryBytes);
    float* qscale = reinterpret_cast<float*>(reinterpret_cast<unsigned char*>(sums) + Sh::kSums);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const float ninf = __int_as_float(0xff800000);
    griddep_wait();

    // this block's part of the work: sequence, head, tile and block of places
    const int me = blockIdx.x;
    int4 slot_head[2] = {make_int4(0, 0, 0, 0), make_int4(0, 0, 0, 0)};
    int64_t left = 0, rest = 0;
    int b = 0, head = 0, tile = 0;
    {
        int64_t w = work_of<R>(a, 0, sh), total = 0;
        if (a.seqs <= kAtThreads) total = block_sum(w, sh);
        else
            for (int b0 = 0; b0 < a.seqs; b0 += kAtThreads) total += block_sum(b0 ? work_of<R>(a, b0, sh) : w, sh);
        const int64_t least = total / kAtMinBlocks, n = least < 1 ? 1 : (least < gridDim.x ? least : gridDim.x);
        if (me < n && total > 0) {
            int64_t at = total * me / n;
            left = total * (me + 1) / n - at;
            for (int b0 = 0; b0 < a.seqs; b0 += kAtThreads) {
                if (b0) w = work_of<R>(a, b0, sh);
                int64_t sum;
                const Found f = find(w, at, sh, sum);
                if (f.who >= 0) { b = b0 + f.who; rest = f.rest; break; }
                at -= sum;
            }
            const Seq s = sequence(a, b);
            const int n_tiles = tiles_of<R>(a, s);
            if (n_tiles == 1) {
                const int per = tile_of<R>(a, s, 0).blocks;
                head = (int)(rest / per);
                rest -= (int64_t)head * per;
            } else {
                int64_t per = 0;
                for (int i = threadIdx.x; i < n_tiles; i += kAtThreads) per += tile_of<R>(a, s, i).blocks;
                per = block_sum(per, sh);
                head = (int)(rest / per);
                rest -= (int64_t)head * per;
                for (int i0 = 0; i0 < n_tiles; i0 += kAtThreads) {
                    const int i = i0 + threadIdx.x;
                    int64_t sum;
                    const Found f = find(i < n_tiles ? tile_of<R>(a, s, i).blocks : 0, rest, sh, sum);
                    if (f.who >= 0) { tile = i0 + f.who; rest = f.rest; break; }
                    rest -= sum;
                }
            }
        }
    }

    // where this lane's copies of a stage go
    const int copies = kAtPlaces * a.chunks;
    uint32_t to[W / 8];
#pragma unroll
    for (int i = 0; i < W / 8; i++) {
        const int c = lane + 32 * i;
        to[i] = c < copies ? St::at(c / a.chunks, c % a.chunks) : 0xffffffffu;
    }
    const uint32_t my_ring = smem_u32(ring) + warp * ST * St::kBytes;

    while (left > 0) {
        const Seq s = sequence(a, b);
        const Tile tl = tile_of<R>(a, s, tile);
        const int blocks = (int)min((int64_t)tl.blocks - rest, left), first_block = (int)rest;
        const int64_t rows = (int64_t)s.nq * a.group, row0 = (int64_t)tile * R;
        const int n_rows = (int)min((int64_t)R, rows - row0);

        // queries: rotated, scaled, each row by a power of two that puts its
        // largest below 2^15, as operands of the matrix instruction
        __syncthreads();                                // the last tile's shared memory has been read
        for (int nt = warp; nt < NT; nt += kAtWarps) {
            const int r = nt * 8 + g;
            const bool on = r < n_rows;
            const int64_t row = row0 + (on ? r : 0), token = row / a.group;
            const int64_t at = (s.row0 + token) * a.ldq + ((int64_t)head * a.group + (row - token * a.group)) * a.D;
            const int64_t pos = (int64_t)s.len - s.nq + token;
            float v[WK][8];
            float big = 0.0f;
#pragma unroll
            for (int k = 0; k < WK; k++) {
                const int word = DP == 256 ? (k < 4 ? 4 * t + k : 16 + 4 * t + k - 4) : WK * t + k, d = 8 * word;
                if (on && d < a.D) {
                    if (a.rot.dim) {
                        if (a.q_type == ESB_F32) rotated8(static_cast<const float*>(a.q) + at, a.D, d, a.qvec, a.rot, pos, v[k]);
                        else if (a.q_type == ESB_F16) rotated8(static_cast<const __half*>(a.q) + at, a.D, d, a.qvec, a.rot, pos, v[k]);
                        else rotated8(static_cast<const __nv_bfloat16*>(a.q) + at, a.D, d, a.qvec, a.rot, pos, v[k]);
                    } else {
                        load8_any(a.q, a.q_type, at + d, a.D - d, a.qvec, v[k]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; i++) v[k][i] = 0.0f;
                }
#pragma unroll
                for (int i = 0; i < 8; i++) big = fmaxf(big, fabsf(v[k][i]));
            }
            big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
            big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
            // 2^e takes the largest to 2^14 .. 2^15; the ends of fp32 stay in range
            const int e = big > 0.0f && big < __int_as_float(0x7f800000) ? 14 - max(-112, min(126, ((int)(__float_as_uint(big) >> 23) - 127))) : 0;
            const float up = __uint_as_float((uint32_t)(e / 2 + 127) << 23), up2 = __uint_as_float((uint32_t)(e - e / 2 + 127) << 23);
            if (t == 0) qscale[r] = a.scale2 * __uint_as_float((uint32_t)(127 - e / 2) << 23) * __uint_as_float((uint32_t)(127 - (e - e / 2)) << 23);
#pragma unroll
            for (int k = 0; k < WK; k++) {
#pragma unroll
                for (int i = 0; i < 8; i++) v[k][i] = v[k][i] * up * up2;
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    uint2 hi, lo;
                    hi.x = pack2<__half>(v[k][4 * h], v[k][4 * h + 1]);
                    hi.y = pack2<__half>(v[k][4 * h + 2], v[k][4 * h + 3]);
                    qf[((nt * NP) * STEPS + 2 * k + h) * 32 + lane] = hi;
                    if constexpr (NP == 2) {
                        float x[4];
                        unpack2<__half>(hi.x, x[0], x[1]);
                        unpack2<__half>(hi.y, x[2], x[3]);
                        lo.x = pack2<__half>(v[k][4 * h] - x[0], v[k][4 * h + 1] - x[1]);
                        lo.y = pack2<__half>(v[k][4 * h + 2] - x[2], v[k][4 * h + 3] - x[3]);
                        qf[((nt * NP + 1) * STEPS + 2 * k + h) * 32 + lane] = lo;
                    }
                }
            }
        }
        __syncthreads();
        uint2 qr[Sh::kQueryRegs ? NT * NP * STEPS : 1];
        if constexpr (Sh::kQueryRegs) {
#pragma unroll
            for (int i = 0; i < NT * NP * STEPS; i++) qr[i] = qf[i * 32 + lane];
        }
        // this lane's columns: rows 2 t and 2 t + 1 of every eight
        float fq[NT][2], M[NT][2], L[NT][2];
        int qhi[NT][2], qlo[NT][2];                     // places that they see
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int c = 0; c < 2; c++) {
                const int r = nt * 8 + 2 * t + c;
                const int64_t pos = (int64_t)s.len - s.nq + (row0 + r) / a.group;
                fq[nt][c] = qscale[r];
                M[nt][c] = ninf;
                L[nt][c] = 0.0f;
                qhi[nt][c] = r < n_rows ? (int)max((int64_t)0, min(pos + 1, (int64_t)s.seen)) : 0;
                qlo[nt][c] = a.window > 0 ? (int)max((int64_t)0, pos - a.window + 1) : 0;
            }
        // stages between these are seen by every row
        const int64_t p0 = (int64_t)s.len - s.nq + row0 / a.group, p1 = (int64_t)s.len - s.nq + (row0 + n_rows - 1) / a.group;
        const int all_hi = (int)max((int64_t)0, min(p0 + 1, (int64_t)s.seen)), all_lo = a.window > 0 ? (int)max((int64_t)0, p1 - a.window + 1) : 0;

        float o[DP / 16][NT][4];
#pragma unroll
        for (int i = 0; i < DP / 16; i++)
#pragma unroll
            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                for (int c = 0; c < 4; c++) o[i][nt][c] = 0.0f;

        const int32_t* table = a.pages + (int64_t)b * a.ld_pages;
        const int place0 = tl.lo + (first_block * kAtWarps + warp) * kAtPlaces;
        const int end = min(tl.hi, tl.lo + (first_block + blocks) * kAtBlock);
        const int stages = end > place0 ? (end - place0 + kAtBlock - 1) / kAtBlock : 0;
        auto page_at = [&](int i) {
            const int p = place0 + i * kAtBlock;
            return i < stages ? __ldg(table + (a.page_shift >= 0 ? p >> a.page_shift : p / a.page_size)) : -1;
        };
        int next_page = page_at(0);
        uint32_t there = 0u;                            // which of the ring's stages hold a page that is there
        auto issue = [&](int i) {
            const int page = next_page;
            next_page = page_at(i + 1);
            const uint32_t bit = 1u << (i % ST);
            there &= ~bit;
            if (page >= 0 && page < a.npages) {
                there |= bit;
                const int p = place0 + i * kAtBlock;
                const int in = a.page_shift >= 0 ? p & (a.page_size - 1) : p % a.page_size;
                const int64_t row = (int64_t)head * a.page_size + in;
                const int64_t from = page * a.page_ld + row * (a.chunks * 4);
                const uint32_t base = my_ring + (i % ST) * St::kBytes;
                const uint4* kg = reinterpret_cast<const uint4*>(a.kc + from) + lane;
                const uint4* vg = reinterpret_cast<const uint4*>(a.vc + from) + lane;
#pragma unroll
                for (int k = 0; k < W / 8; k++)
                    if (to[k] != 0xffffffffu) {
                        copy16(base + to[k], kg + 32 * k);
                        copy16(base + St::kV + to[k], vg + 32 * k);
                    }
                const int64_t sc = page * a.page_lds + row;
                copy4(base + St::kKs + 4 * lane, lane < 16 ? a.ks + sc + lane : a.vs + sc + lane - 16);
            }
            copies_end_stage();
        };
#pragma unroll
        for (int i = 0; i < ST - 1; i++) issue(i);

        for (int i = 0; i < stages; i++) {
            copies_wait<ST - 2>();
            __syncwarp();                               // every lane's copies of this stage; all have read the one before
            const bool here = there >> (i % ST) & 1u;
            const unsigned char* sm = ring + warp * ST * St::kBytes + (i % ST) * St::kBytes;
            issue(i + ST - 1);
            if (!here) continue;
            const int place = place0 + i * kAtBlock;

            // scores: rows g and g + 8 of the stage
            float sc[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                for (int c = 0; c < 4; c++) sc[nt][c] = 0.0f;
            {
                uint32_t k0[WK], k1[WK];
                auto words = [&](int row, uint32_t (&w)[WK]) {
                    if constexpr (DP == 64) {
                        const uint2 v = *reinterpret_cast<const uint2*>(sm + St::at(row, t >> 1) + (t & 1) * 8);
                        w[0] = v.x; w[1] = v.y;
                    } else {
#pragma unroll
                        for (int h = 0; h < WK / 4; h++) {
                            const uint4 v = *reinterpret_cast<const uint4*>(sm + St::at(row, t + 4 * h));
                            w[4 * h] = v.x; w[4 * h + 1] = v.y; w[4 * h + 2] = v.z; w[4 * h + 3] = v.w;
                        }
                    }
                };
                words(g, k0);
                words(g + 8, k1);
#pragma unroll
                for (int k = 0; k < WK; k++) {
                    uint32_t x[4], y[4];
                    decode8(k0[k], a.klut, x);
                    decode8(k1[k], a.klut, y);
#pragma unroll
                    for (int h = 0; h < 2; h++)
#pragma unroll
                        for (int nt = 0; nt < NT; nt++)
#pragma unroll
                            for (int p = 0; p < NP; p++) {
                                const int at = (nt * NP + p) * STEPS + 2 * k + h;
                                uint2 q;
                                if constexpr (Sh::kQueryRegs) q = qr[at];
                                else q = qf[at * 32 + lane];
                                mma16(sc[nt], x[2 * h], y[2 * h], x[2 * h + 1], y[2 * h + 1], q.x, q.y);
                            }
                }
            }
            const float* scales = reinterpret_cast<const float*>(sm + St::kKs);
            const float ks0 = scales[g], ks1 = scales[g + 8], vs0 = scales[16 + g], vs1 = scales[24 + g];
            // log2 of v's scales, where they have one
            const float lv0 = fmaxf(fminf(lg2(fabsf(vs0)), 100.0f), -100.0f), lv1 = fmaxf(fminf(lg2(fabsf(vs1)), 100.0f), -100.0f);
            const bool whole = place + kAtPlaces <= all_hi && place >= all_lo;
            bool raise = false;
#pragma unroll
            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                for (int c = 0; c < 2; c++) {
                    sc[nt][c] = sc[nt][c] * ks0 * fq[nt][c];
                    sc[nt][2 + c] = sc[nt][2 + c] * ks1 * fq[nt][c];
                    if (!whole) {
                        if (place + g >= qhi[nt][c] || place + g < qlo[nt][c]) sc[nt][c] = ninf;
                        if (place + g + 8 >= qhi[nt][c] || place + g + 8 < qlo[nt][c]) sc[nt][2 + c] = ninf;
                    }
                    raise |= fmaxf(sc[nt][c] + lv0, sc[nt][2 + c] + lv1) > M[nt][c] + 8.0f;
                }
            if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                    for (int c = 0; c < 2; c++) {
                        float m = fmaxf(sc[nt][c] + lv0, sc[nt][2 + c] + lv1);
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
                        m = fmaxf(m, M[nt][c]);
                        const float f = m > M[nt][c] ? ex2(M[nt][c] - m) : 1.0f;
                        M[nt][c] = m;
                        L[nt][c] *= f;
#pragma unroll
                        for (int k = 0; k < DP / 16; k++) {
                            o[k][nt][c] *= f;
                            o[k][nt][2 + c] *= f;
                        }
                    }
            }
            // weights, turned into the second product's operand
            uint32_t p0[NT][NP], p1[NT][NP];
#pragma unroll
            for (int nt = 0; nt < NT; nt++) {
                float w[4];
#pragma unroll
                for (int c = 0; c < 4; c++) {
                    const float e = sc[nt][c] == ninf ? 0.0f : ex2(sc[nt][c] - M[nt][c & 1]);
                    L[nt][c & 1] += e;
                    w[c] = sc[nt][c] == ninf ? 0.0f : e * (c < 2 ? vs0 : vs1);
                }
                const uint32_t h0 = pack2<__half>(w[0], w[1]), h1 = pack2<__half>(w[2], w[3]);
                p0[nt][0] = transposed(h0);
                p1[nt][0] = transposed(h1);
                if constexpr (NP == 2) {
                    float x[4];
                    unpack2<__half>(h0, x[0], x[1]);
                    unpack2<__half>(h1, x[2], x[3]);
                    p0[nt][NP - 1] = transposed(pack2<__half>(w[0] - x[0], w[1] - x[1]));
                    p1[nt][NP - 1] = transposed(pack2<__half>(w[2] - x[2], w[3] - x[3]));
                }
            }
            // values: this lane's words of places 2 t, 2 t + 1, 2 t + 8, 2 t + 9
            uint32_t v[4][WV];
#pragma unroll
            for (int k = 0; k < 4; k++) {
                const int row = 2 * t + (k & 1) + 8 * (k >> 1);
                const unsigned char* vm = sm + St::kV;
                if constexpr (DP == 64) v[k][0] = *reinterpret_cast<const uint32_t*>(vm + St::at(row, g >> 2) + (g & 3) * 4);
                else if constexpr (DP == 128) {
                    const uint2 x = *reinterpret_cast<const uint2*>(vm + St::at(row, g >> 1) + (g & 1) * 8);
                    v[k][0] = x.x; v[k][1] = x.y;
                } else {
                    const uint4 x = *reinterpret_cast<const uint4*>(vm + St::at(row, g));
                    v[k][0] = x.x; v[k][1] = x.y; v[k][2] = x.z; v[k][3] = x.w;
                }
            }
            // a pair of places' codes of one value next to one another: even values of a word, then odd ones
            auto pair_codes = [](uint32_t x, uint32_t y, int odd) {
                return odd ? ((x >> 4) & 0x0F0F0F0Fu) | (y & 0xF0F0F0F0u) : (x & 0x0F0F0F0Fu) | ((y << 4) & 0xF0F0F0F0u);
            };
            constexpr int PAIRS = WV > 1 ? WV / 2 : 1;
#pragma unroll
            for (int wp = 0; wp < PAIRS; wp++)
#pragma unroll
                for (int odd = 0; odd < 2; odd++) {
                    uint32_t x0[4], x1[4];
                    decode8(pair_codes(v[0][WV > 1 ? 2 * wp : 0], v[1][WV > 1 ? 2 * wp : 0], odd), a.vlut, x0);
                    decode8(pair_codes(v[2][WV > 1 ? 2 * wp : 0], v[3][WV > 1 ? 2 * wp : 0], odd), a.vlut, x1);
                    if constexpr (WV > 1) {
                        // rows g: the first word's values, rows g + 8: the second's
                        uint32_t y0[4], y1[4];
                        decode8(pair_codes(v[0][2 * wp + 1], v[1][2 * wp + 1], odd), a.vlut, y0);
                        decode8(pair_codes(v[2][2 * wp + 1], v[3][2 * wp + 1], odd), a.vlut, y1);
#pragma unroll
                        for (int k = 0; k < 4; k++)
#pragma unroll
                            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                                for (int p = 0; p < NP; p++) mma16(o[8 * wp + 2 * k + odd][nt], x0[k], y0[k], x1[k], y1[k], p0[nt][p], p1[nt][p]);
                    } else {
                        // rows g: values 0..3 of the word, rows g + 8: values 4..7
#pragma unroll
                        for (int k = 0; k < 2; k++)
#pragma unroll
                            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                                for (int p = 0; p < NP; p++) mma16(o[2 * k + odd][nt], x0[k], x0[k + 2], x1[k], x1[k + 2], p0[nt][p], p1[nt][p]);
                    }
                }
        }
        copies_wait<0>();

        // the warps' sums together: each against the largest maximum
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int c = 0; c < 2; c++) {
                float l = L[nt][c];
                l += __shfl_xor_sync(0xffffffffu, l, 4);
                l += __shfl_xor_sync(0xffffffffu, l, 8);
                l += __shfl_xor_sync(0xffffffffu, l, 16);
                if (g == 0) sums[warp * R + nt * 8 + 2 * t + c] = make_float2(M[nt][c], l);
            }
        __syncthreads();                                // the warps are done with their rings
        // value e of a lane's column: the lane's 16 (8, 32) values in a row
        constexpr int PER = DP / 8;
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int c = 0; c < 2; c++) {
                float* to_row = merge + (warp * R + nt * 8 + 2 * t + c) * DP + g * PER;
#pragma unroll
                for (int e = 0; e < PER; e += 4) {
                    float x[4];
#pragma unroll
                    for (int k = 0; k < 4; k++) {
                        const int d = e + k;
                        // words of a lane in pairs: rows g of the first word's tiles, rows g + 8 of the second's
                        const int i = DP == 64 ? d & 3 : (d >> 4) * 8 + (d & 7), up = DP == 64 ? d >> 2 : (d >> 3) & 1;
                        x[k] = o[i][nt][2 * up + c];
                    }
                    *reinterpret_cast<float4*>(to_row + e) = make_float4(x[0], x[1], x[2], x[3]);
                }
            }
        __syncthreads();
        const bool begins = first_block == 0, ends = first_block + blocks == tl.blocks;
        const int which = begins ? 1 : 0;
        float* slot = a.partial + (int64_t)(2 * me + which) * Sh::kSlot;
        for (int i = threadIdx.x; i < n_rows * (DP / 8); i += kAtThreads) {
            const int r = i / (DP / 8), d = (i - r * (DP / 8)) * 8;
            if (d >= a.D) continue;
            float m = ninf, l = 0.0f, f[kAtWarps], y[8];
#pragma unroll
            for (int w = 0; w < kAtWarps; w++) m = fmaxf(m, sums[w * R + r].x);
#pragma unroll
            for (int k = 0; k < 8; k++) y[k] = 0.0f;
#pragma unroll
            for (int w = 0; w < kAtWarps; w++) {
                const float2 x = sums[w * R + r];
                f[w] = x.x == ninf ? 0.0f : ex2(x.x - m);
                // a sum that is NaN without a maximum stays NaN
                l += x.x == ninf ? (x.y == x.y ? 0.0f : x.y) : f[w] * x.y;
                const float* from = merge + (w * R + r) * DP + d;
#pragma unroll
                for (int k = 0; k < 8; k++) y[k] = x.x == ninf ? y[k] : fmaf(f[w], from[k], y[k]);
            }
            if (begins && ends) {
                const int64_t row = row0 + r, token = row / a.group;
                const int64_t qh = (int64_t)head * a.group + (row - token * a.group);
                const float inv = l == 0.0f ? 0.0f : __fdiv_rn(1.0f, l);
#pragma unroll
                for (int k = 0; k < 8; k++) y[k] = l == 0.0f ? 0.0f : (l == l ? y[k] * inv : l);
                store8_any(a.out, a.out_type, (s.row0 + token) * a.ldo + qh * a.D + d, a.D - d, a.ovec, y);
                if (a.lse && d == 0)
                    a.lse[(s.row0 + token) * ((int64_t)a.heads * a.group) + qh] = l == 0.0f ? ninf : (m == ninf ? l : m * 0.69314718f + logf(l));
            } else {
                store8<float>(slot + (int64_t)r * DP + d, y);
                if (d == 0) {
                    slot[R * DP + r] = m;
                    slot[R * DP + R + r] = l;
                }
            }
        }
        if (!(begins && ends)) {
            const int4 h = make_int4(ends ? 3 : 1, b, head, tile);
            if (begins) slot_head[1] = h;
            else slot_head[0] = h;
        }
        left -= blocks;
        rest = 0;
        if (ends) {
            if (++tile >= tiles_of<R>(a, s)) {
                tile = 0;
                if (++head >= a.heads) {
                    head = 0;
                    // the next sequence with queries
                    while (left > 0 && ++b < a.seqs)
                        if (sequence(a, b).nq > 0) break;
                    if (b >= a.seqs) break;
                }
            }
        }
    }
    if (threadIdx.x < 2) a.head[2 * me + threadIdx.x] = slot_head[threadIdx.x];
}

// Joins the parts of a tile that begins in part `x` of the work and goes on in
// the following ones.
template <int DP, int R>
__global__ void __launch_bounds__(128) attention_join_kernel(const AttnArgs a, int parts)
{
    constexpr int SLOT = R * (DP + 2);
    griddep_wait();
    const int p0 = blockIdx.x;
    const int4 h = a.head[2 * p0 + 1];
    if (!(h.x & 1)) return;
    const Seq s = sequence(a, h.y);
    const int64_t row = (int64_t)h.w * R + blockIdx.y, rows = (int64_t)s.nq * a.group;
    if (row >= rows) return;
    const int r = blockIdx.y;
    // the part that ends the tile
    __shared__ int last;
    if (threadIdx.x == 0) last = parts - 1;
    __syncthreads();
    for (int base = p0 + 1; base < parts; base += 128) {
        const int p = base + threadIdx.x;
        if (p < parts && (a.head[2 * p].x & 3) == 3) atomicMin(&last, p);
        __syncthreads();
        const bool found = last < base + 128;
        __syncthreads();
        if (found) break;
    }
    const int n = last - p0 + 1;
    auto slot = [&](int i) { return a.partial + (int64_t)(i == 0 ? 2 * p0 + 1 : 2 * (p0 + i)) * SLOT; };
    __shared__ float wm[4];
    const float ninf = __int_as_float(0xff800000);
    float m = ninf;
    for (int i = threadIdx.x; i < n; i += 128) m = fmaxf(m, slot(i)[R * DP + r]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if ((threadIdx.x & 31) == 0) wm[threadIdx.x >> 5] = m;
    __syncthreads();
    m = fmaxf(fmaxf(wm[0], wm[1]), fmaxf(wm[2], wm[3]));
    // four values a thread and, where a row has fewer than 128 threads' worth, every few parts
    constexpr int T = DP / 4, WAYS = 128 / T > 0 ? 128 / T : 1;
    const int d = threadIdx.x % T * 4, way = threadIdx.x / T;
    float y[4] = {0.0f, 0.0f, 0.0f, 0.0f}, l = 0.0f;
#pragma unroll 4
    for (int i = way; i < n; i += WAYS) {
        const float* p = slot(i);
        const float pm = p[R * DP + r], pl = p[R * DP + R + r];
        const float4 v = *reinterpret_cast<const float4*>(p + r * DP + d);
        if (pm == ninf) {
            l += pl == pl ? 0.0f : pl;
            continue;
        }
        const float f = ex2(pm - m);
        l = fmaf(f, pl, l);
        y[0] = fmaf(f, v.x, y[0]); y[1] = fmaf(f, v.y, y[1]); y[2] = fmaf(f, v.z, y[2]); y[3] = fmaf(f, v.w, y[3]);
    }
    __shared__ float parts_of[WAYS][T][5];
    float* mine = parts_of[way][threadIdx.x % T];
    mine[0] = y[0]; mine[1] = y[1]; mine[2] = y[2]; mine[3] = y[3]; mine[4] = l;
    __syncthreads();
    if (way != 0 || d >= a.D) return;
#pragma unroll
    for (int k = 1; k < WAYS; k++) {
        const float* p = parts_of[k][threadIdx.x % T];
        y[0] += p[0]; y[1] += p[1]; y[2] += p[2]; y[3] += p[3]; l += p[4];
    }
    const int64_t token = row / a.group, qh = (int64_t)h.z * a.group + (row - token * a.group);
    const float inv = l == 0.0f ? 0.0f : __fdiv_rn(1.0f, l);
    const int64_t at = (s.row0 + token) * a.ldo + qh * a.D + d;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        const float v = l == 0.0f ? 0.0f : (l == l ? y[k] * inv : l);
        if (a.out_type == ESB_F32) static_cast<float*>(a.out)[at + k] = v;
        else if (a.out_type == ESB_F16) static_cast<__half*>(a.out)[at + k] = from_f32<__half>(v);
        else static_cast<__nv_bfloat16*>(a.out)[at + k] = from_f32<__nv_bfloat16>(v);
    }
    if (a.lse && d == 0)
        a.lse[(s.row0 + token) * ((int64_t)a.heads * a.group) + qh] = l == 0.0f ? ninf : (m == ninf ? l : m * 0.69314718f + logf(l));
}

template <int DP, int NT, int NP>
cudaError_t run_attention(const AttnArgs& in, void* workspace, cudaStream_t st)
{
    using Sh = Shape<DP, NT, NP>;
    AttnArgs a = in;
    const int parts = device_sm_count() * Sh::kSm;
    a.head = static_cast<int4*>(workspace);
    a.partial = reinterpret_cast<float*>(a.head + 2 * parts);
    cudaError_t e = cudaFuncSetAttribute(attention_kernel<DP, NT, NP>, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::kBytes);
    if (e != cudaSuccess) return e;
    e = launch_pdl(attention_kernel<DP, NT, NP>, dim3((unsigned)parts), dim3(kAtThreads), Sh::kBytes, st, a);
    if (e != cudaSuccess) return e;
    return launch_pdl(attention_join_kernel<DP, Sh::R>, dim3((unsigned)parts, Sh::R), dim3(128), 0, st, a, parts);
}
template <int DP, int NT, int NP> size_t workspace_of()
{
    using Sh = Shape<DP, NT, NP>;
    return (size_t)(device_sm_count() * Sh::kSm) * 2 * (sizeof(int4) + sizeof(float) * Sh::kSlot);
}

// Eights of rows in a tile: those of an average sequence, as far as their sums fit the registers.
int eights_of(int64_t tokens, int64_t seqs, int group, int DP, int NP)
{
    const int64_t rows = (tokens + seqs - 1) / seqs * group;
    const int most = DP == 256 ? (NP == 1 ? 2 : 1) : (DP == 128 && NP == 2 ? 2 : 4);
    return rows <= 8 || most == 1 ? 1 : (rows <= 16 || most == 2 ? 2 : 4);
}
int padded(int D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }
int planes(int q_type) { return q_type == ESB_BF16 ? 1 : 2; }

// f<DP, NT, NP>() for a shape
template <class F>
auto with_shape(int DP, int NT, int NP, F f)
{
#define CASE(D, N, P) if (DP == D && NT == N && NP == P) return f.template operator()<D, N, P>()
    CASE(64, 1, 1); CASE(64, 2, 1); CASE(64, 4, 1); CASE(64, 1, 2); CASE(64, 2, 2); CASE(64, 4, 2);
    CASE(128, 1, 1); CASE(128, 2, 1); CASE(128, 4, 1); CASE(128, 1, 2); CASE(128, 2, 2);
    CASE(256, 1, 1); CASE(256, 2, 1);
#undef CASE
    return f.template operator()<256, 1, 2>();
}
struct RunShape {
    const AttnArgs& a;
    void* workspace;
    cudaStream_t st;
    template <int DP, int NT, int NP> cudaError_t operator()() const { return run_attention<DP, NT, NP>(a, workspace, st); }
};
struct SizeShape {
    template <int DP, int NT, int NP> size_t operator()() const { return workspace_of<DP, NT, NP>(); }
};

// High bytes of the fp16 numbers of codes 0..7 of a 4-bit set.
uint2 lut_of(int k)
{
    uint32_t w[2] = {0u, 0u};
    const int n = (1 << (3 - k)) - 1;
    for (int c = 0; c < 8; c++) {
        const int e = (c >> k) & n, f = c & ((1 << k) - 1);
        const double v = e == n ? std::ldexp((double)f, -k) : std::ldexp(1.0 + std::ldexp((double)f, -k), e);
        uint32_t h = 0u;
        if (v > 0.0) {
            int x;
            const double m = std::frexp(v, &x) * 2.0 - 1.0;     // v = (1 + m) 2^(x - 1)
            h = (uint32_t)((x - 1 + 15) << 2) | (uint32_t)(m * 4.0);
        }
        w[c / 4] |= h << (8 * (c % 4));
    }
    return make_uint2(w[0], w[1]);
}

}  // namespace

size_t attention_workspace_bytes(int64_t tokens, int64_t seqs, int q_heads, int heads, int head_dim, int q_type)
{
    const int DP = padded(head_dim), NP = planes(q_type);
    return with_shape(DP, eights_of(tokens, seqs, q_heads / heads, DP, NP), NP, SizeShape());
}

cudaError_t launch_attention(int64_t tokens, const esb_kv_cache& c, const esb_attention& n, void* workspace, cudaStream_t st)
{
    AttnArgs a = {};
    auto rows16 = [](const void* p, int64_t ld, int type) {
        return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld * type_bytes(type) % 16 == 0;
    };
    a.q = n.q; a.ldq = n.ldq; a.out = n.out; a.ldo = n.ldo; a.lse = n.lse;
    a.starts = n.starts; a.lens = n.lens; a.pages = n.pages; a.ld_pages = n.ld_pages; a.tokens = tokens;
    a.kc = c.k_codes; a.vc = c.v_codes; a.ks = c.k_scales; a.vs = c.v_scales;
    a.npages = c.pages; a.page_ld = c.page_ld; a.page_lds = c.page_lds;
    a.klut = lut_of(c.k_fmt.k); a.vlut = lut_of(c.v_fmt.k);
    a.seqs = n.seqs; a.max_pages = n.max_pages; a.heads = c.heads; a.group = n.q_heads / c.heads; a.D = c.head_dim;
    a.chunks = (c.head_dim + 31) / 32; a.page_size = c.page_size;
    a.page_shift = -1;
    for (int i = 4; i < 31; i++)
        if (c.page_size == 1 << i) a.page_shift = i;
    a.window = n.window; a.q_type = n.q_type; a.out_type = n.out_type;
    a.qvec = rows16(n.q, n.ldq, n.q_type); a.ovec = rows16(n.out, n.ldo, n.out_type);
    a.scale2 = (float)((double)n.scale * 1.4426950408889634);
    a.rot = make_rot(n.rotation, c.head_dim);
    const int DP = padded(a.D), NP = planes(n.q_type);
    return with_shape(DP, eights_of(tokens, n.seqs, a.group, DP, NP), NP, RunShape{a, workspace, st});
}

}  // namespace esb
