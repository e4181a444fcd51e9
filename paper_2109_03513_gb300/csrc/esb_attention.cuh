// esb_attention.cuh -- attention of queries over a paged cache of keys and
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
// M) v_scale is of order 1 whatever the scales are.  It is rounded to fp16 as
// 2^7 times that, so that the largest lies in 2^7 .. 2^15 and fp16's fixed steps
// of 2^-24, of which a long rest behind one large weight is made, are 2^-31 of it
// or less.  With two planes the second holds 2^11 times what the first leaves,
// in steps of 2^-35 (2^-42 of the largest), and is summed apart.
//
// The work, blocks of places (a stage of each of four warps) of all tiles in a
// row, is cut into equal parts, one for each thread block, wherever that cuts a
// tile; parts of tiles go to the workspace, and a second kernel joins them in
// their order.
//
// 4 x 131072 places, 8 heads of 128, 4 queries each (570 MB): 134 us, 4.25 TB/s,
// 63% of the copy rate.  More than half of the instructions go to the pipe of
// integer and permute work, which does 64 lanes a clock and is 65% busy (a launch by
// itself, its starts among it); after it warps wait for fixed latencies and one
// another.  A prompt's 512 tokens over 4096 places, four of them (129 GFLOP):
// 614 us, 210 TFLOP/s; its tiles' sums leave two warps a scheduler, which wait for
// fixed latencies.  One sequence of 2048 places: 11 us, two kernels' starts,
// look-ups and loads one after the other.
#pragma once

#include <algorithm>
#include <atomic>
#include <cstdint>
#include <cuda_runtime.h>

#include "esb_attention_plan.h"
#include "esb_internal.h"
#include "esb_rotate.cuh"
#include "esb_rows.cuh"

namespace esb {

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
    int64_t npages;
    uint32_t page16, page_lds;                          // a page in 16 bytes of codes, and in scales
    uint2 klut, vlut;                                   // high bytes of the fp16 numbers of codes 0..7; LIN: x = what turns a code into its place
    int seqs, max_pages, heads, group, group_shift, D, chunks, page_size, window;
    int q_type, out_type, qvec, ovec;
    float scale2, vunit;                                // scale log2(e) and K's unit, below 1 and times 2^scale_up; V's unit, and the weights'
    int scale_up;
    RotArgs rot;
    float* partial;                                     // slots of R x (DP + 2) floats
    int4* head;                                         // of each part: (the last part of the tile that begins in it and goes on) + 1, sequence, head, tile
};

namespace {

constexpr int kAtWarps = 4, kAtThreads = 32 * kAtWarps;
constexpr int kAtPlaces = 16;                           // of a part of a stage, the matrix instruction's rows
// The maximum of no scores: the least finite number, from which a score of -inf
// (a seen place's, or one that is not seen) is still -inf away, not NaN.
constexpr int kNone = (int)0xff7fffffu;

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
// What a weight is multiplied by before it is rounded to fp16, and what its first
// plane's remainder is before that is.
constexpr float kWeightUp = 128.0f, kLowUp = 2048.0f;

__device__ __forceinline__ void mma16_zero(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}
// The instruction's sums are truncated, not rounded: where queries and weights
// have 22 bits, a place's products are summed on their own and added in fp32.
__device__ __forceinline__ void mma16_add(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, const uint32_t (&b0)[2], const uint32_t (&b1)[2])
{
    float x[4], y[4];
    mma16_zero(x, a0, a1, a2, a3, b0[1], b1[1]);
    mma16_zero(y, a0, a1, a2, a3, b0[0], b1[0]);
#pragma unroll
    for (int i = 0; i < 4; i++) d[i] = fmaf(x[i], 1.0f / kLowUp, d[i]) + y[i];
}
__device__ __forceinline__ void mma16_add(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, const uint32_t (&b0)[1], const uint32_t (&b1)[1])
{
    mma16(d, a0, a1, a2, a3, b0[0], b1[0]);
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
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
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

template <int N>
__device__ __forceinline__ void lds(uint32_t at, uint32_t (&w)[N])
{
    if constexpr (N == 1) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[0]) : "r"(at) : "memory");
    else if constexpr (N == 2) asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at) : "memory");
    else asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ float lds_f32(uint32_t at)
{
    uint32_t w[1];
    lds(at, w);
    return __uint_as_float(w[0]);
}

// Eight codes to four pairs of fp16 numbers, codes i and i + 4 in pair i.
// LIN, sets of one spacing (k = 2, 3): a number is its place among 0..7 with a
// sign, and a place in bits 8..10 of an fp16 number is that many 2^-16 (below
// 2^11 of its last places fp16 is fixed point), so no table is needed.  Other
// sets: a number is its high byte, found by a permute with its code.  Signs and
// places are put in order for four codes at once, then spread; a shift to the
// left is a multiplication, on the pipe that has nothing to do.
// Ten instructions a word (thirteen with the table), nine and twelve of them on
// the pipe that bounds the kernel.  (Signs spread by a second permute and tables
// for all sets: fourteen, and 4 x 131072 places in 237 us where these took 186.)
template <bool LIN>
__device__ __forceinline__ void decode8(uint32_t w, const uint2& lut, uint32_t (&r)[4])
{
    uint32_t a, b;                                      // codes 0, 2, 4, 6 and 1, 3, 5, 7 as bytes
    if constexpr (LIN) {
        a = (w & 0x07070707u) ^ (((w * 16u) & 0x80808080u) | lut.x);
        b = ((w >> 4) & 0x07070707u) ^ ((w & 0x80808080u) | lut.x);
    } else {
        const uint32_t m = w & 0x77777777u;
        const uint32_t x = prmt(lut.x, lut.y, m), y = prmt(lut.x, lut.y, m >> 16);
        a = prmt(x, y, 0x6420u) | ((w * 16u) & 0x80808080u);
        b = prmt(x, y, 0x7531u) | (w & 0x80808080u);
    }
    r[0] = prmt(a, 0u, 0x2404u);
    r[1] = prmt(b, 0u, 0x2404u);
    r[2] = a & 0xFF00FF00u;
    r[3] = b & 0xFF00FF00u;
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
    static constexpr int kParts = NT == 1 ? 2 : 1;      // of a stage: few rows share its fixed work over more places (169 us, 180 with one, for 4 x 131072 then)
    static constexpr int kBlock = kAtPlaces * kParts * kAtWarps;    // places of a block of work
    static constexpr int kMinBlocks = NT == 1 ? 1 : 2;  // of a thread block, while there is enough work
    static constexpr int kStages = DP == 256 ? (NT == 1 ? 3 : 4) : NT == 1 ? 3 : 6;
    static constexpr bool kQueryRegs = NT * NP * kSteps <= 16;   // else queries are read from shared memory for every stage
    // Blocks on an SM.  Tiles of 16 rows: 49 us for 24 x 10000 places, 55 with three blocks, whose registers spill;
    // heads of 64: 37 us for 48 windows of 1000, 39.5 with three; of 128: 137 us for 4 x 131072 places, 148 with four
    // (measured then; 45, 35 and 134 us now).  One plane each but for the windows: two planes of heads of 128 spill 88 bytes
    // at three blocks, and were not measured with two.
    static constexpr int kSm = NT > 1 || DP == 256 ? 2 : DP == 64 ? 4 : 3;
    static constexpr int kQueryBytes = NT * NP * kSteps * 32 * 8;
    static constexpr int kRing = kAtWarps * kStages * kParts * Stage<DP>::kBytes, kMerge = kAtWarps * R * DP * 4;
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
// Rows of a sequence's tiles: below 2^31.
__device__ __forceinline__ uint32_t token_of(const AttnArgs& a, uint32_t row) { return a.group_shift >= 0 ? row >> a.group_shift : row / (uint32_t)a.group; }
// Most quotients of 64 bits are of numbers of 32.
__device__ __forceinline__ int64_t quotient(int64_t x, int64_t y)
{
    return ((x | y) >> 32) == 0 ? (int64_t)((uint32_t)x / (uint32_t)y) : x / y;
}
template <class Sh> __device__ __forceinline__ int tiles_of(const AttnArgs& a, const Seq& s) { return (s.nq * a.group + Sh::R - 1) / Sh::R; }

template <class Sh> __device__ __forceinline__ Tile tile_of(const AttnArgs& a, const Seq& s, int i)
{
    const uint32_t rows = (uint32_t)(s.nq * a.group), first = (uint32_t)i * Sh::R, last = min(first + Sh::R, rows) - 1u;
    const int64_t p0 = (int64_t)s.len - s.nq + token_of(a, first), p1 = (int64_t)s.len - s.nq + token_of(a, last);
    return tile_places(p0, p1, s.seen, a.window, kAtPlaces * Sh::kParts, Sh::kBlock);
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

// Work of sequence first + thread * step, for the first `count` threads; those
// with many tiles by the whole block.  A single query's tiles see the same places.
// (One copy of it: a block runs this once, out of a cold instruction cache.)
template <class Sh>
__device__ __noinline__ int64_t work_of(const AttnArgs& a, int64_t first, int64_t step, int count, int64_t* sh)
{
    const int64_t b = first + threadIdx.x * step;
    int64_t w = 0;
    bool many = false;
    if ((int)threadIdx.x < count && b < a.seqs) {
        const Seq s = sequence(a, (int)b);
        const int n = tiles_of<Sh>(a, s);
        many = s.nq > 1 && n > 8;
        if (s.nq == 1) w = (int64_t)n * tile_of<Sh>(a, s, 0).blocks;
        else if (!many)
            for (int i = 0; i < n; i++) w += tile_of<Sh>(a, s, i).blocks;
    }
    if (a.starts && __syncthreads_or(many)) {          // else every sequence has one query
        __shared__ unsigned list[kAtWarps];
        const unsigned m = __ballot_sync(0xffffffffu, many);
        if ((threadIdx.x & 31) == 0) list[threadIdx.x >> 5] = m;
        __syncthreads();
        for (int k = 0; k < kAtThreads; k++) {
            if (!(list[k >> 5] >> (k & 31) & 1u)) continue;
            const Seq s = sequence(a, (int)(first + k * step));
            const int n = tiles_of<Sh>(a, s);
            int64_t part = 0;
            for (int i = threadIdx.x; i < n; i += kAtThreads) part += tile_of<Sh>(a, s, i).blocks;
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
__device__ __noinline__ Found find(int64_t w, int64_t at, int64_t* sh, int64_t& total)
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

template <int DP, int NT, int NP, bool LIN>
__global__ void __launch_bounds__(kAtThreads, Shape<DP, NT, NP>::kSm) attention_kernel(const __grid_constant__ AttnArgs a)
{
    using Sh = Shape<DP, NT, NP>;
    using St = Stage<DP>;
    constexpr int R = Sh::R, W = DP / 8, WK = W / 4, WV = W / 8, ST = Sh::kStages, SUB = Sh::kParts, BLOCK = Sh::kBlock, BYTES = SUB * St::kBytes;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ int64_t sh[kAtWarps + 2];
    unsigned char* ring = smem;
    float* merge = reinterpret_cast<float*>(smem);
    uint4* qf = reinterpret_cast<uint4*>(smem + (Sh::kRing > Sh::kMerge ? Sh::kRing : Sh::kMerge));
    float2* sums = reinterpret_cast<float2*>(reinterpret_cast<unsigned char*>(qf) + Sh::kQueryBytes);
    float* qscale = reinterpret_cast<float*>(reinterpret_cast<unsigned char*>(sums) + Sh::kSums);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const float ninf = __int_as_float(0xff800000), none = __int_as_float(kNone);
    griddep_wait();
    griddep_launch_dependents();        // every block runs at once, so those of the join only fill what is left

    // this block's part of the work: sequence, head, tile and block of places
    const int me = blockIdx.x;
    int4 goes_on = make_int4(0, 0, 0, 0);
    int64_t left = 0, rest = 0, at_block = 0, share = 1, larger = 0;    // the first `larger` blocks have one more than `share`
    int b = 0, head = 0, tile = 0;
    {
        // each thread sums a run of sequences
        const int run = run_of(a.seqs, kAtThreads);
        int64_t w = 0;
#pragma unroll 1
        for (int i = 0; i < run; i++) w += work_of<Sh>(a, i, run, kAtThreads, sh);
        const int64_t total = block_sum(w, sh);
        const int64_t least = total / Sh::kMinBlocks, n = least < 1 ? 1 : (least < gridDim.x ? least : gridDim.x);
        if (me < n && total > 0) {
            share = quotient(total, n);
            larger = total - share * n;
            int64_t at = share * me + min((int64_t)me, larger);
            left = share + (me < larger ? 1 : 0);
            at_block = at;
            int64_t sum;
            Found f = find(w, at, sh, sum);
            b = f.who * run;
            rest = f.rest;
            for (int i = 0; run > 1 && i < run; i += kAtThreads) {
                f = find(work_of<Sh>(a, b + i, 1, min(run - i, kAtThreads), sh), rest, sh, sum);
                if (f.who >= 0) { b += i + f.who; rest = f.rest; break; }
                rest -= sum;
            }
            const Seq s = sequence(a, b);
            const int n_tiles = tiles_of<Sh>(a, s);
            if (n_tiles == 1) {
                const int per = tile_of<Sh>(a, s, 0).blocks;
                head = (int)quotient(rest, per);
                rest -= (int64_t)head * per;
            } else {
                int64_t per = 0;
                for (int i = threadIdx.x; i < n_tiles; i += kAtThreads) per += tile_of<Sh>(a, s, i).blocks;
                per = block_sum(per, sh);
                head = (int)quotient(rest, per);
                rest -= (int64_t)head * per;
                for (int i0 = 0; i0 < n_tiles; i0 += kAtThreads) {
                    const int i = i0 + threadIdx.x;
                    int64_t sum;
                    const Found f = find(i < n_tiles ? tile_of<Sh>(a, s, i).blocks : 0, rest, sh, sum);
                    if (f.who >= 0) { tile = i0 + f.who; rest = f.rest; break; }
                    rest -= sum;
                }
            }
        }
    }

    // where this lane's copies of a stage go
    const int copies = kAtPlaces * a.chunks;
    uint32_t to[W / 8];
    bool mine[W / 8];
#pragma unroll
    for (int i = 0; i < W / 8; i++) {
        const int c = lane + 32 * i;
        mine[i] = c < copies;
        to[i] = mine[i] ? St::at(c / a.chunks, c % a.chunks) : 0u;
    }
    const uint32_t my_ring = smem_u32(ring) + warp * ST * BYTES, ring_end = my_ring + ST * BYTES;
    // and where it reads: rows g (and 8 further) of K, rows 2 t and 2 t + 1 of V
    const uint32_t k_from = DP == 64 ? St::at(g, t >> 1) + (t & 1) * 8 : St::at(g, t);
    const uint32_t v_in = DP == 64 ? (g & 3) * 4 : DP == 128 ? (g & 1) * 8 : 0, v_chunk = DP == 64 ? g >> 2 : DP == 128 ? g >> 1 : g;
    const uint32_t v_from0 = St::kV + St::at(2 * t, v_chunk) + v_in, v_from1 = St::kV + St::at(2 * t + 1, v_chunk) + v_in;

    while (left > 0) {
        const Seq s = sequence(a, b);
        const Tile tl = tile_of<Sh>(a, s, tile);
        const int blocks = (int)min((int64_t)tl.blocks - rest, left), first_block = (int)rest;
        const uint32_t row0 = (uint32_t)tile * R;
        const int n_rows = (int)min((uint32_t)R, (uint32_t)(s.nq * a.group) - row0);

        __syncthreads();                                // the last tile's shared memory has been read
        const int32_t* table = a.pages + (int64_t)b * a.ld_pages;
        const int place0 = first_place(tl, first_block, warp, kAtWarps, kAtPlaces * SUB), end = end_place(tl, first_block, blocks, BLOCK);
        const int stages = end > place0 ? (end - place0 + BLOCK - 1) / BLOCK : 0;
        const int64_t head_row = (int64_t)head * a.page_size;
        const char* kg = reinterpret_cast<const char*>(a.kc) + (head_row * a.chunks + lane) * 16;
        const char* vg = reinterpret_cast<const char*>(a.vc) + (head_row * a.chunks + lane) * 16;
        const float* sg = (lane < 16 ? a.ks : a.vs) + head_row + (lane & 15);
        // The next stage that is copied: its places' page in the table and place in
        // it, and the page's number; the second part's, where that may be another page.
        const bool one_page = SUB == 1 || a.page_size % (kAtPlaces * SUB) == 0;
        int look_place = place0, entry = place0 / a.page_size, in = place0 - entry * a.page_size;
        const int step_entry = BLOCK / a.page_size, step_in = BLOCK - step_entry * a.page_size;
        int next_page[SUB], next_in[SUB];
        auto look = [&]() {
            next_in[0] = in;
            next_page[0] = look_place < end ? __ldg(table + entry) : -1;
            if constexpr (SUB == 2) {
                next_page[SUB - 1] = next_page[0];
                next_in[SUB - 1] = in + kAtPlaces;
                if (!one_page && in + kAtPlaces == a.page_size) {
                    next_page[SUB - 1] = look_place + kAtPlaces < end ? __ldg(table + entry + 1) : -1;
                    next_in[SUB - 1] = 0;
                }
            }
            look_place += BLOCK;
            entry += step_entry;
            in += step_in;
            if (in >= a.page_size) { in -= a.page_size; entry++; }
        };
        look();
        uint32_t issue_to = my_ring, there = 0u;        // the ring's next stage; which of the last parts hold a page that is there
        auto issue = [&]() {
            int pages[SUB], ins[SUB];
#pragma unroll
            for (int h = 0; h < SUB; h++) { pages[h] = next_page[h]; ins[h] = next_in[h]; }
            look();
#pragma unroll
            for (int h = 0; h < SUB; h++) {
                const uint32_t page = (uint32_t)pages[h];
                there *= 2u;
                if (page >= (uint32_t)a.npages) continue;
                there++;
                const uint64_t at = (uint64_t)page * a.page16 + (uint32_t)(ins[h] * a.chunks);
                const char *k = kg + at * 16, *v = vg + at * 16;
                const uint32_t dst = issue_to + h * St::kBytes;
#pragma unroll
                for (int c = 0; c < W / 8; c++)
                    if (mine[c]) {
                        copy16(dst + to[c], k + 512 * c);
                        copy16(dst + to[c] + St::kV, v + 512 * c);
                    }
                copy4(dst + St::kKs + 4 * lane, sg + (uint64_t)page * a.page_lds + ins[h]);
            }
            copies_end_stage();
            issue_to = issue_to + BYTES == ring_end ? my_ring : issue_to + BYTES;
        };
#pragma unroll
        for (int i = 0; i < ST - 1; i++) issue();

        // queries: rotated, scaled, each row by a power of two that puts its
        // largest below 2^15, as operands of the matrix instruction
        // (a thread for each eight values, which are a word of K's codes)
        for (int i = threadIdx.x; i < R * W; i += kAtThreads) {
            const int r = i / W, word = i % W, d = 8 * word;
            const bool on = r < n_rows && d < a.D;
            const uint32_t row = row0 + (r < n_rows ? r : 0), token = token_of(a, row);
            const int64_t at = (s.row0 + token) * a.ldq + ((int64_t)head * a.group + (row - token * a.group)) * a.D;
            const int64_t pos = (int64_t)s.len - s.nq + token;
            float v[8], big = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; e++) v[e] = 0.0f;
            if (on) {
                if (!a.rot.dim) load8_any(a.q, a.q_type, at + d, a.D - d, a.qvec, v);
                else if (a.q_type == ESB_F32) rotated8(static_cast<const float*>(a.q) + at, a.D, d, a.qvec, a.rot, pos, v);
                else if (a.q_type == ESB_F16) rotated8(static_cast<const __half*>(a.q) + at, a.D, d, a.qvec, a.rot, pos, v);
                else rotated8(static_cast<const __nv_bfloat16*>(a.q) + at, a.D, d, a.qvec, a.rot, pos, v);
            }
#pragma unroll
            for (int e = 0; e < 8; e++) big = fmaxf(big, fabsf(v[e]));
#pragma unroll
            for (int o = W / 2; o > 0; o >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
            // 2^e takes the largest to 2^14 .. 2^15; the ends of fp32 stay in range
            const int e = big > 0.0f && big < __int_as_float(0x7f800000) ? 14 - max(-112, min(126, ((int)(__float_as_uint(big) >> 23) - 127))) : 0;
            const float up = __uint_as_float((uint32_t)(e / 2 + 127) << 23), up2 = __uint_as_float((uint32_t)(e - e / 2 + 127) << 23);
            // what takes a product back to its score: finite, so that a product of 0 is one of 0
            const int back = max(-252, min(127, a.scale_up - e));
            if (word == 0) qscale[r] = a.scale2 * __uint_as_float((uint32_t)(127 + back / 2) << 23) * __uint_as_float((uint32_t)(127 + back - back / 2) << 23);
#pragma unroll
            for (int x = 0; x < 8; x++) v[x] = v[x] * up * up2;
            // the lane and step that take this word: quads' words as K's are read
            const int to_t = DP == 64 ? word >> 1 : (word & 15) >> 2, k = DP == 64 ? word & 1 : (word & 3) + 4 * (word >> 4);
            uint4* q = qf + ((r >> 3) * NP * WK + k) * 32 + (r & 7) * 4 + to_t;
            // values x and x + 4 are a pair, as decoded codes are
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int x = 0; x < 4; x++) {
                hi[x] = pack2<__half>(v[x], v[x + 4]);
                float y, z;
                unpack2<__half>(hi[x], y, z);
                lo[x] = pack2<__half>(v[x] - y, v[x + 4] - z);
            }
            q[0] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            if constexpr (NP == 2) q[WK * 32] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
        __syncthreads();
        uint4 qr[Sh::kQueryRegs ? NT * NP * WK : 1];
        if constexpr (Sh::kQueryRegs) {
#pragma unroll
            for (int i = 0; i < NT * NP * WK; i++) qr[i] = qf[i * 32 + lane];
        }
        // this lane's columns: rows 2 t and 2 t + 1 of every eight
        float fq[NT][2], M[NT][2], L[NT][2];
        int qhi[NT][2], qlo[NT][2];                     // places that they see
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int c = 0; c < 2; c++) {
                const int r = nt * 8 + 2 * t + c;
                const int64_t pos = (int64_t)s.len - s.nq + token_of(a, row0 + r);
                fq[nt][c] = qscale[r];
                M[nt][c] = none;
                L[nt][c] = 0.0f;
                qhi[nt][c] = r < n_rows ? (int)max((int64_t)0, min(pos + 1, (int64_t)s.seen)) : 0;
                qlo[nt][c] = a.window > 0 ? (int)max((int64_t)0, pos - a.window + 1) : 0;
            }
        // stages between these are seen by every row
        const int64_t p0 = (int64_t)s.len - s.nq + token_of(a, row0), p1 = (int64_t)s.len - s.nq + token_of(a, row0 + n_rows - 1);
        const int all_hi = (int)max((int64_t)0, min(p0 + 1, (int64_t)s.seen)), all_lo = a.window > 0 ? (int)max((int64_t)0, p1 - a.window + 1) : 0;

        float o[DP / 16][NT][4];
#pragma unroll
        for (int i = 0; i < DP / 16; i++)
#pragma unroll
            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                for (int c = 0; c < 4; c++) o[i][nt][c] = 0.0f;

        uint32_t use = my_ring;
        for (int i = 0, place = place0; i < stages; i++, place += BLOCK) {
            copies_wait<ST - 2>();
            __syncwarp();                               // every lane's copies of this stage; all have read the one before
            const uint32_t here = there >> (SUB * (ST - 2)) & ((1u << SUB) - 1u), sm = use;
            use = use + BYTES == ring_end ? my_ring : use + BYTES;
            issue();
            if (here == 0u) continue;

            // scores: rows g and g + 8 of each part (the planes' sums apart)
            constexpr int CH = NP == 2 || (NT == 1 && SUB == 1) ? 2 : 1;
            float part[SUB][CH][NT][4];
#pragma unroll
            for (int sub = 0; sub < SUB; sub++) {
#pragma unroll
                for (int h = 0; h < CH; h++)
#pragma unroll
                    for (int nt = 0; nt < NT; nt++)
#pragma unroll
                        for (int c = 0; c < 4; c++) part[sub][h][nt][c] = 0.0f;
                uint32_t k0[WK], k1[WK];
                auto words = [&](uint32_t at, uint32_t (&w)[WK]) {
                    if constexpr (DP == 256) {
                        uint32_t x[4], y[4];
                        lds(at, x);
                        lds(at ^ 64u, y);               // chunk t + 4
#pragma unroll
                        for (int i = 0; i < 4; i++) { w[i] = x[i]; w[(4 + i) % WK] = y[i]; }
                    } else {
                        lds(at, w);
                    }
                };
                words(sm + sub * St::kBytes + k_from, k0);
                words(sm + sub * St::kBytes + k_from + 8 * St::kRow, k1);
#pragma unroll
                for (int k = 0; k < WK; k++) {
                    uint32_t x[4], y[4];
                    decode8<LIN>(k0[k], a.klut, x);
                    decode8<LIN>(k1[k], a.klut, y);
                    // both steps of a word: products that follow one another have other sums
                    uint2 second[NT][NP];
#pragma unroll
                    for (int nt = 0; nt < NT; nt++)
#pragma unroll
                        for (int p = 0; p < NP; p++) {
                            const int at = (nt * NP + p) * WK + k;
                            uint4 q;
                            if constexpr (Sh::kQueryRegs) q = qr[at];
                            else q = qf[at * 32 + lane];
                            mma16(part[sub][NP == 2 ? p : 0][nt], x[0], y[0], x[1], y[1], q.x, q.y);
                            second[nt][p] = make_uint2(q.z, q.w);
                        }
#pragma unroll
                    for (int nt = 0; nt < NT; nt++)
#pragma unroll
                        for (int p = 0; p < NP; p++)
                            mma16(part[sub][NP == 2 ? p : CH - 1][nt], x[2], y[2], x[3], y[3], second[nt][p].x, second[nt][p].y);
                }
            }
            const bool whole = place + kAtPlaces * SUB <= all_hi && place >= all_lo && here == (1u << SUB) - 1u;
            float sc[SUB][NT][4], vs[SUB][2], lv[SUB][2];
            // scores less the maximum
#pragma unroll
            for (int sub = 0; sub < SUB; sub++) {
                const uint32_t scales = sm + sub * St::kBytes + St::kKs + 4 * g;
                const float ks0 = lds_f32(scales), ks1 = lds_f32(scales + 32);
                vs[sub][0] = lds_f32(scales + 64);
                vs[sub][1] = lds_f32(scales + 96);
                // log2 of v's scales, where they have one (2^30 places have a sum below 2^128: 2^(8 + 90) each)
#pragma unroll
                for (int c = 0; c < 2; c++) {
                    lv[sub][c] = fmaxf(fminf(lg2(fabsf(vs[sub][c])), 100.0f), -90.0f);
                    vs[sub][c] *= kWeightUp;
                }
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                    for (int c = 0; c < 2; c++) {
                        float x = part[sub][0][nt][c], y = part[sub][0][nt][2 + c];
                        if constexpr (CH == 2) {
                            x += part[sub][CH - 1][nt][c];
                            y += part[sub][CH - 1][nt][2 + c];
                        }
                        part[sub][0][nt][c] = x * ks0;
                        part[sub][0][nt][2 + c] = y * ks1;
                        sc[sub][nt][c] = fmaf(part[sub][0][nt][c], fq[nt][c], -M[nt][c]);
                        sc[sub][nt][2 + c] = fmaf(part[sub][0][nt][2 + c], fq[nt][c], -M[nt][c]);
                    }
            }
            // what is not seen: -inf (apart from the rest, which whole stages have to
            // themselves)
            uint32_t unseen = 0u;
            if (!whole) {
#pragma unroll
                for (int sub = 0; sub < SUB; sub++)
#pragma unroll
                    for (int nt = 0; nt < NT; nt++)
#pragma unroll
                        for (int c = 0; c < 4; c++) {
                            const int at = place + sub * kAtPlaces + g + 8 * (c >> 1);
                            if (!(here >> (SUB - 1 - sub) & 1u) || at >= qhi[nt][c & 1] || at < qlo[nt][c & 1]) {
                                unseen |= 1u << ((sub * NT + nt) * 4 + c);
                                sc[sub][nt][c] = ninf;
                            }
                        }
            }
            float over = ninf;                          // how far scores (with their values' scales) pass the maximum
#pragma unroll
            for (int sub = 0; sub < SUB; sub++)
#pragma unroll
                for (int row = 0; row < 2; row++) {
                    float m = sc[sub][0][2 * row];
#pragma unroll
                    for (int i = 1; i < 2 * NT; i++) m = fmaxf(m, sc[sub][i >> 1][2 * row + (i & 1)]);
                    over = fmaxf(over, m + lv[sub][row]);
                }
            if (__any_sync(0xffffffffu, over > 8.0f)) {
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                    for (int c = 0; c < 2; c++) {
                        float m = M[nt][c];
#pragma unroll
                        for (int sub = 0; sub < SUB; sub++) {
                            float &x = sc[sub][nt][c], &y = sc[sub][nt][2 + c];
                            x = x == ninf ? ninf : part[sub][0][nt][c] * fq[nt][c];
                            y = y == ninf ? ninf : part[sub][0][nt][2 + c] * fq[nt][c];
                            m = fmaxf(m, fmaxf(x + lv[sub][0], y + lv[sub][1]));
                        }
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
                        const float f = m > M[nt][c] ? ex2(M[nt][c] - m) : 1.0f;
                        M[nt][c] = m;
                        L[nt][c] *= f;
#pragma unroll
                        for (int sub = 0; sub < SUB; sub++) {
                            float &x = sc[sub][nt][c], &y = sc[sub][nt][2 + c];
                            x = x == ninf ? ninf : x - m;
                            y = y == ninf ? ninf : y - m;
                        }
#pragma unroll
                        for (int k = 0; k < DP / 16; k++) {
                            o[k][nt][c] *= f;
                            o[k][nt][2 + c] *= f;
                        }
                    }
            }
            // weights; a scale that is not seen may be NaN
#pragma unroll
            for (int sub = 0; sub < SUB; sub++)
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                    for (int c = 0; c < 4; c++) {
                        const float e = ex2(sc[sub][nt][c]);
                        L[nt][c & 1] += e;
                        sc[sub][nt][c] = e * vs[sub][c >> 1];
                    }
            if (!whole) {
#pragma unroll
                for (int sub = 0; sub < SUB; sub++)
#pragma unroll
                    for (int nt = 0; nt < NT; nt++)
#pragma unroll
                        for (int c = 0; c < 4; c++)
                            if (unseen >> ((sub * NT + nt) * 4 + c) & 1u) sc[sub][nt][c] = 0.0f;
            }
#pragma unroll
            for (int sub = 0; sub < SUB; sub++) {
                // turned into the second product's operand
                uint32_t p0[NT][NP], p1[NT][NP];
#pragma unroll
                for (int nt = 0; nt < NT; nt++) {
                    const float (&w)[4] = sc[sub][nt];
                    const uint32_t h0 = pack2<__half>(w[0], w[1]), h1 = pack2<__half>(w[2], w[3]);
                    p0[nt][0] = transposed(h0);
                    p1[nt][0] = transposed(h1);
                    if constexpr (NP == 2) {
                        float x[4];
                        unpack2<__half>(h0, x[0], x[1]);
                        unpack2<__half>(h1, x[2], x[3]);
#pragma unroll
                        for (int c = 0; c < 4; c++) x[c] = (w[c] - x[c]) * kLowUp;
                        p0[nt][NP - 1] = transposed(pack2<__half>(x[0], x[1]));
                        p1[nt][NP - 1] = transposed(pack2<__half>(x[2], x[3]));
                    }
                }
                // values: this lane's words of places 2 t, 2 t + 1, 2 t + 8, 2 t + 9
                uint32_t v[4][WV];
#pragma unroll
                for (int k = 0; k < 4; k++) lds(sm + sub * St::kBytes + (k & 1 ? v_from1 : v_from0) + 8 * St::kRow * (k >> 1), v[k]);
                // a pair of places' codes of the same four values, the second place's above
                auto pair_codes = [](uint32_t x, uint32_t y, int upper) { return prmt(x, y, upper ? 0x7632u : 0x5410u); };
                if constexpr (WV == 1) {
                    // rows g: values 0..3 of the word, rows g + 8: values 4..7
                    uint32_t x0[4], x1[4], y0[4], y1[4];
                    decode8<LIN>(pair_codes(v[0][0], v[1][0], 0), a.vlut, x0);
                    decode8<LIN>(pair_codes(v[2][0], v[3][0], 0), a.vlut, x1);
                    decode8<LIN>(pair_codes(v[0][0], v[1][0], 1), a.vlut, y0);
                    decode8<LIN>(pair_codes(v[2][0], v[3][0], 1), a.vlut, y1);
#pragma unroll
                    for (int k = 0; k < 4; k++)
#pragma unroll
                        for (int nt = 0; nt < NT; nt++)
                        mma16_add(o[k][nt], x0[k], y0[k], x1[k], y1[k], p0[nt], p1[nt]);
                } else {
                    // rows g: the first word's values, rows g + 8: the second's
#pragma unroll
                    for (int wp = 0; wp < WV / 2; wp++)
#pragma unroll
                        for (int up = 0; up < 2; up++) {
                            uint32_t x0[4], x1[4], y0[4], y1[4];
                            constexpr int LAST = WV - 1;
                            const int second = 2 * wp + 1 < LAST ? 2 * wp + 1 : LAST;
                            decode8<LIN>(pair_codes(v[0][2 * wp], v[1][2 * wp], up), a.vlut, x0);
                            decode8<LIN>(pair_codes(v[2][2 * wp], v[3][2 * wp], up), a.vlut, x1);
                            decode8<LIN>(pair_codes(v[0][second], v[1][second], up), a.vlut, y0);
                            decode8<LIN>(pair_codes(v[2][second], v[3][second], up), a.vlut, y1);
#pragma unroll
                            for (int k = 0; k < 4; k++)
#pragma unroll
                                for (int nt = 0; nt < NT; nt++)
                                mma16_add(o[8 * wp + 4 * up + k][nt], x0[k], y0[k], x1[k], y1[k], p0[nt], p1[nt]);
                        }
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
            float m = none, l = 0.0f, f[kAtWarps], y[8];
#pragma unroll
            for (int w = 0; w < kAtWarps; w++) m = fmaxf(m, sums[w * R + r].x);
#pragma unroll
            for (int k = 0; k < 8; k++) y[k] = 0.0f;
#pragma unroll
            for (int w = 0; w < kAtWarps; w++) {
                const float2 x = sums[w * R + r];
                f[w] = ex2(x.x - m);
                l = fmaf(f[w], x.y, l);
                const float* from = merge + (w * R + r) * DP + d;
#pragma unroll
                for (int k = 0; k < 8; k++) y[k] = fmaf(f[w], from[k], y[k]);
            }
            if (begins && ends) {
                const uint32_t row = row0 + r, token = token_of(a, row);
                const int64_t qh = (int64_t)head * a.group + (row - token * a.group);
                const float inv = l == 0.0f ? 0.0f : __fdiv_rn(a.vunit, l);
#pragma unroll
                for (int k = 0; k < 8; k++) y[k] = l == 0.0f ? 0.0f : (l == l ? y[k] * inv : l);
                store8_any(a.out, a.out_type, (s.row0 + token) * a.ldo + qh * a.D + d, a.D - d, a.ovec, y);
                if (a.lse && d == 0)
                    a.lse[(s.row0 + token) * ((int64_t)a.heads * a.group) + qh] = l == 0.0f ? ninf : m * 0.69314718f + logf(l);
            } else {
                store8<float>(slot + (int64_t)r * DP + d, y);
                if (d == 0) {
                    slot[R * DP + r] = m;
                    slot[R * DP + R + r] = l;
                }
            }
        }
        if (begins && !ends) {
            const int64_t end_block = at_block + tl.blocks - 1, few = (share + 1) * larger;
            const int64_t last = end_block < few ? quotient(end_block, share + 1) : larger + quotient(end_block - few, share);
            goes_on = make_int4((int)last + 1, b, head, tile);
        }
        at_block += blocks;
        left -= blocks;
        rest = 0;
        if (ends) {
            if (++tile >= tiles_of<Sh>(a, s)) {
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
    if (threadIdx.x == 0) a.head[me] = goes_on;
}

// Joins the parts of a tile that begins in part `x` of the work and goes on in
// the following ones.
template <int DP, int R>
__global__ void __launch_bounds__(128) attention_join_kernel(const AttnArgs a)
{
    constexpr int SLOT = R * (DP + 2);
    griddep_wait();
    const int p0 = blockIdx.x;
    const int4 h = a.head[p0];
    if (h.x == 0) return;
    const Seq s = sequence(a, h.y);
    const int r = blockIdx.y;
    const uint32_t row = (uint32_t)h.w * R + r;
    if (row >= (uint32_t)(s.nq * a.group)) return;
    const int n = h.x - p0;             // parts
    auto slot = [&](int i) { return a.partial + (int64_t)(i == 0 ? 2 * p0 + 1 : 2 * (p0 + i)) * SLOT; };
    __shared__ float wm[4];
    const float ninf = __int_as_float(0xff800000);
    float m = __int_as_float(kNone);
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
    const uint32_t token = token_of(a, row);
    const int64_t qh = (int64_t)h.z * a.group + (row - token * a.group);
    const float inv = l == 0.0f ? 0.0f : __fdiv_rn(a.vunit, l);
    const int64_t at = (s.row0 + token) * a.ldo + qh * a.D + d;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        const float v = l == 0.0f ? 0.0f : (l == l ? y[k] * inv : l);
        if (a.out_type == ESB_F32) static_cast<float*>(a.out)[at + k] = v;
        else if (a.out_type == ESB_F16) static_cast<__half*>(a.out)[at + k] = from_f32<__half>(v);
        else static_cast<__nv_bfloat16*>(a.out)[at + k] = from_f32<__nv_bfloat16>(v);
    }
    if (a.lse && d == 0)
        a.lse[(s.row0 + token) * ((int64_t)a.heads * a.group) + qh] = l == 0.0f ? ninf : m * 0.69314718f + logf(l);
}

template <int DP, int NT, int NP, bool LIN>
cudaError_t run_attention(const AttnArgs& in, void* workspace, cudaStream_t st)
{
    using Sh = Shape<DP, NT, NP>;
    AttnArgs a = in;
    const int parts = device_sm_count() * Sh::kSm;
    a.head = static_cast<int4*>(workspace);
    a.partial = reinterpret_cast<float*>(a.head + parts);
    // once for a device
    static std::atomic<unsigned long long> configured{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const unsigned long long bit = dev < 64 ? 1ull << dev : 0ull;
    if (!(configured.load(std::memory_order_relaxed) & bit)) {
        e = cudaFuncSetAttribute(attention_kernel<DP, NT, NP, LIN>, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::kBytes);
        if (e != cudaSuccess) return e;
        configured.fetch_or(bit, std::memory_order_relaxed);
    }
    e = launch_pdl(attention_kernel<DP, NT, NP, LIN>, dim3((unsigned)parts), dim3(kAtThreads), Sh::kBytes, st, a);
    if (e != cudaSuccess) return e;
    return launch_pdl(attention_join_kernel<DP, Sh::R>, dim3((unsigned)parts, (unsigned)(a.starts ? Sh::R : std::min(a.group, Sh::R))), dim3(128), 0, st, a);
}
template <int DP, int NT, int NP> size_t workspace_of()
{
    using Sh = Shape<DP, NT, NP>;
    return (size_t)(device_sm_count() * Sh::kSm) * (sizeof(int4) + 2 * sizeof(float) * Sh::kSlot);
}

// One of a head size's shapes: NT eights of rows, NP planes of queries and weights.
template <int DP, int NT, int NP> struct Variant {
    static cudaError_t run(const AttnArgs& a, bool lin, void* workspace, cudaStream_t st)
    {
        return lin ? run_attention<DP, NT, NP, true>(a, workspace, st) : run_attention<DP, NT, NP, false>(a, workspace, st);
    }
    static size_t bytes() { return workspace_of<DP, NT, NP>(); }
};

}  // namespace

// What each head size's translation unit has: the most eights of rows for a
// number of planes, a launch, and the bytes of its workspace.
#define ESB_ATTENTION_SHAPES(X) X(64) X(128) X(256)
#define ESB_DECLARE(DP)                                                                                              \
    int attention_most_##DP(int planes);                                                                             \
    cudaError_t attention_run_##DP(const AttnArgs& a, int nt, int planes, bool lin, void* workspace, cudaStream_t st); \
    size_t attention_bytes_##DP(int nt, int planes);
ESB_ATTENTION_SHAPES(ESB_DECLARE)
#undef ESB_DECLARE

}  // namespace esb
