// esb_heads.cuh -- heads of tokens held as the rotation pairs their values, and
// how a kernel goes through them; shared by esb_headnorm.cu and esb_cache.cu.
#pragma once

#include <algorithm>
#include <cstdint>
#include <cuda_runtime.h>

#include "esb_rotate.cuh"
#include "esb_rows.cuh"

namespace esb {

// How a lane's 8 pairs lie in memory: two vectors half a rotation apart, 16
// values in a row (neighbouring pairs, or none), either by the lane (a part of
// the head is not rotated), or no vectors at all.
enum { kPairHalves, kPairRows, kPairMixed, kPairAny };

// The pairs that a lane holds: (first, second) of `count` from pair j0 on.
struct PairPlace {
    int j0, count;
    bool rows;                          // neighbours in memory: 16 values in a row
    int half;
    __device__ __forceinline__ PairPlace(int j, int pairs, const RotArgs& r)
    {
        j0 = j;
        count = min(8, max(0, pairs - j));
        half = r.dim >> 1;
        rows = r.inter || j0 >= half;
    }
    __device__ __forceinline__ int first(int i, const RotArgs& r) const { return r.inter || j0 + i >= half ? 2 * (j0 + i) : j0 + i; }
    __device__ __forceinline__ int second(int i, const RotArgs& r) const { return r.inter || j0 + i >= half ? 2 * (j0 + i) + 1 : j0 + i + half; }
    // the lane's two vectors
    template <int MODE> __device__ __forceinline__ bool in_rows() const { return MODE == kPairRows || (MODE == kPairMixed && rows); }
    template <int MODE> __device__ __forceinline__ int vec0() const { return in_rows<MODE>() ? 2 * j0 : j0; }
    template <int MODE> __device__ __forceinline__ int vec1() const { return in_rows<MODE>() ? 2 * j0 + 8 : j0 + half; }
};

// 16 values in a row to 8 pairs, and back.
__device__ __forceinline__ void rows_to_pairs(const float (&x)[8], const float (&y)[8], float (&a)[8], float (&b)[8])
{
#pragma unroll
    for (int i = 0; i < 8; i++) {
        a[i] = i < 4 ? x[(2 * i) & 7] : y[(2 * i) & 7];
        b[i] = i < 4 ? x[(2 * i + 1) & 7] : y[(2 * i + 1) & 7];
    }
}
__device__ __forceinline__ void pairs_to_rows(const float (&a)[8], const float (&b)[8], float (&x)[8], float (&y)[8])
{
#pragma unroll
    for (int i = 0; i < 8; i++) {
        x[i] = (i & 1) ? b[i / 2] : a[i / 2];
        y[i] = (i & 1) ? b[4 + i / 2] : a[4 + i / 2];
    }
}

// A lane's 16 values as they lie in memory.
template <class T, int MODE>
struct RawPairs {
    Raw8<T> u, w;
    // x: the head's first value
    __device__ __forceinline__ void load(const T* x, const PairPlace& p, const RotArgs& r, bool on)
    {
        if constexpr (MODE != kPairAny) {
            const bool in = on && p.count > 0;
            u.load(x + p.vec0<MODE>(), in ? 8 : 0, true);
            w.load(x + p.vec1<MODE>(), in ? 8 : 0, true);
        } else {
            uint32_t a[8], b[8];
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const bool in = on && i < p.count;
                if constexpr (sizeof(T) == 4) {
                    a[i] = in ? __float_as_uint(x[p.first(i, r)]) : 0u;
                    b[i] = in ? __float_as_uint(x[p.second(i, r)]) : 0u;
                } else {
                    const uint16_t* h = reinterpret_cast<const uint16_t*>(x);
                    a[i] = in ? h[p.first(i, r)] : 0u;
                    b[i] = in ? h[p.second(i, r)] : 0u;
                }
            }
#pragma unroll
            for (int i = 0; i < (int)(2 * sizeof(T)); i++) {
                u.w[i] = sizeof(T) == 4 ? a[i] : a[(2 * i) & 7] | (a[(2 * i + 1) & 7] << 16);
                w.w[i] = sizeof(T) == 4 ? b[i] : b[(2 * i) & 7] | (b[(2 * i + 1) & 7] << 16);
            }
        }
    }
    __device__ __forceinline__ void values(const PairPlace& p, float (&a)[8], float (&b)[8]) const
    {
        u.values(a);
        w.values(b);
        if (p.in_rows<MODE>()) {
            float x[8], y[8];
#pragma unroll
            for (int i = 0; i < 8; i++) { x[i] = a[i]; y[i] = b[i]; }
            rows_to_pairs(x, y, a, b);
        }
    }
};

template <class T, int MODE>
__device__ __forceinline__ void store_pairs(T* y, const PairPlace& p, const RotArgs& r, const float (&a)[8], const float (&b)[8])
{
    if constexpr (MODE != kPairAny) {
        if (p.count <= 0) return;
        if (p.in_rows<MODE>()) {
            float u[8], w[8];
            pairs_to_rows(a, b, u, w);
            store8<T>(y + 2 * p.j0, u);
            store8<T>(y + 2 * p.j0 + 8, w);
        } else {
            store8<T>(y + p.j0, a);
            store8<T>(y + p.j0 + p.half, b);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (i < p.count) {
                y[p.first(i, r)] = from_f32<T>(a[i]);
                y[p.second(i, r)] = from_f32<T>(b[i]);
            }
    }
}

// cos and sin of a lane's pairs; pairs past the rotated ones are left as they are.
__device__ __forceinline__ void load_turn(const RotArgs& r, bool vec, const PairPlace& p, int64_t pos, float (&c)[8], float (&s)[8])
{
    if (vec && p.j0 + 8 <= p.half) {
        const bool in = pos >= 0 && pos < r.positions;
        const float* t = r.table + (in ? pos : 0) * r.ld + p.j0;
        const float4 c0 = __ldg(reinterpret_cast<const float4*>(t)), c1 = __ldg(reinterpret_cast<const float4*>(t + 4));
        const float4 s0 = __ldg(reinterpret_cast<const float4*>(t + p.half)), s1 = __ldg(reinterpret_cast<const float4*>(t + p.half + 4));
        c[0] = c0.x; c[1] = c0.y; c[2] = c0.z; c[3] = c0.w; c[4] = c1.x; c[5] = c1.y; c[6] = c1.z; c[7] = c1.w;
        s[0] = s0.x; s[1] = s0.y; s[2] = s0.z; s[3] = s0.w; s[4] = s1.x; s[5] = s1.y; s[6] = s1.z; s[7] = s1.w;
        if (!in) {
#pragma unroll
            for (int i = 0; i < 8; i++) c[i] = s[i] = __int_as_float(0x7fffffff);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; i++) {
        c[i] = 1.0f;
        s[i] = 0.0f;
        if (i < p.count && p.j0 + i < p.half) rot_at(r, pos, p.j0 + i, c[i], s[i]);
    }
}

// A warp's work: groups of lanes take a token's heads side by side, and several
// tokens where it has few heads.
struct HeadSplit {
    int side;                           // heads side by side, a power of two
    int iter, chunks;                   // heads of a group, one after the other, in an item; items of a token
    int heads;
    int64_t items;
};
struct HeadWork {
    HeadSplit part[2];
    int64_t tokens;
};

// A warp's way through a part's items: where its lanes' group stands, one head
// after the other.  The grid's warps take the items of both parts in turn, as
// one row of them.
template <int L, int WARPS>
struct HeadWalk {
    uint32_t row, rows, drow, token, tokens;    // there are fewer than 2^31 tokens
    int chunk, dchunk, chunks, side, iter, heads, it, head;
    bool on;                            // there is a head here for this group
    __device__ __forceinline__ HeadWalk(const HeadWork& w, int k)
    {
        const HeadSplit& s = w.part[k];
        const int64_t warp = (int64_t)blockIdx.x * WARPS + (threadIdx.x >> 5), warps = (int64_t)gridDim.x * WARPS;
        int64_t first = warp;
        if (k) {
            const int64_t before = w.part[0].items % warps;
            first = warp >= before ? warp - before : warp + warps - before;
        }
        chunks = s.chunks; side = s.side; iter = s.iter; heads = s.heads; tokens = (uint32_t)w.tokens;
        rows = (uint32_t)(s.items / chunks);
        row = (uint32_t)(first / chunks);
        chunk = (int)(first - (int64_t)row * chunks);
        drow = (uint32_t)(warps / chunks);
        dchunk = (int)(warps - (int64_t)drow * chunks);
        it = 0;
        place();
    }
    __device__ __forceinline__ void place()
    {
        const int group = (threadIdx.x & 31) / L;
        token = row * (32 / L / side) + group / side;
        head = chunk * iter * side + group % side;
        on = row < rows && token < tokens && head < heads;
    }
    __device__ __forceinline__ bool more() const { return row < rows; }
    __device__ __forceinline__ void next()
    {
        if (++it < iter) {
            head += side;
            on = on && head < heads;
            return;
        }
        it = 0;
        row += drow;
        chunk += dchunk;
        if (chunk >= chunks) { chunk -= chunks; row++; }
        place();
    }
};
// A place on it.
struct HeadAt {
    uint32_t token;
    int head;
    bool on, first, more;               // first: of an item
    int64_t pos, slot;                  // of its token (in the first head of an item)
    HeadAt() = default;
    template <class W>
    __device__ __forceinline__ explicit HeadAt(const W& w) : token(w.token), head(w.head), on(w.on), first(w.it == 0), more(w.more()), pos(0), slot(-1) {}
};

// 1 / sqrt(x): the hardware's, and one step that leaves two units in the last place.
__device__ __forceinline__ float rsqrt_of(float x)
{
    float r;
    asm("rsqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return x > 0.0f && x < __int_as_float(0x7f800000) ? fmaf(0.5f * r, fmaf(-x * r, r, 1.0f), r) : r;
}

// Pairs (a, b) turned: (a c - b s, b c + a s), two at a time; back: the other way.
template <bool BACK>
__device__ __forceinline__ void turn_pairs(float (&a)[8], float (&b)[8], const float (&c)[8], const float (&s)[8])
{
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const Pair x = pair_of(a[i], a[i + 1]), y = pair_of(b[i], b[i + 1]), cc = pair_of(c[i], c[i + 1]);
        const Pair sp = pair_of(s[i], s[i + 1]), sm = pair_of(-s[i], -s[i + 1]);
        split(fma2(x, cc, mul2(y, BACK ? sp : sm)), a[i], a[i + 1]);
        split(fma2(y, cc, mul2(x, BACK ? sm : sp)), b[i], b[i + 1]);
    }
}

// Heads side by side and one after the other.  An item costs its heads and some
// half of one for its token's cos and sin; the grid's last round should be full.
inline HeadWork split_heads(int64_t tokens, int heads0, int heads1, int L, int64_t warps)
{
    HeadWork a;
    a.tokens = tokens;
    for (int k = 0; k < 2; k++) {
        HeadSplit& s = a.part[k];
        const int heads = k ? heads1 : heads0;
        s = {1, 1, 1, heads, 0};
        if (heads == 0) continue;
        while (s.side < 32 / L && s.side < heads) s.side *= 2;
        const int full = (heads + s.side - 1) / s.side, together = 32 / L / s.side;
        const int64_t rows = (a.tokens + together - 1) / together;
        double best = 0.0;
        for (int chunks = 1; chunks <= std::min(full, 64); chunks++) {
            const int iter = (full + chunks - 1) / chunks;
            const double cost = (double)((rows * chunks + warps - 1) / warps) * (iter + 0.5);
            if (chunks > 1 && cost >= best) continue;
            best = cost;
            s.iter = iter;
            s.chunks = (full + iter - 1) / iter;
        }
        s.items = rows * s.chunks;
    }
    return a;
}

inline int lanes_of(int D) { return D <= 64 ? 4 : D <= 128 ? 8 : 16; }

// How lanes hold pairs: by vectors where there are whole eights of pairs on both
// sides of the rotation's end.
inline int pair_mode(int D, int rot_dim, bool interleaved, bool vectors)
{
    if (!vectors || D % 16 != 0 || (!interleaved && rot_dim % 16 != 0)) return kPairAny;
    return interleaved || rot_dim == 0 ? kPairRows : rot_dim == D ? kPairHalves : kPairMixed;
}

// Whole eights of a table's cosines and sines are vectors.
inline bool table_vectors(const RotArgs& r) { return r.dim % 8 == 0 && r.ld % 4 == 0 && (reinterpret_cast<uintptr_t>(r.table) & 15u) == 0; }

inline bool rows16(const void* p, int64_t ld, int type)
{
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld * type_bytes(type) % 16 == 0;
}

}  // namespace esb
