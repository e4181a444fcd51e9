// esb_heads.cuh -- heads of tokens held as the rotation pairs their values, and
// how a kernel goes through them; shared by esb_headnorm.cu and esb_cache.cu.
#pragma once

#include <algorithm>
#include <cstdint>
#include <cuda_runtime.h>

#include "esb_rotate.cuh"
#include "esb_rows.cuh"

namespace esb {

// The pairs that a lane holds: (first, first + i) of `count`.
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
};

// A lane's 16 values as they lie in memory.
template <class T, bool VEC>
struct RawPairs {
    Raw8<T> u, w;
    __device__ __forceinline__ void load(const T* x, const PairPlace& p, const RotArgs& r, bool on)
    {
        if constexpr (VEC) {
            const bool in = on && p.count > 0;
            const int at = p.rows ? 2 * p.j0 : p.j0;
            u.load(x + at, in ? 8 : 0, true);
            w.load(x + (p.rows ? at + 8 : at + p.half), in ? 8 : 0, true);
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
        float x[8], y[8];
        u.values(x);
        w.values(y);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const bool rows = VEC && p.rows;
            a[i] = rows ? (i < 4 ? x[(2 * i) & 7] : y[(2 * i) & 7]) : x[i];
            b[i] = rows ? (i < 4 ? x[(2 * i + 1) & 7] : y[(2 * i + 1) & 7]) : y[i];
        }
    }
};

template <class T, bool VEC>
__device__ __forceinline__ void store_pairs(T* y, const PairPlace& p, const RotArgs& r, const float (&a)[8], const float (&b)[8])
{
    if constexpr (VEC) {
        if (p.count <= 0) return;
        float u[8], w[8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            u[i] = p.rows ? ((i & 1) ? b[i / 2] : a[i / 2]) : a[i];
            w[i] = p.rows ? ((i & 1) ? b[4 + i / 2] : a[4 + i / 2]) : b[i];
        }
        const int at = p.rows ? 2 * p.j0 : p.j0;
        store8<T>(y + at, u);
        store8<T>(y + (p.rows ? at + 8 : at + p.half), w);
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

// Where a lane's group stands: item, head in it, and what that is.  All items of
// the first part come before those of the second, so a warp changes what it
// keeps of a part (weights, sums) once.  WARPS: of a block.
template <int L, int WARPS>
struct HeadWalk {
    int64_t item, token;
    int it, part, head;
    bool on;
    __device__ __forceinline__ void start(const HeadWork& a)
    {
        item = (int64_t)blockIdx.x * WARPS + (threadIdx.x >> 5);
        it = 0;
        place(a);
    }
    __device__ __forceinline__ void place(const HeadWork& a)
    {
        const int group = (threadIdx.x & 31) / L;
        part = item >= a.part[0].items;
        const HeadSplit& s = a.part[part];
        const int64_t i = part ? item - a.part[0].items : item, row = i / s.chunks;
        const int side = s.side;
        token = row * (32 / L / side) + group / side;
        head = ((int)(i - row * s.chunks) * s.iter + it) * side + group % side;
        on = item < a.part[0].items + a.part[1].items && token < a.tokens && head < a.part[part].heads;
    }
    // the next head of the item, or the next item
    __device__ __forceinline__ void next(const HeadWork& a)
    {
        if (++it < a.part[part].iter) {
            head += a.part[part].side;
            on = on && head < a.part[part].heads;
            return;
        }
        it = 0;
        item += (int64_t)gridDim.x * WARPS;
        place(a);
    }
    __device__ __forceinline__ bool more(const HeadWork& a) const { return item < a.part[0].items + a.part[1].items; }
};

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

// A lane's values are two vectors: whole eights of pairs on both sides of the rotation's end.
inline bool pairs_of_vectors(int D, int rot_dim, bool interleaved) { return D % 16 == 0 && (interleaved || rot_dim % 16 == 0); }

inline bool rows16(const void* p, int64_t ld, int type)
{
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld * type_bytes(type) % 16 == 0;
}

}  // namespace esb
