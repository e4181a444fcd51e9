// esb_attention_plan.h -- arithmetic of esb_cache_attention that needs no CUDA:
// the places that a tile's queries see, and those that a warp goes through.
#pragma once

#include <cstdint>

#ifndef ESB_HOST_DEVICE
#ifdef __CUDACC__
#define ESB_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define ESB_HOST_DEVICE inline
#endif
#endif

namespace esb {

struct Tile {
    int lo, hi, blocks;                 // places lo .. hi - 1, lo at a stage's start; blocks of work (one where there are none)
};

// Queries with places p0 .. p1 of a sequence whose page table holds its first
// `seen` places (2^30 at most); a stage is a power of two, a block some stages.
// Lengths may be far past the table: there lo ends with what is held, so that no
// later sum passes 32 bits.
ESB_HOST_DEVICE Tile tile_places(int64_t p0, int64_t p1, int seen, int window, int stage, int block)
{
    Tile t;
    const int64_t hi = p1 + 1 < seen ? p1 + 1 : seen, lo = window > 0 ? p0 - window + 1 : 0;
    t.hi = hi > 0 ? (int)hi : 0;
    t.lo = lo <= 0 ? 0 : (int)(lo < t.hi ? lo : t.hi) & ~(stage - 1);
    t.blocks = t.hi > t.lo ? (t.hi - t.lo + block - 1) / block : 1;
    return t;
}

// Of `blocks` of a tile's blocks from `first` on: where a warp's stages begin (they
// are a block apart), and the end of them all.
ESB_HOST_DEVICE int first_place(const Tile& t, int first, int warp, int warps, int stage) { return t.lo + (first * warps + warp) * stage; }
ESB_HOST_DEVICE int end_place(const Tile& t, int first, int blocks, int block)
{
    const int end = t.lo + (first + blocks) * block;
    return end < t.hi ? end : t.hi;
}

// Sequences (at least one) that each of a block's threads counts, in a run.
ESB_HOST_DEVICE int run_of(int seqs, int threads) { return (seqs - 1) / threads + 1; }

}  // namespace esb
