// The tiles of the rows of all experts.  Nothing here but wave functions, so
// that a program on the host can run it with its own (Args: offsets, rows and
// experts, as the experts' products have them).
#pragma once

#include <stdint.h>

namespace agn {
namespace {

template <class Args>
__device__ __forceinline__ int clamped_offset(const Args& g, int e) {
  return min(max(g.offsets[e], 0), g.rows);
}

// The tiles of TR rows of all experts, counted expert by expert.  Every lane
// holds up to 64 experts' part of the count (one load of the offsets where
// there are no more; the functions are called with every lane active and
// give every lane the same).
struct RowTile {
  int e, r0, rend;   // expert (-1: no such tile), first row, the expert's end
  int of, of_expert;  // the tile's number among its expert's, and how many those are
};
struct RowTiles {
  int TR;                // rows a tile
  int first, end, upto;  // this lane's expert's rows; tiles up to and with it (of the 64 at e0)
  int e0, base;          // the loaded experts' first; tiles before it
  int total;             // tiles of all experts

  template <class Args>
  __device__ void load(const Args& g, int at) {
    const int lane = threadIdx.x & 63, e = at + lane;
    first = end = 0;
    if (e < g.experts) {
      first = clamped_offset(g, e);
      end = max(first, clamped_offset(g, e + 1));
    }
    upto = (end - first + TR - 1) / TR;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(upto, d);
      if (lane >= d) upto += o;
    }
    e0 = at;
  }
  template <class Args>
  __device__ void init(const Args& g, int rows_a_tile) {
    TR = rows_a_tile;
    total = 0;
    for (int at = 0; at < g.experts; at += 64) {
      base = total;
      load(g, at);
      total += __builtin_amdgcn_readlane(upto, 63);
    }
  }
  template <class Args>
  __device__ RowTile find(const Args& g, int tile) {
    if (g.experts > 64) {
      // (past the last tile the search would end with the last group's counts, added once more)
      if (tile >= total) return {-1, 0, 0, 0, 0};
      base = 0;
      for (int at = 0; at < g.experts; at += 64) {
        load(g, at);
        const int n = __builtin_amdgcn_readlane(upto, 63);
        if (tile < base + n) break;
        base += n;
      }
    }
    const uint64_t hit = __ballot(tile < base + upto);
    if (!hit) return {-1, 0, 0, 0, 0};
    const int l = __builtin_ctzll(hit);
    const int b = __builtin_amdgcn_readlane(first, l), en = __builtin_amdgcn_readlane(end, l);
    const int n = (en - b + TR - 1) / TR, of = tile - base - __builtin_amdgcn_readlane(upto, l) + n;
    return {e0 + l, b + of * TR, en, of, n};
  }
};

}  // namespace
}  // namespace agn
