// The experts' products: arguments, and what every tile shape shares.
#pragma once

#include "block_common.h"
#include "block_experts_rules.h"
#include "block_row_tiles.h"

namespace agn {

// One of the three products over all experts (all sizes below 2^31):
//   FWD: out[r][n] = epilogue(sum_k a[r][k] b_e[n][k])    a = x,  b = w
//   DX:  out[r][n] = epilogue(sum_k a[r][k] b_e[k][n])    a = dy, b = w
//   DW:  out_e[m][n] = sum_r a[r][m] b[r][n]              a = dy, b = x
struct ProductArgs : ProductSizes {
  const void *a, *b;
  int64_t lda, ldb, bstride;  // bstride: from one expert's b to the next (FWD, DX)
  bool a_pad, b_pad;          // rows go on with zeros to a multiple of eight
  const int32_t* offsets;
  void* out;
  int64_t ldo;
  const float* bias;  // FWD: or null
  int relu;
  MaskArgs mask;
  const void* gate;  // DX: x, whose positive elements let the gradient through, or null
  int64_t ldgate;
  float gate_scale;
  float* dbias;  // DW: or null
  // DW: rows a part (0: no parts), and the parts' sums (see weight_tile_of)
  int part_rows, parts_most;
  float *parts, *parts_bias;
};

// operands whose every chunk of eight is a 16-byte aligned piece of one row
inline bool direct_ok(int prod, const ProductArgs& g) {
  if ((((uintptr_t)g.a | (uintptr_t)g.b) & 15) || g.lda % 8 || g.ldb % 8 || g.bstride % 8) return false;
  return whole_chunks(prod, g, g.a_pad, g.b_pad);
}

// (k: as product_kernel chose for this product)
hipError_t launch_product_bf16(int prod, const ProductKernel& k, const ProductArgs& g, hipStream_t s);
hipError_t launch_product_f32(int prod, const ProductKernel& k, const ProductArgs& g, hipStream_t s);
hipError_t launch_product_few(const ProductKernel& k, int dtype, const ProductArgs& g, hipStream_t s);

constexpr int kTailBlocks = 64;  // workgroups that clear the output rows of no expert

namespace {

// The rows, tile and output of workgroup `pid` of the weight gradients, whose
// tiles are `per` an expert.
//
// Without parts (g.part_rows 0) a tile sums all rows of its expert; experts
// with more rows come first, so that the longest tiles are not the last to
// start, and each XCD takes one contiguous share of every expert's tiles,
// since experts differ in rows.
//
// With parts, where the tiles alone would not fill the chip, a tile sums one
// part of at most part_rows rows.  The sums of an expert of several parts go
// to the workspace, to be added in order by sum_weight_parts.
struct WeightTile {
  int e, r0, rows;  // (e < 0: nothing to do)
  int t;            // of `per`
  float *out, *dbias;
};
__device__ __forceinline__ WeightTile weight_tile_of(const ProductArgs& g, int pid, int per) {
  const int64_t size = (int64_t)g.M * g.N;
  if (g.part_rows) {
    RowTiles parts;
    parts.init(g, g.part_rows);
    // (more parts than the workspace holds: offsets that do not rise)
    if (parts.total > g.parts_most || pid >= parts.total * per) return {-1, 0, 0, 0, nullptr, nullptr};
    const int logical = xcd_remap(pid, parts.total * per), q = logical / per;
    const RowTile p = parts.find(g, q);
    if (p.e < 0) return {-1, 0, 0, 0, nullptr, nullptr};
    const bool whole = p.of_expert == 1;
    float* dbias = !g.dbias ? nullptr : whole ? g.dbias + (int64_t)p.e * g.M : g.parts_bias + (int64_t)q * g.M;
    return {p.e, p.r0, min(g.part_rows, p.rend - p.r0), logical % per,
            whole ? (float*)g.out + p.e * size : g.parts + q * size, dbias};
  }
  int e = pid / per;
  if (g.experts <= 64) {
    const int lane = threadIdx.x & 63;
    const int n = lane < g.experts ? clamped_offset(g, lane + 1) - clamped_offset(g, lane) : -1;
    int rank = 0;
    for (int o = 0; o < g.experts; ++o) {
      const int no = __builtin_amdgcn_readlane(n, o);
      rank += no > n || (no == n && o < lane) ? 1 : 0;
    }
    e = __builtin_ctzll(__ballot(lane < g.experts && rank == e));
  }
  const int b = clamped_offset(g, e);
  return {e, b, max(0, clamped_offset(g, e + 1) - b), xcd_remap(pid % per, per), (float*)g.out + e * size,
          g.dbias ? g.dbias + (int64_t)e * g.M : nullptr};
}

// output rows of no expert become zero; workgroup b of kTailBlocks
template <class T, int THREADS>
__device__ __forceinline__ void clear_rows(const ProductArgs& g, int b) {
  T* out = (T*)g.out;
  for (int r = clamped_offset(g, g.experts) + b; r < g.rows; r += kTailBlocks)
    for (int c = threadIdx.x * 8; c < g.N; c += THREADS * 8) store8_row(out + (int64_t)r * g.ldo, c, g.N, zero8(out));
}

// eight columns c .. c+7 of output row r of expert e from their sums: bias,
// activation and mask (FWD), or the gate (DX)
// (bias: of the eight columns, zeros for none; gate: x's eight elements)
template <int PROD, class T>
__device__ __forceinline__ void finish8(const ProductArgs& g, uint32_t step, int r, int c, const float (&bias)[8],
                                        const Raw8<T>& gate, float (&v)[8]) {
  if (PROD == PROD_FWD) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += bias[j];
    if (g.relu)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = v[j] > 0.f ? v[j] : (v[j] != v[j] ? v[j] : 0.f);  // (a NaN stays one)
    if (g.mask.thr) mask_apply(g.mask, step, r, (uint32_t)(c >> 3), v);
  }
  if (PROD == PROD_DX && g.gate) {
    float x[8];
    widen(gate, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = x[j] > 0.f ? v[j] * g.gate_scale : 0.f;
  }
}

__device__ __forceinline__ void load_bias(const ProductArgs& g, int e, int c, float (&b)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) b[j] = 0.f;
  if (g.bias && c < g.N) widen(load8_row(g.bias + (int64_t)e * g.N, c, g.N), b);
}
template <class T>
__device__ __forceinline__ Raw8<T> load_gate(const ProductArgs& g, int r, int c) {
  const T* x = (const T*)g.gate;
  return g.gate && c < g.N ? load8_row(x + (int64_t)r * g.ldgate, c, g.N) : zero8(x);
}

inline int64_t weight_parts_most(const ProductArgs& g) {
  return g.part_rows ? g.rows / g.part_rows + g.experts : g.experts;
}

}  // namespace
}  // namespace agn
