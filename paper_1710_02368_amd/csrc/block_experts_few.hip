// The experts' forward product for few rows an expert, where the weights'
// bytes are the work: a workgroup takes 16 RB rows of one expert and 16 CB
// columns, its eight waves share K in pieces of 64 (32 in float32), and their
// sums are added in order through LDS.  Operands go from memory straight into
// MFMA fragments (v_mfma_f32_16x16x32_bf16, v_mfma_f32_16x16x4_f32), with 4
// pieces of both in flight; any alignment will do.
//
// The order of k within a sum is free, so that lane group g = lane / 16 takes
// k 16g .. 16g+15 of a piece (8g .. 8g+7 in float32): its loads are adjacent
// and a row's four groups read one 128-byte line.
#include "block_experts.h"

namespace agn {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int NT = 512, NW = 8;

template <class T>
struct Piece;  // what a lane holds of one row in one piece of K
template <>
struct Piece<uint16_t> {
  static constexpr int K = 64, G = 16;  // k a piece, k a lane group
  Raw8<uint16_t> v[2];
};
template <>
struct Piece<float> {
  static constexpr int K = 32, G = 8;
  Raw8<float> v[1];
};

template <class T>
__device__ __forceinline__ void load(Piece<T>& p, const T* row, int k, int K) {
#pragma unroll
  for (int i = 0; i < Piece<T>::G / 8; ++i) p.v[i] = k + 8 * i < K ? load8_row(row, k + 8 * i, K) : zero8(row);
}
__device__ __forceinline__ f32x4 mfma(const Piece<uint16_t>& a, const Piece<uint16_t>& b, f32x4 c) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.v[i].a), __builtin_bit_cast(bf16x8, b.v[i].a),
                                                c, 0, 0, 0);
  return c;
}
__device__ __forceinline__ f32x4 mfma(const Piece<float>& a, const Piece<float>& b, f32x4 c) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float((i < 4 ? a.v[0].a : a.v[0].b)[i & 3]),
                                             __uint_as_float((i < 4 ? b.v[0].a : b.v[0].b)[i & 3]), c, 0, 0, 0);
  return c;
}

template <class T, int RB, int CB>
__global__ __launch_bounds__(NT) void product_few_kernel(ProductArgs g, int tiles_most) {
  constexpr int PK = Piece<T>::K, RT = 16 * RB, CT = 16 * CB, UN = 4;
  __shared__ float part[NW][RT][CT + 1];
  const int tn = (g.N + CT - 1) / CT;
  if ((int)blockIdx.x >= tiles_most * tn) return clear_rows<T, NT>(g, blockIdx.x - tiles_most * tn);
  RowTiles tiles;
  tiles.init(g, RT);
  // (adjacent columns on adjacent workgroups: all XCDs share an expert's weights)
  const RowTile t = tiles.find(g, blockIdx.x / tn);
  if (t.e < 0) return;
  const int n0 = (blockIdx.x % tn) * CT;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, li = lane & 15, lg = lane >> 4;
  const T *pw[CB], *px[RB];
  int kx[RB];  // (rows past the expert's last are not loaded)
#pragma unroll
  for (int i = 0; i < CB; ++i) pw[i] = (const T*)g.b + t.e * g.bstride + min(n0 + 16 * i + li, g.N - 1) * g.ldb;
#pragma unroll
  for (int i = 0; i < RB; ++i) {
    px[i] = (const T*)g.a + min(t.r0 + 16 * i + li, t.rend - 1) * g.lda;
    kx[i] = t.r0 + 16 * i + li < t.rend ? g.K : 0;
  }
  f32x4 acc[RB][CB];
#pragma unroll
  for (int r = 0; r < RB; ++r)
#pragma unroll
    for (int c = 0; c < CB; ++c) acc[r][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int np = (g.K + PK - 1) / PK;
  for (int p0 = wave; p0 < np; p0 += NW * UN) {
    Piece<T> w[UN][CB], x[UN][RB];
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int k = (p0 + NW * u) * PK + lg * Piece<T>::G;
#pragma unroll
      for (int i = 0; i < CB; ++i) load(w[u][i], pw[i], k, g.K);
#pragma unroll
      for (int i = 0; i < RB; ++i) load(x[u][i], px[i], k, kx[i]);
    }
#pragma unroll
    for (int u = 0; u < UN; ++u)
#pragma unroll
      for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int c = 0; c < CB; ++c) acc[r][c] = mfma(x[u][r], w[u][c], acc[r][c]);
  }
  // lane (li, lg) holds rows 4 lg + q, column li of a block
#pragma unroll
  for (int r = 0; r < RB; ++r)
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int q = 0; q < 4; ++q) part[wave][16 * r + 4 * lg + q][16 * c + li] = acc[r][c][q];
  __syncthreads();
  const int rl = threadIdx.x / (CT / 8), cl = 8 * (threadIdx.x % (CT / 8)), row = t.r0 + rl, c = n0 + cl;
  if (rl >= RT || row >= t.rend || c >= g.N) return;
  float bias[8], v[8];
  load_bias(g, t.e, c, bias);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    v[j] = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) v[j] += part[w][rl][cl + j];
  }
  finish8<PROD_FWD, T>(g, mask_step(g.mask), row, c, bias, zero8((const T*)nullptr), v);
  Raw8<T> o;
  narrow(v, o);
  store8_row((T*)g.out + (int64_t)row * g.ldo, c, g.N, o);
}

template <class T, int RB, int CB>
void launch(const ProductArgs& g, hipStream_t s) {
  static_assert(16 * RB * 2 * CB <= NT, "a thread a chunk of outputs");
  const int most = row_tiles_most(g, 16 * RB), tn = (g.N + 16 * CB - 1) / (16 * CB);
  hipLaunchKernelGGL((product_few_kernel<T, RB, CB>), dim3(most * tn + kTailBlocks), dim3(NT), 0, s, g, most);
}

}  // namespace

hipError_t launch_product_few(const ProductKernel& k, int dtype, const ProductArgs& g, hipStream_t s) {
  if (dtype == AGN_BF16) k.tm == 16 ? launch<uint16_t, 1, 1>(g, s) : launch<uint16_t, 2, 2>(g, s);
  else k.tm == 16 ? launch<float, 1, 1>(g, s) : launch<float, 2, 2>(g, s);
  return hipGetLastError();
}

}  // namespace agn
