// Rows to their experts' places and back (agn_dispatch, agn_combine,
// agn_combine_backward).
#include <algorithm>

#include "block_common.h"

namespace agn {
namespace {

struct Tokens {
  int64_t rows;
  int cols, k;
  uint32_t pairs;  // rows * k
  const int32_t* slot;
  const int32_t* total;
  const float* weights;
  void* x;
  int64_t ldx;
  void* y;
  int64_t ldy;
  void* dy;
  int64_t lddy;
  float* dweights;
};

constexpr int kZeroBlocks = 64;  // workgroups that clear the rows past the last place

// rows of `y` from *total on become zero; workgroup b of kZeroBlocks
// (columns are counted without a sign: the last step of a row of almost 2^31 passes 2^31)
template <class T>
__device__ __forceinline__ void clear_tail(T* y, int64_t ldy, const Tokens& a, int b) {
  const uint32_t total = (uint32_t)max(0, *a.total);
  for (uint32_t r = total + b; r < a.pairs; r += kZeroBlocks)
    for (uint32_t c = threadIdx.x * 8; c < (uint32_t)a.cols; c += 256 * 8) store8_row(y + (int64_t)r * ldy, c, a.cols, zero8(y));
}

// A thread takes eight columns of one row: one load, k stores.
template <class T>
__global__ __launch_bounds__(256) void dispatch_kernel(Tokens a, uint32_t row0, uint32_t items, FastDiv chunks,
                                                       uint32_t nblk) {
  const T* x = (const T*)a.x;
  T* y = (T*)a.y;
  if (blockIdx.x >= nblk) return clear_tail(y, a.ldy, a, blockIdx.x - nblk);
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  if (i >= items) return;
  const uint32_t r = div_by(i, chunks);
  const int c = (int)(i - r * chunks.d) * 8;
  const int64_t row = (int64_t)row0 + r;
  const Raw8<T> v = load8_row(x + row * a.ldx, c, a.cols);
  for (int j = 0; j < a.k; ++j) {
    const uint32_t s = (uint32_t)a.slot[row * a.k + j];
    if (s < a.pairs) store8_row(y + (int64_t)s * a.ldy, c, a.cols, v);
  }
}

// A thread takes eight columns of one row and sums its k places in order, the
// loads of four of them in flight together.
template <class T>
__global__ __launch_bounds__(256) void combine_kernel(Tokens a, uint32_t row0, uint32_t items, FastDiv chunks) {
  const T* y = (const T*)a.y;
  T* x = (T*)a.x;
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  if (i >= items) return;
  const uint32_t r = div_by(i, chunks);
  const int c = (int)(i - r * chunks.d) * 8;
  const int64_t row = (int64_t)row0 + r;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int j0 = 0; j0 < a.k; j0 += 4) {
    uint32_t s[4];
    Raw8<T> r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) s[j] = j0 + j < a.k ? (uint32_t)a.slot[row * a.k + j0 + j] : a.pairs;
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = s[j] < a.pairs ? load8_row(y + (int64_t)s[j] * a.ldy, c, a.cols) : zero8(y);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (s[j] >= a.pairs) continue;
      const float w = a.weights ? a.weights[row * a.k + j0 + j] : 1.f;
      float v[8];
      widen(r[j], v);
#pragma unroll
      for (int q = 0; q < 8; ++q) acc[q] += w * v[q];
    }
  }
  Raw8<T> o;
  narrow(acc, o);
  store8_row(x + row * a.ldx, c, a.cols, o);
}

// A wave takes one row and up to KB of its places at once, so that the loads
// of all are in flight together and the row's gradient is read once for them.
template <class T, int KB>
__global__ __launch_bounds__(256) void combine_backward_kernel(Tokens a, int64_t row0, int64_t rows, uint32_t nblk) {
  const T* x = (const T*)a.x;
  const T* y = (const T*)a.y;
  T* dy = (T*)a.dy;
  if (blockIdx.x >= nblk) return clear_tail(dy, a.lddy, a, blockIdx.x - nblk);
  const int64_t row = row0 + (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (row >= row0 + rows) return;
  for (int j0 = 0; j0 < a.k; j0 += KB) {
    uint32_t s[KB];
    float w[KB], dot[KB];
#pragma unroll
    for (int j = 0; j < KB; ++j) {
      const bool there = j0 + j < a.k;
      s[j] = there ? (uint32_t)a.slot[row * a.k + j0 + j] : a.pairs;
      w[j] = there ? a.weights[row * a.k + j0 + j] : 0.f;
      dot[j] = 0.f;
    }
    for (uint32_t c = lane * 8; c < (uint32_t)a.cols; c += 512) {
      const Raw8<T> gr = load8_row(x + row * a.ldx, c, a.cols);
      Raw8<T> yr[KB];
#pragma unroll
      for (int j = 0; j < KB; ++j) yr[j] = s[j] < a.pairs ? load8_row(y + (int64_t)s[j] * a.ldy, c, a.cols) : zero8(y);
      float g[8];
      widen(gr, g);
#pragma unroll
      for (int j = 0; j < KB; ++j) {
        if (s[j] >= a.pairs) continue;
        float v[8], d[8];
        widen(yr[j], v);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          dot[j] += g[q] * v[q];
          d[q] = g[q] * w[j];
        }
        Raw8<T> o;
        narrow(d, o);
        store8_row(dy + (int64_t)s[j] * a.lddy, c, a.cols, o);
      }
    }
#pragma unroll
    for (int j = 0; j < KB; ++j) {
      const float d = wave_sum(dot[j]);
      if (lane == 0 && j0 + j < a.k) a.dweights[row * a.k + j0 + j] = d;
    }
  }
}

Tokens tokens(const agn_tokens_args& a) {
  return {a.rows, a.cols, a.k,  (uint32_t)(a.rows * a.k), a.slot, a.total, a.weights, a.x.p,
          a.x.ld, a.y.p,  a.y.ld, a.dy.p,                 a.dy.ld, a.dweights};
}

// what the three calls have in common
int check(const agn_tokens_args* a, const char* fn) {
  AGN_BLOCK_REQUIRE(a, fn, "null arguments");
  AGN_BLOCK_REQUIRE(block_dtype_ok(a->dtype), fn, "dtype must be AGN_FP32 or AGN_BF16");
  AGN_BLOCK_REQUIRE(a->rows >= 0 && a->cols >= 0, fn, "negative size");
  AGN_BLOCK_REQUIRE(a->k >= 1 && a->k <= AGN_ROUTE_MAX_K, fn, "k must be in [1, AGN_ROUTE_MAX_K]");
  AGN_BLOCK_REQUIRE(a->rows < (INT64_C(1) << 31) / a->k, fn, "rows * k must be below 2^31");
  if (a->rows == 0) return AGN_OK;
  AGN_BLOCK_REQUIRE(a->slot && a->total, fn, "null plan");
  AGN_BLOCK_VECTOR(a->slot, fn, "slot");
  AGN_BLOCK_VECTOR(a->total, fn, "total");
  AGN_BLOCK_ROWS(a->x, a->rows, a->cols, a->dtype, fn, "x");
  AGN_BLOCK_ROWS(a->y, a->rows * a->k, a->cols, a->dtype, fn, "y");
  return AGN_OK;
}

// Calls f(row0, items) for slabs of rows with fewer than 2^31 chunks each.
template <class F>
void slabs(int64_t rows, uint32_t n8, F&& f) {
  const int64_t slab = std::max<int64_t>(1, ((INT64_C(1) << 31) - 1) / n8);
  for (int64_t r = 0; r < rows; r += slab) f((uint32_t)r, (uint32_t)(std::min(slab, rows - r) * n8), r + slab >= rows);
}

template <class T>
void launch_dispatch(const agn_tokens_args& a, hipStream_t s) {
  const uint32_t n8 = chunks_of(a.cols);
  slabs(a.rows, n8, [&](uint32_t r0, uint32_t items, bool last) {
    const uint32_t nblk = (items + 255) / 256;
    hipLaunchKernelGGL(dispatch_kernel<T>, dim3(nblk + (last ? kZeroBlocks : 0)), dim3(256), 0, s, tokens(a), r0, items,
                       fast_div(n8), nblk);
  });
}
template <class T>
void launch_combine(const agn_tokens_args& a, hipStream_t s) {
  const uint32_t n8 = chunks_of(a.cols);
  slabs(a.rows, n8, [&](uint32_t r0, uint32_t items, bool) {
    hipLaunchKernelGGL(combine_kernel<T>, dim3((items + 255) / 256), dim3(256), 0, s, tokens(a), r0, items,
                       fast_div(n8));
  });
}
template <class T>
void launch_combine_backward(const agn_tokens_args& a, hipStream_t s) {
  // (a launch has fewer than 2^32 threads, a wave a row)
  constexpr int64_t kSlab = INT64_C(1) << 25;
  auto go = [&](auto kernel) {
    for (int64_t r = 0; r < a.rows; r += kSlab) {
      const int64_t rows = std::min(kSlab, a.rows - r);
      const uint32_t nblk = (uint32_t)((rows + 3) / 4), zero = r + rows == a.rows ? kZeroBlocks : 0;
      hipLaunchKernelGGL(kernel, dim3(nblk + zero), dim3(256), 0, s, tokens(a), r, rows, nblk);
    }
  };
  if (a.k == 1) go(combine_backward_kernel<T, 1>);
  else if (a.k == 2) go(combine_backward_kernel<T, 2>);
  else go(combine_backward_kernel<T, 4>);
}

}  // namespace
}  // namespace agn

using namespace agn;

extern "C" int agn_dispatch(const agn_tokens_args* a, void* stream) {
  const char* fn = "agn_dispatch";
  if (const int e = check(a, fn)) return e;
  if (a->rows == 0 || a->cols == 0) return AGN_OK;
  if (a->dtype == AGN_BF16)
    launch_dispatch<uint16_t>(*a, (hipStream_t)stream);
  else
    launch_dispatch<float>(*a, (hipStream_t)stream);
  return block_launched(fn);
}

extern "C" int agn_combine(const agn_tokens_args* a, void* stream) {
  const char* fn = "agn_combine";
  if (const int e = check(a, fn)) return e;
  AGN_BLOCK_VECTOR(a->weights, fn, "weights");
  if (a->rows == 0 || a->cols == 0) return AGN_OK;
  if (a->dtype == AGN_BF16)
    launch_combine<uint16_t>(*a, (hipStream_t)stream);
  else
    launch_combine<float>(*a, (hipStream_t)stream);
  return block_launched(fn);
}

extern "C" int agn_combine_backward(const agn_tokens_args* a, void* stream) {
  const char* fn = "agn_combine_backward";
  if (const int e = check(a, fn)) return e;
  if (a->rows == 0) return AGN_OK;
  AGN_BLOCK_REQUIRE(a->weights && a->dweights, fn, "null weights or dweights");
  AGN_BLOCK_VECTOR(a->weights, fn, "weights");
  AGN_BLOCK_VECTOR(a->dweights, fn, "dweights");
  AGN_BLOCK_ROWS(a->dy, a->rows * a->k, a->cols, a->dtype, fn, "dy");
  if (a->dtype == AGN_BF16)
    launch_combine_backward<uint16_t>(*a, (hipStream_t)stream);
  else
    launch_combine_backward<float>(*a, (hipStream_t)stream);
  return block_launched(fn);
}
