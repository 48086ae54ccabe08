// Shared by the block operators (agn_block.h): element types, chunks of eight
// elements, the counter-based random mask, argument checks.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "agn_block.h"
#include "device_common.h"

namespace agn {

// sets agn_block_error() to "fn: what", or "fn: name: what"
int block_fail(int code, const char* fn, const char* what, const char* name = nullptr);
int block_launched(const char* fn);                          // the last launch's status

// the kept draws' threshold round(65536 rate), or -1 for a rate that is not allowed
inline int mask_threshold(float rate) {
  if (!(rate >= 0.f && rate < 1.f)) return -1;
  const long t = lrintf(rate * 65536.f);
  return t <= 65535 ? (int)t : -1;
}

// chunks of eight columns a row (any cols >= 0)
inline uint32_t chunks_of(int32_t cols) { return ((uint32_t)cols + 7) / 8; }

inline bool block_dtype_ok(int32_t d) { return d == AGN_FP32 || d == AGN_BF16; }
inline bool element_aligned(const void* p, int32_t dtype) { return ((uintptr_t)p & (dtype == AGN_BF16 ? 1 : 3)) == 0; }

// nullptr, or what is wrong with a matrix of rows
inline const char* rows_error(const agn_rows& m, int64_t rows, int64_t cols, int32_t dtype) {
  if (rows == 0 || cols == 0) return nullptr;
  if (!m.p) return "null pointer";
  if (!element_aligned(m.p, dtype)) return "pointer not aligned to its element";
  if (rows > 1 && m.ld < cols) return "row stride below the row's length";
  if (rows > 1 && m.ld > (INT64_C(1) << 48) / rows) return "matrix too large";
  return nullptr;
}

#define AGN_BLOCK_REQUIRE(cond, fn, what)                             \
  do {                                                                \
    if (!(cond)) return ::agn::block_fail(AGN_EINVAL, fn, what);      \
  } while (0)
#define AGN_BLOCK_ROWS(m, rows, cols, dtype, fn, name)                                                     \
  do {                                                                                                     \
    if (const char* e_ = ::agn::rows_error(m, rows, cols, dtype))                                          \
      return ::agn::block_fail(AGN_EINVAL, fn, e_, name);                                                  \
  } while (0)
// a vector of 32-bit elements (null: nothing to look at)
#define AGN_BLOCK_VECTOR(p, fn, name)                                                                   \
  do {                                                                                                  \
    if ((uintptr_t)(p) & 3) return ::agn::block_fail(AGN_EINVAL, fn, "pointer not aligned to its element", name); \
  } while (0)

// the mask as the kernels take it: threshold 0 draws nothing
struct MaskArgs {
  uint32_t thr, step;
  uint32_t key0, key1;
  const uint32_t* step_dev;
  float scale;
};
inline MaskArgs mask_args(const agn_mask& m) {
  MaskArgs a{};
  a.thr = (uint32_t)mask_threshold(m.rate);
  a.step = m.step;
  a.key0 = (uint32_t)m.seed;
  a.key1 = (uint32_t)(m.seed >> 32);
  a.step_dev = a.thr ? m.step_dev : nullptr;
  a.scale = 65536.f / (float)(65536u - a.thr);
  return a;
}

// n / d and n % d for n < 2^31 by a product (d >= 1): with s = ceil(log2 d)
// and m = floor(2^32 (2^s - d) / d) + 1, n / d = (umulhi(m, n) + n) >> s
struct FastDiv {
  uint32_t d, mul, shift;
};
inline FastDiv fast_div(uint32_t d) {
  uint32_t s = 0;
  while ((UINT64_C(1) << s) < d) ++s;
  return {d, (uint32_t)(((UINT64_C(1) << 32) * ((UINT64_C(1) << s) - d)) / d + 1), s};
}

namespace {

__device__ __forceinline__ uint32_t div_by(uint32_t n, const FastDiv& f) { return (__umulhi(f.mul, n) + n) >> f.shift; }

__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) {
#if defined(__gfx950__)
  return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96);  // (from a ^ b ^ c the compiler makes two instructions)
#else
  return a ^ b ^ c;
#endif
}

// The ten rounds of Philox4x32.
__device__ __forceinline__ uint4 philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t p = (uint64_t)c0 * 0xD2511F53u, q = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = xor3((uint32_t)(q >> 32), c1, k0);
    c1 = (uint32_t)q;
    c2 = xor3((uint32_t)(p >> 32), c3, k1);
    c3 = (uint32_t)p;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}

__device__ __forceinline__ uint32_t mask_step(const MaskArgs& m) { return m.step + (m.step_dev ? *m.step_dev : 0u); }

// the draws of columns 8*c8 .. 8*c8+7 of a row
__device__ __forceinline__ uint4 mask_draws(const MaskArgs& m, uint32_t step, int64_t row, uint32_t c8) {
  return philox(c8, (uint32_t)row, (uint32_t)((uint64_t)row >> 32), step, m.key0, m.key1);
}
__device__ __forceinline__ bool mask_kept(const uint4& d, int j, uint32_t thr) {
  const uint32_t w = (j >> 1) == 0 ? d.x : (j >> 1) == 1 ? d.y : (j >> 1) == 2 ? d.z : d.w;
  return ((j & 1) ? w >> 16 : w & 0xFFFFu) >= thr;
}
// v = mask * v (a dropped element is 0 whatever it was)
__device__ __forceinline__ void mask_apply(const MaskArgs& m, uint32_t step, int64_t row, uint32_t c8, float (&v)[8]) {
  const uint4 d = mask_draws(m, step, row, c8);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = mask_kept(d, j, m.thr) ? v[j] * m.scale : 0.f;
}

// float32 -> bfloat16, to nearest even, NaN kept a NaN (v_cvt_pk_bf16_f32)
__device__ __forceinline__ uint16_t to_bf16(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }

typedef uint32_t blk_u32x4 __attribute__((ext_vector_type(4)));
// 16 bytes at an address aligned to the element only: gfx950 serves unaligned
// global accesses, and the compiler emits the wide load for them
typedef uint32_t blk_u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t blk_u32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));

// Eight elements as they lie in memory.
template <class T>
struct Raw8;
template <>
struct Raw8<float> {
  blk_u32x4 a, b;
};
template <>
struct Raw8<uint16_t> {
  blk_u32x4 a;
};

__device__ __forceinline__ Raw8<uint16_t> zero8(const uint16_t*) { return {blk_u32x4{0, 0, 0, 0}}; }
__device__ __forceinline__ Raw8<float> zero8(const float*) { return {blk_u32x4{0, 0, 0, 0}, blk_u32x4{0, 0, 0, 0}}; }

__device__ __forceinline__ Raw8<uint16_t> load8(const uint16_t* p) {
  return {*reinterpret_cast<const blk_u32x4_a2*>(p)};
}
__device__ __forceinline__ Raw8<float> load8(const float* p) {
  const blk_u32x4_a4* q = reinterpret_cast<const blk_u32x4_a4*>(p);
  return {q[0], q[1]};
}
// the first n < 8 of them, zeros after
__device__ __forceinline__ Raw8<uint16_t> load8_part(const uint16_t* p, int n) {
  Raw8<uint16_t> r = zero8(p);
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < n) r.a[j >> 1] |= (uint32_t)p[j] << (16 * (j & 1));
  return r;
}
__device__ __forceinline__ Raw8<float> load8_part(const float* p, int n) {
  Raw8<float> r = zero8(p);
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < n) (j < 4 ? r.a : r.b)[j & 3] = __float_as_uint(p[j]);
  return r;
}
// element j becomes element j + d's (0 <= d <= 8), zeros come in above: a chunk
// of n < 8 elements at the end of a row is loaded as the row's last eight and
// moved down by 8 - n, without a branch
__device__ __forceinline__ void move_down(Raw8<uint16_t>& r, int d) {
  uint64_t lo = ((uint64_t)r.a[1] << 32) | r.a[0], hi = ((uint64_t)r.a[3] << 32) | r.a[2];
  if (d >= 4) {
    lo = hi;
    hi = 0;
  }
  if (d >= 8) lo = 0;
  const int s = 16 * (d & 3);
  lo = (lo >> s) | ((hi << 1) << (63 - s));
  hi >>= s;
  r.a = blk_u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}
// the same for four floats (0 <= d <= 4)
__device__ __forceinline__ void move_down(blk_u32x4& v, int d) {
  const blk_u32x4 t = (d & 1) ? blk_u32x4{v[1], v[2], v[3], 0u} : v;
  v = (d & 2) ? blk_u32x4{t[2], t[3], 0u, 0u} : t;
  if (d >= 4) v = blk_u32x4{0u, 0u, 0u, 0u};
}
__device__ __forceinline__ void move_down(Raw8<float>& r, int d) {
  if (d >= 4) {
    r.a = r.b;
    r.b = blk_u32x4{0u, 0u, 0u, 0u};
    d -= 4;
  }
#pragma unroll
  for (int s = 1; s <= 2; s <<= 1)
    if (d & s) {
      r.a = s == 1 ? blk_u32x4{r.a[1], r.a[2], r.a[3], r.b[0]} : blk_u32x4{r.a[2], r.a[3], r.b[0], r.b[1]};
      r.b = s == 1 ? blk_u32x4{r.b[1], r.b[2], r.b[3], 0u} : blk_u32x4{r.b[2], r.b[3], 0u, 0u};
    }
  if (d >= 4) r.a = blk_u32x4{0u, 0u, 0u, 0u};
}
// columns c .. c+7 of a row of `cols`, zeros past its end (c < cols; c + 8 may pass 2^31)
template <class T>
__device__ __forceinline__ Raw8<T> load8_row(const T* row, int c, int cols) {
  if (cols < 8) return load8_part(row + c, cols - c);
  Raw8<T> r = load8(row + min(c, cols - 8));
  if (c > cols - 8) move_down(r, c - (cols - 8));
  return r;
}

__device__ __forceinline__ void widen(const Raw8<uint16_t>& r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(r.a[i] << 16);
    v[2 * i + 1] = __uint_as_float(r.a[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void widen(const Raw8<float>& r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = __uint_as_float(r.a[i]);
    v[4 + i] = __uint_as_float(r.b[i]);
  }
}
__device__ __forceinline__ void narrow(const float (&v)[8], Raw8<uint16_t>& r) {
#pragma unroll
  for (int i = 0; i < 4; ++i) r.a[i] = (uint32_t)to_bf16(v[2 * i]) | ((uint32_t)to_bf16(v[2 * i + 1]) << 16);
}
__device__ __forceinline__ void narrow(const float (&v)[8], Raw8<float>& r) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r.a[i] = __float_as_uint(v[i]);
    r.b[i] = __float_as_uint(v[4 + i]);
  }
}

__device__ __forceinline__ void store8(uint16_t* p, const Raw8<uint16_t>& r) {
  *reinterpret_cast<blk_u32x4_a2*>(p) = r.a;
}
__device__ __forceinline__ void store8(float* p, const Raw8<float>& r) {
  blk_u32x4_a4* q = reinterpret_cast<blk_u32x4_a4*>(p);
  q[0] = r.a;
  q[1] = r.b;
}
__device__ __forceinline__ void store8_part(uint16_t* p, const Raw8<uint16_t>& r, int n) {
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < n) p[j] = (uint16_t)(r.a[j >> 1] >> (16 * (j & 1)));
}
__device__ __forceinline__ void store8_part(float* p, const Raw8<float>& r, int n) {
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < n) p[j] = __uint_as_float((j < 4 ? r.a : r.b)[j & 3]);
}
template <class T>
__device__ __forceinline__ void store8_row(T* row, int c, int cols, const Raw8<T>& r) {
  if (cols - c >= 8)
    store8(row + c, r);
  else
    store8_part(row + c, r, cols - c);
}

}  // namespace
}  // namespace agn
