// Routing: the k largest logits of a row and their softmax weights, and the
// stable sort of the rows' choices by expert (agn_route), with the gradient
// of the weights (agn_route_backward).
#include <algorithm>
#include <type_traits>

#include "block_common.h"

namespace agn {
namespace {

// Total order of the logits as unsigned integers: a NaN above every number,
// -0 equal to 0; -inf is kMinusInf.  0 is below every logit.
constexpr uint32_t kMinusInf = 0x007FFFFFu;
__device__ __forceinline__ uint32_t order_key(float l) {
  if (l != l) return 0xFFFFFFFFu;
  const uint32_t b = __float_as_uint(l + 0.f);
  return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float key_logit(uint32_t k) {
  if (k == 0xFFFFFFFFu) return __uint_as_float(0x7FC00000u);
  return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}

// ---- the choice --------------------------------------------------------------
// T lanes take a row, NE adjacent experts a lane.  Each of the k choices is a
// maximum over the row's lanes of (order key, lowest expert): over the lane's
// own experts first, then over the lanes, by DPP moves within 16 of them.

template <int T>
__device__ __forceinline__ void best_of(uint32_t& key, uint32_t& expert) {
  auto take = [&](uint32_t k, uint32_t e) {
    const bool better = k > key || (k == key && e < expert);
    key = better ? k : key;
    expert = better ? e : expert;
  };
#define AGN_MOVE(v, ctrl) __builtin_amdgcn_mov_dpp((int)(v), ctrl, 0xF, 0xF, false)
  take(AGN_MOVE(key, 0xB1), AGN_MOVE(expert, 0xB1));    // quad_perm(1, 0, 3, 2)
  take(AGN_MOVE(key, 0x4E), AGN_MOVE(expert, 0x4E));    // quad_perm(2, 3, 0, 1)
  take(AGN_MOVE(key, 0x141), AGN_MOVE(expert, 0x141));  // row_half_mirror
  if constexpr (T >= 16) take(AGN_MOVE(key, 0x140), AGN_MOVE(expert, 0x140));  // row_mirror
#undef AGN_MOVE
#pragma unroll
  for (int d = 16; d < T; d <<= 1) take(__shfl_xor(key, d), __shfl_xor(expert, d));
}
template <int T>
__device__ __forceinline__ float group_sum(float v) {
  v += dpp_move<0xB1>(v);
  v += dpp_move<0x4E>(v);
  v += dpp_move<0x141>(v);
  if constexpr (T >= 16) v += dpp_move<0x140>(v);
#pragma unroll
  for (int d = 16; d < T; d <<= 1) v += __shfl_xor(v, d);
  return v;
}

// The choices of row `row` (every lane of the wave calls; lanes of rows past
// the last work on the last one and write nothing).
template <class E, int T, int NE>
__device__ __forceinline__ void choose_row(const E* logits, int64_t ldl, int64_t row, int64_t rows, int experts, int k,
                                           int over_all, int32_t* chosen, float* weights) {
  const int t = threadIdx.x & (T - 1), e0 = t * NE;
  const bool live = row < rows;
  const E* p = logits + (live ? row : rows - 1) * ldl;
  float l[NE];
  if constexpr (NE == 8) {
    if (e0 < experts) {
      widen(load8_row(p, e0, experts), l);
    }
  }
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    if constexpr (NE == 8) {
      if (e0 + i >= experts) l[i] = -INFINITY;
    } else {
      l[i] = -INFINITY;
      if (e0 + i < experts) {
        if constexpr (sizeof(E) == 2) l[i] = bf16_to_f32(p[e0 + i]);
        else l[i] = p[e0 + i];
      }
    }
  }
  uint32_t key[NE];
#pragma unroll
  for (int i = 0; i < NE; ++i) key[i] = order_key(l[i]);
  // lane t keeps choices t, t + T, ...
  constexpr int KL = (AGN_ROUTE_MAX_K + T - 1) / T;
  uint32_t mine[KL], top = kMinusInf;
  int expert[KL];
#pragma unroll
  for (int q = 0; q < KL; ++q) {
    mine[q] = kMinusInf;
    expert[q] = -1;
  }
  for (int j = 0; j < k; ++j) {
    uint32_t bk = key[0], be = e0;
#pragma unroll
    for (int i = 1; i < NE; ++i) {
      const bool better = key[i] > bk;
      bk = better ? key[i] : bk;
      be = better ? e0 + i : be;
    }
    best_of<T>(bk, be);
    if (j == 0) top = bk;
    const bool has = bk > kMinusInf;
#pragma unroll
    for (int q = 0; q < KL; ++q)
      if (has && j == q * T + t) {
        mine[q] = bk;
        expert[q] = (int)be;
      }
#pragma unroll
    for (int i = 0; i < NE; ++i)
      if (be == (uint32_t)(e0 + i)) key[i] = 0;
  }
  const float m = key_logit(top);
  float e[KL], sum = 0.f;
#pragma unroll
  for (int q = 0; q < KL; ++q) {
    e[q] = expert[q] >= 0 ? expf(key_logit(mine[q]) - m) : 0.f;
    sum += e[q];
  }
  if (over_all) {
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < NE; ++i)
      if (l[i] != -INFINITY) sum += expf(l[i] - m);
  }
  sum = group_sum<T>(sum);
#pragma unroll
  for (int q = 0; q < KL; ++q) {
    const int j = q * T + t;
    if (live && j < k) {
      chosen[row * k + j] = expert[q];
      weights[row * k + j] = expert[q] >= 0 ? e[q] / sum : 0.f;
    }
  }
}

// ---- the sort ---------------------------------------------------------------
// A counting sort over experts + 1 bins, the last for pairs without an
// expert.  A workgroup takes a segment of the rows: the first kernel chooses
// for them and counts their pairs by bin; in the second each workgroup adds up
// the counts before its own, and its waves walk over their parts of the
// segment in order.  Where one workgroup takes all rows, one kernel does both.

constexpr int kThreads = 512, kWaves = kThreads / 64;

struct RouteArgs {
  const void* logits;  // or null: chosen is given
  int64_t ldl, rows;
  int64_t seg;  // rows a segment
  int nseg, experts, k, over_all, bits;
  int32_t* chosen;
  float* weights;
  int32_t *offsets, *source, *slot;
  int32_t* counts;  // [segment][bin]
};

__device__ __forceinline__ uint32_t bin_of(int32_t expert, int experts) {
  return (uint32_t)expert < (uint32_t)experts ? (uint32_t)expert : (uint32_t)experts;
}

// lanes with the same bin as this one (bits: enough for the number of bins)
__device__ __forceinline__ uint64_t same_bin(uint32_t bin, bool live, int bits) {
  uint64_t same = __ballot(live);
  for (int b = 0; b < bits; ++b) {
    const uint64_t m = __ballot((bin >> b) & 1u);
    same &= ((bin >> b) & 1u) ? m : ~m;
  }
  return same;
}

template <class E, int T, int NE>
__device__ __forceinline__ void choose_segment(const RouteArgs& a, int64_t r0, int64_t r1) {
  constexpr int RPW = 64 / T;  // rows a wave
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int64_t r = r0 + wave * RPW; r < r1; r += kWaves * RPW)
    choose_row<E, T, NE>((const E*)a.logits, a.ldl, r + lane / T, r1, a.experts, a.k, a.over_all, a.chosen, a.weights);
}

// Places of the pairs p0 .. p1 - 1 (a workgroup): base[bin] is the first
// place of the segment's pairs of a bin.  lds: (kWaves + 1) * bins ints, the
// first `bins` of them base.
__device__ __forceinline__ void place_segment(const RouteArgs& a, int64_t p0, int64_t p1, int32_t* lds) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, bins = a.experts + 1;
  int32_t* next = lds + bins * (1 + wave);
  for (int i = threadIdx.x; i < kWaves * bins; i += kThreads) lds[bins + i] = 0;
  __syncthreads();
  // a wave's part: a multiple of 64 pairs
  const int64_t part = ((p1 - p0 + kWaves - 1) / kWaves + 63) / 64 * 64;
  const int64_t w0 = min(p0 + wave * part, p1), w1 = min(w0 + part, p1);
  for (int64_t p = w0 + lane; p < w1; p += 64) atomicAdd(&next[bin_of(a.chosen[p], a.experts)], 1);
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += kThreads) {
    int32_t at = lds[b];
    for (int w = 0; w < kWaves; ++w) {
      const int32_t n = lds[bins * (1 + w) + b];
      lds[bins * (1 + w) + b] = at;
      at += n;
    }
  }
  __syncthreads();
  volatile int32_t* mine = next;
  for (int64_t p = w0; p < w1; p += 64) {
    const bool live = p + lane < w1;
    const uint32_t bin = live ? bin_of(a.chosen[p + lane], a.experts) : 0;
    const uint64_t same = same_bin(bin, live, a.bits);
    const int before = __popcll(same & ((UINT64_C(1) << lane) - 1));
    int at = 0;
    if (live) at = mine[bin];
    __builtin_amdgcn_wave_barrier();
    if (live && before == 0) mine[bin] = at + __popcll(same);
    __builtin_amdgcn_wave_barrier();
    if (live) {
      const bool has = bin < (uint32_t)a.experts;
      a.source[at + before] = has ? (int32_t)(p + lane) : -1;
      a.slot[p + lane] = has ? at + before : -1;
    }
  }
}

// exclusive prefix sums of v[0 .. bins) in LDS (a workgroup)
__device__ __forceinline__ void scan_bins(int32_t* v, int bins) {
  __syncthreads();
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x;
    int32_t base = 0;
    for (int b0 = 0; b0 < bins; b0 += 64) {
      const int b = b0 + lane;
      const int32_t n = b < bins ? v[b] : 0;
      int32_t inc = n;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int32_t o = __shfl_up(inc, d);
        if (lane >= d) inc += o;
      }
      if (b < bins) v[b] = base + inc - n;
      base += __shfl(inc, 63);
    }
  }
  __syncthreads();
}

// the segment's choices, and their counts by bin into lds[0 .. bins)
template <class E, int T, int NE>
__device__ __forceinline__ void choose_and_count(const RouteArgs& a, int64_t r0, int64_t r1, int32_t* lds) {
  const int bins = a.experts + 1;
  for (int b = threadIdx.x; b < bins; b += kThreads) lds[b] = 0;
  if (a.logits) choose_segment<E, T, NE>(a, r0, r1);
  __syncthreads();  // (and the choices, in memory, are seen by the whole workgroup)
  for (int64_t p = r0 * a.k + threadIdx.x; p < r1 * a.k; p += kThreads)
    atomicAdd(&lds[bin_of(a.chosen[p], a.experts)], 1);
  __syncthreads();
}

template <class E, int T, int NE>
__global__ __launch_bounds__(kThreads) void route_one_kernel(RouteArgs a) {
  extern __shared__ int32_t lds[];
  choose_and_count<E, T, NE>(a, 0, a.rows, lds);
  scan_bins(lds, a.experts + 1);
  for (int b = threadIdx.x; b <= a.experts; b += kThreads) a.offsets[b] = lds[b];
  place_segment(a, 0, a.rows * a.k, lds);
}

template <class E, int T, int NE>
__global__ __launch_bounds__(kThreads) void choose_kernel(RouteArgs a) {
  extern __shared__ int32_t lds[];
  const int64_t r0 = blockIdx.x * a.seg, r1 = min(r0 + a.seg, a.rows);
  choose_and_count<E, T, NE>(a, r0, r1, lds);
  for (int b = threadIdx.x; b <= a.experts; b += kThreads) a.counts[(int64_t)blockIdx.x * (a.experts + 1) + b] = lds[b];
}

// lds: max((kWaves + 1) bins, 2 kThreads) ints
__global__ __launch_bounds__(kThreads) void place_kernel(RouteArgs a) {
  extern __shared__ int32_t lds[];
  const int bins = a.experts + 1, s = blockIdx.x;
  // every bin's pairs in all segments and in those before this one: groups of
  // threads, a thread a bin, each take every so many-th segment
  int32_t all = 0, before = 0;
  if (bins <= kThreads) {
    const int groups = kThreads / bins, grp = threadIdx.x / bins, b = threadIdx.x % bins;
    if (grp < groups) {
#pragma unroll 8
      for (int i = grp; i < a.nseg; i += groups) {
        const int32_t n = a.counts[(int64_t)i * bins + b];
        all += n;
        before += i < s ? n : 0;
      }
    }
    lds[threadIdx.x] = all;
    lds[kThreads + threadIdx.x] = before;
    __syncthreads();
    all = before = 0;
    if ((int)threadIdx.x < bins) {
      for (int q = 0; q < groups; ++q) {
        all += lds[q * bins + threadIdx.x];
        before += lds[kThreads + q * bins + threadIdx.x];
      }
    }
    __syncthreads();
    if ((int)threadIdx.x < bins) {
      lds[threadIdx.x] = all;
      lds[bins + threadIdx.x] = before;
    }
  } else {
    for (int b = threadIdx.x; b < bins; b += kThreads) {
      all = before = 0;
#pragma unroll 8
      for (int i = 0; i < a.nseg; ++i) {
        const int32_t n = a.counts[(int64_t)i * bins + b];
        all += n;
        before += i < s ? n : 0;
      }
      lds[b] = all;
      lds[bins + b] = before;
    }
  }
  scan_bins(lds, bins);
  if (s == 0)
    for (int b = threadIdx.x; b < bins; b += kThreads) a.offsets[b] = lds[b];
  for (int b = threadIdx.x; b < bins; b += kThreads) lds[b] += lds[bins + b];
  __syncthreads();
  const int64_t r0 = s * a.seg, r1 = min(r0 + a.seg, a.rows);
  place_segment(a, r0 * a.k, r1 * a.k, lds);
}

__global__ void no_pairs_kernel(int32_t* offsets, int n) {
  for (int i = threadIdx.x; i < n; i += 256) offsets[i] = 0;
}

// Rows a segment, and segments: one workgroup takes up to 1024 pairs; beyond,
// up to 256 segments, fewer with many experts (every workgroup of the second
// kernel reads all counts: at most 131072 of them).  32768 rows x 64 experts,
// k = 8, with 128, 256, 512 and 1024 segments: 24.8, 19.0, 21.8, 21.5 us.
int64_t segments(int64_t rows, int experts, int k) {
  if (rows * k <= 1024) return 1;
  const int64_t most = std::min<int64_t>(256, 131072 / (experts + 1));
  return std::min<int64_t>(most, (rows * k + 511) / 512);
}
int64_t segment_rows(int64_t rows, int experts, int k) {
  const int64_t n = segments(rows, experts, k);
  return (rows + n - 1) / n;
}

// f(T, NE) for the lanes a row and the experts a lane
template <class F>
void by_experts(int experts, F&& f) {
  using std::integral_constant;
  if (experts <= 8) f(integral_constant<int, 8>(), integral_constant<int, 1>());
  else if (experts <= 32) f(integral_constant<int, 8>(), integral_constant<int, 4>());
  else if (experts <= 64) f(integral_constant<int, 8>(), integral_constant<int, 8>());
  else if (experts <= 128) f(integral_constant<int, 16>(), integral_constant<int, 8>());
  else if (experts <= 512) f(integral_constant<int, 64>(), integral_constant<int, 8>());
  else f(integral_constant<int, 64>(), integral_constant<int, 16>());
}

// ---- gradient ---------------------------------------------------------------

// A thread takes eight experts of one row and reads the row's choices.  The
// softmax over all experts needs no sum: the first choice is the largest
// logit, so p_e = exp(l_e - l_first) w_first.
template <class T>
__global__ __launch_bounds__(256) void route_backward_kernel(const T* logits, int64_t ldl, int64_t row0, uint32_t items,
                                                             FastDiv chunks, int experts, int k, int over_all,
                                                             const int32_t* chosen, const float* weights,
                                                             const float* dweights, T* dlogits, int64_t ldd) {
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  if (i >= items) return;
  const uint32_t r = div_by(i, chunks);
  const int64_t row = row0 + r;
  const int c = (int)(i - r * chunks.d) * 8;
  float s = 0.f;
  for (int j = 0; j < k; ++j)
    if ((uint32_t)chosen[row * k + j] < (uint32_t)experts) s += weights[row * k + j] * dweights[row * k + j];
  float v[8];
#pragma unroll
  for (int q = 0; q < 8; ++q) v[q] = 0.f;
  const int32_t first = chosen[row * k];
  if (over_all && (uint32_t)first < (uint32_t)experts) {
    float l[8], top;
    widen(load8_row(logits + row * ldl, c, experts), l);
    if constexpr (sizeof(T) == 2) top = bf16_to_f32(logits[row * ldl + first]);
    else top = logits[row * ldl + first];
    const float f = -weights[row * k] * s;
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (l[q] != -INFINITY) v[q] = expf(l[q] - top) * f;
  }
  for (int j = 0; j < k; ++j) {
    const int32_t e = chosen[row * k + j] - c;
    if ((uint32_t)e >= 8u || e + c >= experts) continue;
    const float w = weights[row * k + j], g = dweights[row * k + j];
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (q == e) v[q] += over_all ? w * g : w * (g - s);
  }
  Raw8<T> o;
  narrow(v, o);
  store8_row(dlogits + row * ldd, c, experts, o);
}

template <class T>
void launch_backward(const agn_route_grad_args& a, hipStream_t s) {
  const uint32_t n8 = (uint32_t)((a.experts + 7) / 8);
  const int64_t slab = ((INT64_C(1) << 31) - 1) / n8;
  for (int64_t r = 0; r < a.rows; r += slab) {
    const uint32_t items = (uint32_t)(std::min(slab, a.rows - r) * n8);
    hipLaunchKernelGGL(route_backward_kernel<T>, dim3((items + 255) / 256), dim3(256), 0, s, (const T*)a.logits.p,
                       a.logits.ld, r, items, fast_div(n8), a.experts, a.k, a.over_all, a.chosen, a.weights, a.dweights,
                       (T*)a.dlogits.p, a.dlogits.ld);
  }
}

int check_sizes(int64_t rows, int32_t experts, int32_t k, const char* fn) {
  AGN_BLOCK_REQUIRE(experts >= 1 && experts <= AGN_ROUTE_MAX_EXPERTS, fn, "experts must be in [1, AGN_ROUTE_MAX_EXPERTS]");
  AGN_BLOCK_REQUIRE(k >= 1 && k <= AGN_ROUTE_MAX_K && k <= experts, fn, "k must be in [1, min(experts, AGN_ROUTE_MAX_K)]");
  AGN_BLOCK_REQUIRE(rows >= 0 && rows < (INT64_C(1) << 31) / k, fn, "rows must be >= 0 and rows * k below 2^31");
  return AGN_OK;
}

}  // namespace
}  // namespace agn

using namespace agn;

extern "C" int64_t agn_route_workspace(int64_t rows, int32_t experts, int32_t k) {
  if (check_sizes(rows, experts, k, "agn_route_workspace")) return -1;
  const int64_t n = segments(rows, experts, k);
  return n > 1 ? n * (experts + 1) * (int64_t)sizeof(int32_t) : 0;
}

extern "C" int agn_route(const agn_route_args* a, void* stream) {
  const char* fn = "agn_route";
  AGN_BLOCK_REQUIRE(a, fn, "null arguments");
  if (const int e = check_sizes(a->rows, a->experts, a->k, fn)) return e;
  AGN_BLOCK_REQUIRE(a->over_all == 0 || a->over_all == 1, fn, "over_all must be 0 or 1");
  AGN_BLOCK_REQUIRE(a->offsets, fn, "null offsets");
  AGN_BLOCK_VECTOR(a->offsets, fn, "offsets");
  const hipStream_t s = (hipStream_t)stream;
  if (a->rows == 0) {
    hipLaunchKernelGGL(no_pairs_kernel, dim3(1), dim3(256), 0, s, a->offsets, a->experts + 1);
    return block_launched(fn);
  }
  AGN_BLOCK_REQUIRE(a->chosen && a->source && a->slot, fn, "null chosen, source or slot");
  AGN_BLOCK_VECTOR(a->chosen, fn, "chosen");
  AGN_BLOCK_VECTOR(a->source, fn, "source");
  AGN_BLOCK_VECTOR(a->slot, fn, "slot");
  if (a->logits.p) {
    AGN_BLOCK_REQUIRE(block_dtype_ok(a->dtype), fn, "dtype must be AGN_FP32 or AGN_BF16");
    AGN_BLOCK_REQUIRE(a->weights, fn, "null weights");
    AGN_BLOCK_VECTOR(a->weights, fn, "weights");
    AGN_BLOCK_ROWS(a->logits, a->rows, a->experts, a->dtype, fn, "logits");
  }
  const int64_t need = agn_route_workspace(a->rows, a->experts, a->k);
  AGN_BLOCK_REQUIRE(need == 0 || (a->workspace && ((uintptr_t)a->workspace & 15) == 0 && a->workspace_bytes >= need), fn,
                    "workspace missing, unaligned or too small");
  RouteArgs r{};
  r.logits = a->logits.p;
  r.ldl = a->logits.ld;
  r.rows = a->rows;
  r.seg = segment_rows(a->rows, a->experts, a->k);
  r.nseg = (int)((a->rows + r.seg - 1) / r.seg);
  r.experts = a->experts;
  r.k = a->k;
  r.over_all = a->over_all;
  while ((1 << r.bits) < a->experts + 1) ++r.bits;
  r.chosen = a->chosen;
  r.weights = a->weights;
  r.offsets = a->offsets;
  r.source = a->source;
  r.slot = a->slot;
  r.counts = (int32_t*)a->workspace;
  const int bins = a->experts + 1;
  const uint32_t lds = std::max((kWaves + 1) * bins, 2 * kThreads) * sizeof(int32_t);
  by_experts(a->experts, [&](auto t, auto ne) {
    constexpr int T = decltype(t)::value, NE = decltype(ne)::value;
    auto go = [&](auto one, auto many) {
      hipLaunchKernelGGL(r.nseg == 1 ? one : many, dim3(r.nseg), dim3(kThreads), lds, s, r);
    };
    if (a->logits.p && a->dtype == AGN_BF16)
      go(route_one_kernel<uint16_t, T, NE>, choose_kernel<uint16_t, T, NE>);
    else
      go(route_one_kernel<float, T, NE>, choose_kernel<float, T, NE>);
  });
  if (r.nseg > 1) hipLaunchKernelGGL(place_kernel, dim3(r.nseg), dim3(kThreads), lds, s, r);
  return block_launched(fn);
}

extern "C" int agn_route_backward(const agn_route_grad_args* a, void* stream) {
  const char* fn = "agn_route_backward";
  AGN_BLOCK_REQUIRE(a, fn, "null arguments");
  if (const int e = check_sizes(a->rows, a->experts, a->k, fn)) return e;
  AGN_BLOCK_REQUIRE(block_dtype_ok(a->dtype), fn, "dtype must be AGN_FP32 or AGN_BF16");
  AGN_BLOCK_REQUIRE(a->over_all == 0 || a->over_all == 1, fn, "over_all must be 0 or 1");
  if (a->rows == 0) return AGN_OK;
  AGN_BLOCK_REQUIRE(a->chosen && a->weights && a->dweights, fn, "null chosen, weights or dweights");
  AGN_BLOCK_VECTOR(a->chosen, fn, "chosen");
  AGN_BLOCK_VECTOR(a->weights, fn, "weights");
  AGN_BLOCK_VECTOR(a->dweights, fn, "dweights");
  if (a->over_all) AGN_BLOCK_ROWS(a->logits, a->rows, a->experts, a->dtype, fn, "logits");
  AGN_BLOCK_ROWS(a->dlogits, a->rows, a->experts, a->dtype, fn, "dlogits");
  if (a->dtype == AGN_BF16)
    launch_backward<uint16_t>(*a, (hipStream_t)stream);
  else
    launch_backward<float>(*a, (hipStream_t)stream);
  return block_launched(fn);
}
