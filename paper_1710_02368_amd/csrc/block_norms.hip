// The norm after a block, its gate, mask and residual scale, and the norm
// before the next block, in one pass over the row (agn_norms), and the
// gradient of all of it in one pass (agn_norms_backward).
#include <algorithm>

#include "block_common.h"

namespace agn {
namespace {

struct NormsArgs {
  int64_t rows;
  int cols;
  float eps, alpha, inv_cols;
  const void *res, *f, *gate;
  int64_t ldres, ldf, ldgate;
  const float *w_post, *w_pre;
  MaskArgs mask;
  void *res_out, *h;
  int64_t ldres_out, ldh;
  float *rstd_post, *rstd_pre;
};

struct NormsGradArgs {
  int64_t rows;
  int cols;
  float alpha, inv_cols;
  int again;  // res is the forward call's residual: residual' is computed again
  const void *res, *f, *gate, *dres_out, *dh;
  int64_t ldres, ldf, ldgate, lddres_out, lddh;
  const float *w_post, *w_pre, *rstd_post, *rstd_pre;
  MaskArgs mask;
  void *dres, *df, *dgate;
  int64_t lddres, lddf, lddgate;
  float* part;  // [blocks][3][cols]: each workgroup's sums for w_post, w_pre and a channel gate
};

// A team of W waves holds one row, eight columns a lane (thread t columns 8t
// ..): the row is read once and both statistics are taken from registers.  A workgroup walks
// over many rows, with the next row's loads in flight during a row's sums.
template <int W>
struct Team {
  static constexpr int THREADS = W == 1 ? 256 : 64 * W;  // a workgroup
  static constexpr int TEAMS = THREADS / (64 * W);
};

// the sum of v over the team; every thread gets it.  sh: one float a wave,
// two sets, used in turn (a wave may be one sum ahead of another).
template <int W>
__device__ __forceinline__ float team_sum(float v, float (*sh)[W], int& turn) {
  v = wave_sum(v);
  if constexpr (W > 1) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) sh[turn][wave] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) v += sh[turn][w];
    turn ^= 1;
  }
  return v;
}

// eight floats of a vector of `cols`, zeros past the end
__device__ __forceinline__ void load_vec(const float* p, int c, int cols, float (&v)[8]) {
  if (c < cols)
    widen(load8_row(p, c, cols), v);
  else
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 0.f;
}

// A thread's eight columns c .. c+7 of any row, zeros past its end: the row's
// last eight are loaded where c .. c+7 reaches past it, and moved down when
// they are taken apart.
template <class T>
struct Cols {
  int at, down;  // the first column loaded; how far to move
  bool live, ragged, tiny;
  int n;  // of rows shorter than eight: columns from c on
  __device__ Cols(int c, int cols) {
    live = c < cols;
    ragged = cols & 7;
    tiny = cols < 8;
    at = min(c, max(cols - 8, 0));
    down = tiny ? 0 : min(max(c + 8 - cols, 0), 8);
    n = cols - c;
  }
  __device__ Raw8<T> load(const void* p, int64_t ld, int64_t row) const {
    const T* q = (const T*)p + row * ld;
    if (!live) return zero8(q);
    return tiny ? load8_part(q, n) : load8(q + at);
  }
  __device__ void widen_row(Raw8<T> r, float (&v)[8]) const {
    if (ragged) move_down(r, down);
    widen(r, v);
  }
};

// alpha gate mask f (rf w_post): what a row's f adds to the residual
template <int GATE>
__device__ __forceinline__ void added(float (&u)[8], const float (&g)[8], const float (&wo)[8], bool post, float rf,
                                      float alpha) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (post) u[j] *= rf * wo[j];
    u[j] *= alpha;
    if (GATE != AGN_GATE_NONE) u[j] *= g[j];
  }
}

template <class T, int W, int GATE>
__global__ __launch_bounds__(Team<W>::THREADS) void norms_kernel(NormsArgs a) {
  constexpr int TEAMS = Team<W>::TEAMS;
  __shared__ float sh[2][W];
  int turn = 0;
  const int t = threadIdx.x & (64 * W - 1), team = W == 1 ? threadIdx.x >> 6 : 0, c = 8 * t;
  const uint32_t step = mask_step(a.mask);
  const bool has_f = a.f != nullptr, post = a.w_post != nullptr, pre = a.w_pre != nullptr, live = c < a.cols;
  // the weights stay in registers over the workgroup's rows
  float wo[8], wi[8], g[8];
  if (post) load_vec(a.w_post, c, a.cols, wo);
  if (pre) load_vec(a.w_pre, c, a.cols, wi);
  if (GATE == AGN_GATE_CHANNEL) load_vec((const float*)a.gate, c, a.cols, g);
  const Cols<T> cols(c, a.cols);
  const int64_t stride = (int64_t)gridDim.x * TEAMS;
  for (int64_t row = (int64_t)blockIdx.x * TEAMS + team; row < a.rows; row += stride) {
    Raw8<T> fr, gr;
    const Raw8<T> rr = cols.load(a.res, a.ldres, row);
    if (has_f) fr = cols.load(a.f, a.ldf, row);
    if (has_f && GATE == AGN_GATE_FULL) gr = cols.load(a.gate, a.ldgate, row);
    float r[8], u[8];
    cols.widen_row(rr, r);
    if (has_f) cols.widen_row(fr, u);
    if (has_f && GATE == AGN_GATE_FULL) cols.widen_row(gr, g);
    if (has_f) {
      float rf = 1.f;
      if (post) {
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) s += u[j] * u[j];
        rf = 1.f / sqrtf(team_sum<W>(s, sh, turn) * a.inv_cols + a.eps);
        if (a.rstd_post && t == 0) a.rstd_post[row] = rf;
      }
      added<GATE>(u, g, wo, post, rf, a.alpha);
      if (a.mask.thr) mask_apply(a.mask, step, row, (uint32_t)t, u);
#pragma unroll
      for (int j = 0; j < 8; ++j) r[j] += u[j];
      if (live) {
        Raw8<T> o;
        narrow(r, o);
        store8_row((T*)a.res_out + row * a.ldres_out, c, a.cols, o);
      }
    }
    if (pre) {
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (c + j < a.cols) s += r[j] * r[j];
      const float rs = 1.f / sqrtf(team_sum<W>(s, sh, turn) * a.inv_cols + a.eps);
      if (a.rstd_pre && t == 0) a.rstd_pre[row] = rs;
      if (live) {
#pragma unroll
        for (int j = 0; j < 8; ++j) r[j] *= rs * wi[j];
        Raw8<T> o;
        narrow(r, o);
        store8_row((T*)a.h + row * a.ldh, c, a.cols, o);
      }
    }
  }
}

// With residual' = res, computed again from the forward call's residual where
// that is given, n = res rs, dn = dh w_pre:  D = dres' + rs (dn - n mean(dn n)),
// dw_pre += dh n; then m = f rf, u = m w_post, V = alpha mask D:
// dgate = V u, du = V gate, dw_post += du m, dm = du w_post,
// df = rf (dm - m mean(dm m)).  A workgroup keeps its rows' column sums in
// registers, or with 16 waves a row (128 registers a thread: with the sums among
// them 36 to 135 spilled) in LDS, where each thread adds to its own eight
// columns, and leaves them in `part`; sum_parts_kernel adds them in order.
// (Forward and gradient of 8192 x 8192 bf16: 318 us, 377 with the sums in
// registers; the bytes take 261. 4096 x 8192 float32: 275 and 323.)
template <class T, int W, int GATE>
__global__ __launch_bounds__(Team<W>::THREADS) void norms_backward_kernel(NormsGradArgs a) {
  constexpr int TEAMS = Team<W>::TEAMS;
  __shared__ float sh[2][W];
  int turn = 0;
  const int t = threadIdx.x & (64 * W - 1), team = W == 1 ? threadIdx.x >> 6 : 0, c = 8 * t;
  const uint32_t step = mask_step(a.mask);
  const bool has_f = a.f != nullptr, post = a.w_post != nullptr, pre = a.w_pre != nullptr, live = c < a.cols;
  constexpr bool ROOM = W < 16;  // registers for the sums and the next row
  float wo[8], wi[8], g[8], so[8], si[8], sg[8];  // the weights; the sums for w_post, w_pre and a channel gate
  __shared__ float4 sums[ROOM ? 1 : 3][2][ROOM ? 1 : 64 * W];
  if (post) load_vec(a.w_post, c, a.cols, wo);
  if (pre) load_vec(a.w_pre, c, a.cols, wi);
  if (GATE == AGN_GATE_CHANNEL) load_vec((const float*)a.gate, c, a.cols, g);
#pragma unroll
  for (int j = 0; j < 8; ++j) so[j] = si[j] = sg[j] = 0.f;
  if (!ROOM)
    for (int i = 0; i < 3; ++i) sums[i][0][t] = sums[i][1][t] = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](int which, const float(&v)[8]) {  // to the sums in LDS
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float4 q = sums[which][h][t];
      q.x += v[4 * h];
      q.y += v[4 * h + 1];
      q.z += v[4 * h + 2];
      q.w += v[4 * h + 3];
      sums[which][h][t] = q;
    }
  };
  Raw8<T> rn, hn, dn, fn, gn;  // the next row's
  float rfn = 1.f, rsn = 1.f;
  const Cols<T> cols(c, a.cols);
  auto fetch = [&](int64_t row) {
    if (pre) {
      rn = cols.load(a.res, a.ldres, row);
      hn = cols.load(a.dh, a.lddh, row);
      rsn = a.rstd_pre[row];
    }
    dn = a.dres_out ? cols.load(a.dres_out, a.lddres_out, row) : zero8((const T*)nullptr);
    if (has_f) fn = cols.load(a.f, a.ldf, row);
    if (has_f && GATE == AGN_GATE_FULL) gn = cols.load(a.gate, a.ldgate, row);
    if (post) rfn = a.rstd_post[row];
  };
  const int64_t stride = (int64_t)gridDim.x * TEAMS;
  int64_t row = (int64_t)blockIdx.x * TEAMS + team;
  if (ROOM && row < a.rows) fetch(row);
  for (; row < a.rows; row += stride) {
    if (!ROOM) fetch(row);
    const Raw8<T> fr = fn, hr = hn;
    const float rf = rfn, rs = rsn;
    float n[8], D[8];
    cols.widen_row(rn, n);
    cols.widen_row(dn, D);
    if (has_f && GATE == AGN_GATE_FULL) cols.widen_row(gn, g);
    if (ROOM && row + stride < a.rows) fetch(row + stride);
    uint32_t kept = 0xFFu;  // bit j: column c + j
    if (a.mask.thr) {
      const uint4 d = mask_draws(a.mask, step, row, (uint32_t)t);
      kept = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) kept |= (mask_kept(d, j, a.mask.thr) ? 1u : 0u) << j;
    }
    if (pre) {
      if (a.again) {
        float u[8];
        cols.widen_row(fr, u);
        added<GATE>(u, g, wo, post, rf, a.alpha);
#pragma unroll
        for (int j = 0; j < 8; ++j) n[j] += ((kept >> j) & 1u) ? u[j] * a.mask.scale : 0.f;
      }
      float dh[8], p[8], s = 0.f;
      cols.widen_row(hr, dh);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        n[j] *= rs;
        p[j] = dh[j] * n[j];
        if (ROOM) si[j] += p[j];
        s += p[j] * wi[j];
      }
      if constexpr (!ROOM) add(1, p);
      const float k = team_sum<W>(s, sh, turn) * a.inv_cols;
#pragma unroll
      for (int j = 0; j < 8; ++j) D[j] += rs * (dh[j] * wi[j] - n[j] * k);
    }
    if (live) {
      Raw8<T> o;
      narrow(D, o);
      store8_row((T*)a.dres + row * a.lddres, c, a.cols, o);
    }
    if (!has_f) continue;
    float m[8], dg[8], dw[8], s = 0.f;
    cols.widen_row(fr, m);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      // (every factor of a dropped element is 0, as its product is: one may be infinite)
      const bool k = (kept >> j) & 1u;
      const float v = k ? D[j] * a.mask.scale * a.alpha : 0.f;
      const float mj = k ? m[j] * rf : 0.f, wj = post && k ? wo[j] : 0.f;
      float du = v;
      dg[j] = v * (post ? mj * wj : mj);
      if (ROOM && GATE == AGN_GATE_CHANNEL) sg[j] += dg[j];
      if (GATE != AGN_GATE_NONE) du *= k ? g[j] : 0.f;
      if (post) {
        dw[j] = du * mj;
        if (ROOM) so[j] += dw[j];
        du *= wj;
        s += du * mj;
      }
      D[j] = du;  // dm (df without the norm)
    }
    if constexpr (!ROOM) {
      if (GATE == AGN_GATE_CHANNEL) add(2, dg);
      if (post) add(0, dw);
    }
    if (GATE == AGN_GATE_FULL && live) {
      Raw8<T> o;
      narrow(dg, o);
      store8_row((T*)a.dgate + row * a.lddgate, c, a.cols, o);
    }
    if (post) {
      const float k = team_sum<W>(s, sh, turn) * a.inv_cols;
#pragma unroll
      for (int j = 0; j < 8; ++j) D[j] = rf * (D[j] - m[j] * rf * k);
    }
    if (live) {
      Raw8<T> o;
      narrow(D, o);
      store8_row((T*)a.df + row * a.lddf, c, a.cols, o);
    }
  }
  // the workgroup's column sums, its teams' added in order
  __shared__ float acc[TEAMS > 1 ? 512 : 1];
  float* part = a.part + (int64_t)blockIdx.x * 3 * a.cols;
  auto leave = [&](int which, float(&v)[8]) {
    if constexpr (!ROOM) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float4 q = sums[which][h][t];
        v[4 * h] = q.x;
        v[4 * h + 1] = q.y;
        v[4 * h + 2] = q.z;
        v[4 * h + 3] = q.w;
      }
    }
    if constexpr (TEAMS > 1) {
      for (int q = 0; q < TEAMS; ++q) {
        __syncthreads();
        if (team == q)
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[c + j] = q == 0 ? v[j] : acc[c + j] + v[j];
      }
      __syncthreads();
      for (int i = threadIdx.x; i < a.cols; i += Team<W>::THREADS) part[(int64_t)which * a.cols + i] = acc[i];
    } else if (live) {
      Raw8<float> o;
      narrow(v, o);
      store8_row(part + (int64_t)which * a.cols, c, a.cols, o);
    }
  };
  if (post) leave(0, so);
  if (pre) leave(1, si);
  if (has_f && GATE == AGN_GATE_CHANNEL) leave(2, sg);
}

// Column sums of the workgroups' partial sums: 32 columns x 32 threads that
// each add every 32nd workgroup, then those 32 in order.  blockIdx.y: which.
__global__ __launch_bounds__(1024) void sum_parts_kernel(const float* part, int blocks, int cols, float* o0, float* o1,
                                                         float* o2) {
  __shared__ float sh[32][33];
  float* out = blockIdx.y == 0 ? o0 : blockIdx.y == 1 ? o1 : o2;
  if (!out) return;
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
  float s = 0.f;
  if (c < cols) {
    const float* p = part + (int64_t)blockIdx.y * cols + c;
#pragma unroll 8
    for (int b = y; b < blocks; b += 32) s += p[(int64_t)b * 3 * cols];
  }
  sh[y][x] = s;
  __syncthreads();
  if (y == 0 && c < cols) {
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) v += sh[i][x];
    out[c] = v;
  }
}

__global__ void zero_floats_kernel(float* a, float* b, float* c, int n) {
  for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
    if (a) a[i] = 0.f;
    if (b) b[i] = 0.f;
    if (c) c[i] = 0.f;
  }
}

// waves a row: the fewest that hold it, eight columns a lane
int team_waves(int cols) { return cols <= 512 ? 1 : cols <= 1024 ? 2 : cols <= 2048 ? 4 : cols <= 4096 ? 8 : 16; }

int64_t blocks_for(int64_t rows, int cols, int64_t most) {
  const int teams = cols <= 512 ? 4 : 1;
  return std::max<int64_t>(1, std::min<int64_t>((rows + teams - 1) / teams, most));
}
// Workgroups: 64 waves a CU's worth forward (twice what fits: rows even out),
// and backward, where each leaves its column sums to be added up, as many as
// fit, 16 waves a CU, or 24 with short rows (16384 x 4096 bf16 forward with
// 24, 64 and all rows' 122, 116 and 123 us; 30000 x 1001 backward with 16 and 24 144 and 118).
int64_t forward_blocks(int64_t rows, int cols) { return blocks_for(rows, cols, 64 * 256 / std::max(4, team_waves(cols))); }
int64_t backward_blocks(int64_t rows, int cols) {
  // (and at least two rows for each: the sums it leaves are three rows' bytes)
  const int64_t most = (cols <= 1024 ? 24 : 16) * 256 / std::max(4, team_waves(cols));
  return blocks_for(rows, cols, std::min(most, std::max<int64_t>(256, rows / 2)));
}

// f(T, W, GATE) as integral constants
template <class T, int W, class F>
void by_gate(int gate, F&& f) {
  if (gate == AGN_GATE_NONE) f(T(), std::integral_constant<int, W>(), std::integral_constant<int, 0>());
  else if (gate == AGN_GATE_CHANNEL) f(T(), std::integral_constant<int, W>(), std::integral_constant<int, 1>());
  else f(T(), std::integral_constant<int, W>(), std::integral_constant<int, 2>());
}
template <class T, class F>
void by_shape(int cols, int gate, F&& f) {
  const int w = team_waves(cols);
  if (w == 1) by_gate<T, 1>(gate, f);
  else if (w == 2) by_gate<T, 2>(gate, f);
  else if (w == 4) by_gate<T, 4>(gate, f);
  else if (w == 8) by_gate<T, 8>(gate, f);
  else by_gate<T, 16>(gate, f);
}
template <class F>
void dispatch_shape(int dtype, int cols, int gate, F&& f) {
  if (dtype == AGN_BF16) by_shape<uint16_t>(cols, gate, f);
  else by_shape<float>(cols, gate, f);
}

// what both calls look at
int check(const agn_norms_args& a, bool grad, const char* fn) {
  AGN_BLOCK_REQUIRE(block_dtype_ok(a.dtype), fn, "dtype must be AGN_FP32 or AGN_BF16");
  AGN_BLOCK_REQUIRE(a.rows >= 0, fn, "negative number of rows");
  AGN_BLOCK_REQUIRE(a.cols >= 1 && a.cols <= AGN_NORMS_MAX_COLS, fn, "cols must be in [1, AGN_NORMS_MAX_COLS]");
  AGN_BLOCK_REQUIRE(a.eps >= 0.f && isfinite(a.eps), fn, "eps must be finite and not negative");
  AGN_BLOCK_REQUIRE(isfinite(a.alpha), fn, "alpha must be finite");
  AGN_BLOCK_REQUIRE(a.gate_kind >= AGN_GATE_NONE && a.gate_kind <= AGN_GATE_FULL, fn, "unknown gate_kind");
  AGN_BLOCK_REQUIRE(mask_threshold(a.mask.rate) >= 0, fn, "rate must be in [0, 1), below 1 - 2^-17");
  AGN_BLOCK_REQUIRE(element_aligned(a.w_post, AGN_FP32) && element_aligned(a.w_pre, AGN_FP32), fn,
                    "weights not aligned to their element");
  AGN_BLOCK_VECTOR(a.mask.step_dev, fn, "step_dev");
  AGN_BLOCK_VECTOR(a.rstd_post, fn, "rstd_post");
  AGN_BLOCK_VECTOR(a.rstd_pre, fn, "rstd_pre");
  if (a.rows == 0) return AGN_OK;  // (pointers of nothing may be null: the parts cannot be told)
  if (a.f.p) {
    AGN_BLOCK_ROWS(a.f, a.rows, a.cols, a.dtype, fn, "f");
    if (a.gate_kind == AGN_GATE_FULL) AGN_BLOCK_ROWS(a.gate, a.rows, a.cols, a.dtype, fn, "gate");
    if (a.gate_kind == AGN_GATE_CHANNEL)
      AGN_BLOCK_REQUIRE(a.gate.p && element_aligned(a.gate.p, AGN_FP32), fn, "gate: null or unaligned pointer");
  } else {
    AGN_BLOCK_REQUIRE(a.w_pre, fn, "neither f nor w_pre");
    AGN_BLOCK_REQUIRE(!a.w_post && a.gate_kind == AGN_GATE_NONE, fn, "w_post or a gate without f");
  }
  if (!grad || (a.w_pre && a.residual.p)) AGN_BLOCK_ROWS(a.residual, a.rows, a.cols, a.dtype, fn, "residual");
  if (grad ? a.w_pre && !a.residual.p : a.f.p != nullptr)
    AGN_BLOCK_ROWS(a.residual_out, a.rows, a.cols, a.dtype, fn, "residual_out");
  return AGN_OK;
}

}  // namespace
}  // namespace agn

using namespace agn;

extern "C" int agn_norms(const agn_norms_args* a, void* stream) {
  const char* fn = "agn_norms";
  AGN_BLOCK_REQUIRE(a, fn, "null arguments");
  if (const int e = check(*a, false, fn)) return e;
  if (a->w_pre) AGN_BLOCK_ROWS(a->h, a->rows, a->cols, a->dtype, fn, "h");
  if (a->rows == 0) return AGN_OK;
  NormsArgs k{};
  k.rows = a->rows;
  k.cols = a->cols;
  k.eps = a->eps;
  k.alpha = a->alpha;
  k.inv_cols = 1.f / (float)a->cols;
  k.res = a->residual.p;
  k.ldres = a->residual.ld;
  k.f = a->f.p;
  k.ldf = a->f.ld;
  k.gate = a->gate.p;
  k.ldgate = a->gate.ld;
  k.w_post = a->w_post;
  k.w_pre = a->w_pre;
  k.mask = mask_args(a->mask);
  k.res_out = a->residual_out.p;
  k.ldres_out = a->residual_out.ld;
  k.h = a->h.p;
  k.ldh = a->h.ld;
  k.rstd_post = a->rstd_post;
  k.rstd_pre = a->rstd_pre;
  const dim3 grid((uint32_t)forward_blocks(a->rows, a->cols));
  dispatch_shape(a->dtype, a->cols, a->gate_kind, [&](auto t, auto w, auto g) {
    hipLaunchKernelGGL((norms_kernel<decltype(t), decltype(w)::value, decltype(g)::value>), grid,
                       dim3(Team<decltype(w)::value>::THREADS), 0, (hipStream_t)stream, k);
  });
  return block_launched(fn);
}

extern "C" int64_t agn_norms_backward_workspace(int64_t rows, int32_t cols) {
  if (rows < 0 || cols < 1 || cols > AGN_NORMS_MAX_COLS) {
    block_fail(AGN_EINVAL, "agn_norms_backward_workspace", "bad size");
    return -1;
  }
  return backward_blocks(rows, cols) * 3 * cols * (int64_t)sizeof(float);
}

extern "C" int agn_norms_backward(const agn_norms_grad_args* a, void* stream) {
  const char* fn = "agn_norms_backward";
  AGN_BLOCK_REQUIRE(a, fn, "null arguments");
  const agn_norms_args& f = a->fwd;
  if (const int e = check(f, true, fn)) return e;
  const bool has_f = f.f.p != nullptr;
  if (a->dresidual_out.p) AGN_BLOCK_ROWS(a->dresidual_out, f.rows, f.cols, f.dtype, fn, "dresidual_out");
  AGN_BLOCK_ROWS(a->dresidual, f.rows, f.cols, f.dtype, fn, "dresidual");
  if (f.w_pre) {
    AGN_BLOCK_ROWS(a->dh, f.rows, f.cols, f.dtype, fn, "dh");
    AGN_BLOCK_REQUIRE(a->dw_pre, fn, "null dw_pre");
    AGN_BLOCK_REQUIRE(f.rstd_pre || f.rows == 0, fn, "null rstd_pre");
  }
  if (has_f) AGN_BLOCK_ROWS(a->df, f.rows, f.cols, f.dtype, fn, "df");
  if (f.w_post) {
    AGN_BLOCK_REQUIRE(a->dw_post, fn, "null dw_post");
    AGN_BLOCK_REQUIRE(f.rstd_post || f.rows == 0, fn, "null rstd_post");
  }
  AGN_BLOCK_VECTOR(a->dw_pre, fn, "dw_pre");
  AGN_BLOCK_VECTOR(a->dw_post, fn, "dw_post");
  if (f.gate_kind == AGN_GATE_CHANNEL) {
    AGN_BLOCK_REQUIRE(a->dgate.p, fn, "null dgate");
    AGN_BLOCK_VECTOR(a->dgate.p, fn, "dgate");
  }
  if (has_f && f.gate_kind == AGN_GATE_FULL) AGN_BLOCK_ROWS(a->dgate, f.rows, f.cols, f.dtype, fn, "dgate");
  float* dgate = f.gate_kind == AGN_GATE_CHANNEL ? (float*)a->dgate.p : nullptr;
  float* dw_post = f.w_post ? a->dw_post : nullptr;
  float* dw_pre = f.w_pre ? a->dw_pre : nullptr;
  const hipStream_t s = (hipStream_t)stream;
  if (f.rows == 0) {
    hipLaunchKernelGGL(zero_floats_kernel, dim3(16), dim3(256), 0, s, dw_post, dw_pre, dgate, f.cols);
    return block_launched(fn);
  }
  const int64_t need = agn_norms_backward_workspace(f.rows, f.cols);
  AGN_BLOCK_REQUIRE(a->workspace && ((uintptr_t)a->workspace & 15) == 0 && a->workspace_bytes >= need, fn,
                    "workspace missing, unaligned or too small");
  NormsGradArgs k{};
  k.rows = f.rows;
  k.cols = f.cols;
  k.alpha = f.alpha;
  k.inv_cols = 1.f / (float)f.cols;
  k.again = f.residual.p && has_f;
  k.res = f.residual.p ? f.residual.p : f.residual_out.p;
  k.ldres = f.residual.p ? f.residual.ld : f.residual_out.ld;
  k.f = f.f.p;
  k.ldf = f.f.ld;
  k.gate = f.gate.p;
  k.ldgate = f.gate.ld;
  k.dres_out = a->dresidual_out.p;
  k.lddres_out = a->dresidual_out.ld;
  k.dh = a->dh.p;
  k.lddh = a->dh.ld;
  k.w_post = f.w_post;
  k.w_pre = f.w_pre;
  k.rstd_post = f.rstd_post;
  k.rstd_pre = f.rstd_pre;
  k.mask = mask_args(f.mask);
  k.dres = a->dresidual.p;
  k.lddres = a->dresidual.ld;
  k.df = a->df.p;
  k.lddf = a->df.ld;
  k.dgate = a->dgate.p;
  k.lddgate = a->dgate.ld;
  k.part = (float*)a->workspace;
  const uint32_t blocks = (uint32_t)backward_blocks(f.rows, f.cols);
  dispatch_shape(f.dtype, f.cols, f.gate_kind, [&](auto t, auto w, auto g) {
    hipLaunchKernelGGL((norms_backward_kernel<decltype(t), decltype(w)::value, decltype(g)::value>),
                       dim3(blocks), dim3(Team<decltype(w)::value>::THREADS), 0, s, k);
  });
  if (dw_post || dw_pre || dgate)
    hipLaunchKernelGGL(sum_parts_kernel, dim3((f.cols + 31) / 32, 3), dim3(1024), 0, s, k.part, (int)blocks, f.cols,
                       dw_post, dw_pre, dgate);
  return block_launched(fn);
}
