// The experts' products in float32 (v_mfma_f32_32x32x2_f32; one MFMA takes A[i
// = lane % 32][k = lane / 32] and B[k][j = lane % 32]).
//
// Output tiles of 128 x 128, 64 x 64 or 64 x 32, four waves, K in steps of
// BK (32 or 64), operand tiles through registers (16-byte loads, any
// alignment) into two LDS stages: the next step's loads are in flight during a
// step's MFMAs.  (Two, three or four steps ahead were no faster: 3330 rows of
// 5 experts, 517 -> 259, forward in 64 x 64 tiles 28 us with one, 30 to 31 with
// more.)  The tiles lie in LDS as they are loaded, [outer][k] or [k][outer].
// The order of k in a sum is free: of eight k the lanes 0 .. 31 take the first four and the lanes 32 .. 63 the
// last, so that a lane's fragments of four MFMAs are one 16-byte read of a
// K-contiguous tile; they are read while the MFMAs of the eight k before run.
// 3330 rows of 5 experts, 517 -> 259: forward 19 us (48 TFLOP/s), 8192 of 8, 2048
// -> 2048: 622 us (110 TFLOP/s).  What bounds short sums is the latency of a
// step: three workgroups of 64 x 32 lie on a CU (53 KB of LDS each), so that all
// 425 to 513 tiles of the former's products are there at once, and the matrix
// pipe is busy 20 to 29% of their time.
#include <type_traits>

#include "block_experts.h"

namespace agn {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int NT = 256;

// A wave has NB x NB blocks of 32 x 32; in tiles narrower than they are high
// (64 x 32) two waves share a block, each taking every other eight k.
template <int TM_, int TN_>
struct Geo {
  static constexpr int TM = TM_, TN = TN_, NB = TM / 64, BK = 4096 / TM;
  static constexpr int WN = TN / (32 * NB), WK = 2 / WN;  // waves across, waves a block
  // LDS row lengths (4 floats more than a row: 16 rows' 16-byte reads at one k
  // meet different banks) and the larger of an operand's two layouts
  static constexpr int LD_KC = BK + 4;
  static constexpr int size(int t) { return t * LD_KC > BK * (t + 4) ? t * LD_KC : BK * (t + 4); }
  static constexpr int A = size(TM), STAGE = A + size(TN), EPI_LD = TN + 4, EPI = TM * EPI_LD;
  static constexpr int LDS = 2 * STAGE > WK * EPI ? 2 * STAGE : WK * EPI;  // floats
};

// One operand's NL loads of four floats a thread and step, of T outer indices
// and BK k.  KC: outer index r, k 4q; KS: k r, outer 4q.  Rows past the edge of a K-contiguous operand
// repeat the last one (outputs that are not stored); all else past an edge
// is zeros.  Four floats across the end of a row are loaded as the row's last
// four and moved down when they are stored; TINY: element by element, where
// rows have fewer than four.
template <bool KC, int T, int BK, bool TINY>
struct Staged {
  static constexpr int QR = KC ? BK / 4 : T / 4, LD = KC ? BK + 4 : T + 4, NL = T * BK / 4 / NT;
  const float *p[NL], *home;  // the thread's sources at step 0; four floats that are there
  int64_t advance;
  int outer;
  bool edge;
  blk_u32x4 v[NL];

  __device__ static int r(int u) { return (threadIdx.x + NT * u) / QR; }
  __device__ static int q(int u) { return (threadIdx.x + NT * u) % QR; }
  __device__ void init(const float* base, int64_t ld, int outer_) {
    outer = outer_;
    edge = !KC && outer < T;
    home = base + (KC ? 0 : min(0, outer - 4));
    advance = KC ? BK : BK * ld;
#pragma unroll
    for (int u = 0; u < NL; ++u)
      p[u] = KC ? base + (int64_t)min(r(u), outer - 1) * ld + 4 * q(u)
                : base + (int64_t)r(u) * ld + (TINY ? 4 * q(u) : min(4 * q(u), outer - 4));
  }
  __device__ void load(int kt, int K) {
#pragma unroll
    for (int u = 0; u < NL; ++u) {
      const float* src = p[u] + kt * advance;
      const int rest = K - kt * BK - (KC ? 4 * q(u) : r(u));  // k from the first to the end
      if constexpr (!TINY) {
        v[u] = *reinterpret_cast<const blk_u32x4_a4*>(rest > 0 ? (KC ? src + min(0, rest - 4) : src) : home);
      } else {
        const int n = KC ? rest : rest > 0 ? outer - 4 * q(u) : 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[u][j] = j < n ? __float_as_uint(src[j]) : 0u;
      }
    }
  }
  __device__ void store(float* tile, int kt, int K) {
    if (!TINY && (kt + 1) * BK > K) {
#pragma unroll
      for (int u = 0; u < NL; ++u) {
        const int rest = K - kt * BK - (KC ? 4 * q(u) : r(u));
        move_down(v[u], rest > 0 ? (KC ? max(0, 4 - rest) : 0) : 4);
      }
    }
    if (!TINY && edge) {
#pragma unroll
      for (int u = 0; u < NL; ++u) move_down(v[u], min(max(0, 4 * q(u) + 4 - outer), 4));
    }
#pragma unroll
    for (int u = 0; u < NL; ++u) {
      *reinterpret_cast<blk_u32x4*>(tile + r(u) * LD + 4 * q(u)) = v[u];
    }
  }
  // the lane's k 8 g + 4 lh .. + 3 of outer index o
  __device__ static void frag(const float* tile, int g, int lh, int o, float (&f)[4]) {
    if (KC) {
      const float4 w = *reinterpret_cast<const float4*>(tile + o * LD + 8 * g + 4 * lh);
      f[0] = w.x;
      f[1] = w.y;
      f[2] = w.z;
      f[3] = w.w;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = tile[(8 * g + 4 * lh + j) * LD + o];
    }
  }
};

template <int PROD, int TM, int TN, bool TINY>
__global__ __launch_bounds__(NT) void product_kernel(ProductArgs g) {
  using G = Geo<TM, TN>;
  constexpr bool A_KC = PROD != PROD_DW, B_KC = PROD == PROD_FWD;
  constexpr int NB = G::NB, BK = G::BK, WN = G::WN, WK = G::WK;
  __shared__ __attribute__((aligned(16))) float lds[G::LDS];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave >> 1, wn = wave & (WN - 1), wk = wave & (WK - 1), li = lane & 31, lh = lane >> 5;
  const int tn = (g.N + TN - 1) / TN;
  int e, m0, mend, n0, K;
  const float *pa, *pb;
  float *dw = nullptr, *dbias = nullptr;
  if (PROD == PROD_DW) {
    const WeightTile w = weight_tile_of(g, blockIdx.x, weight_tiles(g, TM, TN));
    if (w.e < 0) return;
    e = w.e;
    m0 = (w.t / tn) * TM;
    mend = g.M;
    n0 = (w.t % tn) * TN;
    K = w.rows;
    dw = w.out;
    dbias = w.dbias;
    pa = (const float*)g.a + w.r0 * g.lda + m0;
    pb = (const float*)g.b + w.r0 * g.ldb + n0;
  } else {
    const int nblk = gridDim.x - kTailBlocks;
    if ((int)blockIdx.x >= nblk) return clear_rows<float, NT>(g, blockIdx.x - nblk);
    RowTiles tiles;
    tiles.init(g, TM);
    const int total = tiles.total * tn;
    if ((int)blockIdx.x >= total) return;
    const int logical = xcd_remap(blockIdx.x, total);
    const RowTile t = tiles.find(g, logical / tn);
    if (t.e < 0) return;
    e = t.e;
    m0 = t.r0;
    mend = t.rend;
    n0 = (logical % tn) * TN;
    K = g.K;
    pa = (const float*)g.a + m0 * g.lda;
    pb = (const float*)g.b + e * g.bstride + (B_KC ? n0 * g.ldb : (int64_t)n0);
  }
  Staged<A_KC, TM, BK, TINY> la;
  Staged<B_KC, TN, BK, TINY> lb;
  la.init(pa, g.lda, mend - m0);
  lb.init(pb, g.ldb, g.N - n0);
  f32x16 acc[NB][NB];
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  // the bias gradient (DW, first column of tiles): the waves wn = 0 sum their
  // rows, a block's two waves half of them each
  const bool sums = PROD == PROD_DW && dbias && n0 == 0 && wn == 0;
  float bsum[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) bsum[i] = 0.f;

  const int nk = (K + BK - 1) / BK;
  if (nk > 0) {
    la.load(0, K);
    lb.load(0, K);
    la.store(lds, 0, K);
    lb.store(lds + G::A, 0, K);
  }
  __syncthreads();
  for (int kt = 0; kt < nk; ++kt) {
    const float* rd = lds + (kt & 1) * G::STAGE;
    float* wr = lds + ((kt + 1) & 1) * G::STAGE;
    const bool more = kt + 1 < nk;
    if (more) {
      la.load(kt + 1, K);
      lb.load(kt + 1, K);
    }
    float fa[2][NB][4], fb[2][NB][4];
    auto read = [&](int g) {  // of the wave's, a set of eight k
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        la.frag(rd, g * WK + wk, lh, wm * (TM / 2) + 32 * i + li, fa[g & 1][i]);
        lb.frag(rd + G::A, g * WK + wk, lh, wn * (32 * NB) + 32 * i + li, fb[g & 1][i]);
      }
    };
    read(0);
#pragma unroll
    for (int g = 0; g < BK / (8 * WK); ++g) {
      if (g + 1 < BK / (8 * WK)) read(g + 1);
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
          for (int j = 0; j < NB; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[g & 1][i][q], fb[g & 1][j][q], acc[i][j], 0, 0, 0);
      if (PROD == PROD_DW && sums) {
#pragma unroll
        for (int i = 0; i < NB; ++i) bsum[i] += (fa[g & 1][i][0] + fa[g & 1][i][1]) + (fa[g & 1][i][2] + fa[g & 1][i][3]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if (more) {
      la.store(wr, kt + 1, K);
      lb.store(wr + G::A, kt + 1, K);
    }
    __syncthreads();
  }
  __shared__ float other_sum[WK == 2 ? TM : 1];  // a block's second wave's
  if (PROD == PROD_DW && sums) {  // lanes lh = 0 and 1 hold half of the rows' sums each
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      bsum[i] += __shfl_xor(bsum[i], 32);
      if (WK == 2 && wk == 1 && lh == 0) other_sum[wm * (TM / 2) + 32 * i + li] = bsum[i];
    }
  }
  // The tile goes through LDS; a thread finishes chunks of eight columns,
  // always the same ones, and what it needs for them is loaded before.
  constexpr int CPR = TN / 8, NC = TM * CPR / NT;  // chunks a row; chunks a thread
  const int cl = 8 * (tid % CPR), c = n0 + cl;
  const uint32_t step = mask_step(g.mask);
  float bias[8];
  Raw8<float> gate[NC];
  if (PROD == PROD_FWD) load_bias(g, e, c, bias);
  if (PROD == PROD_DX) {
#pragma unroll
    for (int u = 0; u < NC; ++u) gate[u] = load_gate<float>(g, min(m0 + tid / CPR + (NT / CPR) * u, mend - 1), c);
  }
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        lds[wk * G::EPI + (wm * (TM / 2) + 32 * i + 8 * (r >> 2) + 4 * lh + (r & 3)) * G::EPI_LD + wn * (32 * NB) +
            32 * j + li] = acc[i][j][r];
  __syncthreads();
  if (PROD == PROD_DW && sums && wk == 0 && lh == 0) {
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int o = wm * (TM / 2) + 32 * i + li;
      if (m0 + o < mend) dbias[m0 + o] = WK == 2 ? bsum[i] + other_sum[o] : bsum[i];
    }
  }
  if (c >= g.N) return;
#pragma unroll
  for (int u = 0; u < NC; ++u) {
    const int rl = tid / CPR + (NT / CPR) * u, row = m0 + rl;
    if (row >= mend) continue;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[j] = lds[rl * G::EPI_LD + cl + j];
      if (WK == 2) v[j] += lds[G::EPI + rl * G::EPI_LD + cl + j];
    }
    finish8<PROD, float>(g, step, row, c, bias, gate[u], v);
    Raw8<float> o;
    narrow(v, o);
    store8_row(PROD == PROD_DW ? dw + (int64_t)row * g.N : (float*)g.out + (int64_t)row * g.ldo, c, g.N, o);
  }
}

template <int PROD, int TM, int TN>
void launch_tiles(const ProductKernel& k, const ProductArgs& g, hipStream_t s) {
  const int tn = (g.N + TN - 1) / TN;
  const int blocks =
      PROD == PROD_DW ? (int)weight_parts_most(g) * weight_tiles(g, TM, TN) : row_tiles_most(g, TM) * tn + kTailBlocks;
  hipLaunchKernelGGL((k.way == WAY_TINY ? product_kernel<PROD, TM, TN, true> : product_kernel<PROD, TM, TN, false>),
                     dim3(blocks), dim3(NT), 0, s, g);
}
template <int PROD>
void launch(const ProductKernel& k, const ProductArgs& g, hipStream_t s) {
  if (k.tm == 128) launch_tiles<PROD, 128, 128>(k, g, s);
  else if (k.tn == 32) launch_tiles<PROD, 64, 32>(k, g, s);
  else launch_tiles<PROD, 64, 64>(k, g, s);
}

}  // namespace

hipError_t launch_product_f32(int prod, const ProductKernel& k, const ProductArgs& g, hipStream_t s) {
  if (prod == PROD_DW) launch<PROD_DW>(k, g, s);
  else if (prod == PROD_FWD) launch<PROD_FWD>(k, g, s);
  else launch<PROD_DX>(k, g, s);
  return hipGetLastError();
}

}  // namespace agn
