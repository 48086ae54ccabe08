// The experts' products in bfloat16.
//
// TR x TR output tiles (256 or 128), eight waves: wave (wm, wn) = (w / 4,
// w % 4) owns TR/2 rows and TR/4 columns as blocks of 32 x 32
// (v_mfma_f32_32x32x16_bf16).  K in steps of 64, two LDS stages.  A step is
// two halves of two slices of 16 k; each half's MFMAs run on fragments that
// were read from LDS during the half before, and the one barrier of a step
// lies between the halves, where every wave has the rest of the step's
// fragments in registers and the next step's tiles have landed:
//   read slices 2, 3 of step kt          | MFMAs of slices 0, 1
//   wait, barrier
//   start the loads of step kt + 2, read slices 0, 1 of step kt + 1
//                                        | MFMAs of slices 2, 3
//
// Operand tiles travel straight into LDS (global_load_lds_dwordx4) where every
// chunk of eight elements is a 16-byte aligned piece of one row; else, in
// 128 x 128 tiles only, through registers: loaded where the direct load would
// start, written to LDS half a step later, a step ahead of their use.
//
// LDS layout of an operand tile (TR * 8 chunks of 16 bytes; a wave's load
// instruction fills 64 consecutive chunks, lane l chunk l):
//   K-contiguous: chunk (row r, k 8q) at 8r + (q ^ key(r)), key(r) = (r >> 1)
//     & 7: a load instruction reads whole 128-byte lines (with 32 k a step it
//     read half lines, and the other half again a step later: forward 16384 x
//     2048 x 2048 798 TFLOP/s against 928 of the input gradient); a fragment
//     read's 16 rows at one q fall in 16 distinct bank groups modulo 256 bytes;
//   K-strided (rows = k, TR/8 chunks of 8 outer per row): chunk (k, c) at
//     (TR/8)k + (c ^ key(k)), key(k) = 0, 6, 12, 10 for k % 4 = 0..3.  A
//     fragment is two transposing 8-byte reads (ds_read_b64_tr_b16), each
//     over four consecutive k rows; the key puts those rows in distinct bank
//     windows (32 bytes modulo 128, 64 bytes modulo 256).
#include <type_traits>

#include "block_experts.h"
#include "direct_load.h"

namespace agn {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

constexpr int BK = 64, NT = 512;

template <int TR>
struct Geo {
  static constexpr int NI = TR / 64, NJ = TR / 128;  // blocks of a wave
  static constexpr int IPW = TR / 64;                // load instructions a wave, operand and step
  static constexpr int TILE = TR * BK * 2, STAGE = 2 * TILE;
  static constexpr int CPK = TR / 8, RPI = 64 / CPK;  // K-strided: chunks a k row, k rows a load instruction
  static constexpr int EPI_LD = TR + 4, EPI_BYTES = (TR / 2) * EPI_LD * 4;
  static constexpr int LDS = 2 * STAGE > EPI_BYTES ? 2 * STAGE : EPI_BYTES;
};

__device__ uint4 zero_chunk[4];  // what lanes past the end of K load

__device__ __forceinline__ int line_key(int r) { return (r >> 1) & 7; }
__device__ __forceinline__ int ks_key(int k) { return (0xAC60 >> (4 * (k & 3))) & 15; }
template <int TR>
__device__ __forceinline__ int ks_byte(int k, int c) { return ((TR / 8) * k + (c ^ ks_key(k))) * 16; }

// How operand tiles reach LDS: straight (DIRECT); through registers (STAGED),
// a chunk at the end of a row being loaded as the row's last eight elements
// and moved down when it is written to LDS; or element by element (TINY),
// where rows have fewer than eight.
enum { DIRECT = WAY_DIRECT, STAGED = WAY_STAGED, TINY = WAY_TINY };

// One operand's loads (instruction j = IPW wave + u; lane l fills LDS chunk
// 64 j + l).  Outer indices past the edge repeat the last row or chunk (they
// feed outputs that are not stored), k past the end is zeros.
template <bool KC, int TR, int WAY>
struct Loader {
  static constexpr int IPW = Geo<TR>::IPW;
  const uint16_t *p[IPW], *home;  // the lane's sources at step 0; a chunk that is there
  int k[IPW];                     // its k in a step
  int64_t advance;                // elements from one step to the next
  // not DIRECT
  Raw8<uint16_t> v[IPW];
  int past[IPW];  // K-strided: how far the chunk reaches past the edge
  bool edge;      // some chunk of the tile does

  __device__ void init(const uint16_t* base, int64_t ld, int outer, int wave, int lane) {
    advance = KC ? BK : BK * ld;
    edge = !KC && outer < TR;
    home = base + (KC ? 0 : min(0, outer - 8));
#pragma unroll
    for (int u = 0; u < IPW; ++u) {
      const int j = IPW * wave + u;
      if (KC) {
        const int r = 8 * j + lane / 8;
        k[u] = 8 * ((lane % 8) ^ line_key(r));
        p[u] = base + (int64_t)min(r, outer - 1) * ld + k[u];
      } else {
        const int r = Geo<TR>::RPI * j + lane / Geo<TR>::CPK, o = 8 * ((lane % Geo<TR>::CPK) ^ ks_key(r));
        k[u] = r;
        past[u] = max(0, o + 8 - outer);
        p[u] = base + (int64_t)r * ld + (WAY == TINY ? o : min(o, (WAY == DIRECT ? (outer + 7) & ~7 : outer) - 8));
      }
    }
  }
  // start load u of step kt into the tile at LDS byte `tile`, or into v[u]
  __device__ void start(int u, uint32_t tile, int kt, int K, int wave) {
    const uint16_t* src = p[u] + kt * advance;
    const int rest = K - kt * BK - k[u];  // k from the chunk's first to the end
    if constexpr (WAY == DIRECT) {
      fire(rest > 0 ? (const void*)src : (const void*)zero_chunk, tile + 1024 * (IPW * wave + u));
    } else if constexpr (WAY == STAGED) {
      v[u] = load8(rest > 0 ? (KC ? src + min(0, rest - 8) : src) : home);
    } else {
      const int n = KC ? rest : rest > 0 ? 8 - past[u] : 0;
      v[u] = zero8(src);
      if (n >= 8) v[u] = load8(src);
      else if (n > 0) v[u] = load8_part(src, n);
    }
  }
  __device__ void finish(int u, char* tile, int kt, int K, int wave, int lane) {
    if constexpr (WAY == STAGED) {
      const int rest = K - kt * BK - k[u];
      if ((kt + 1) * BK > K) move_down(v[u], rest > 0 ? (KC ? max(0, 8 - rest) : 0) : 8);
      if (edge) move_down(v[u], min(past[u], 8));
    }
    *reinterpret_cast<blk_u32x4*>(tile + 1024 * (IPW * wave + u) + 16 * lane) = v[u].a;
  }
};

// the fragment of the block at `outer_off` for slice s of the step in `tile`
template <bool KC, int TR>
__device__ __forceinline__ bf16x8 slice_frag(const char* tile, int s, int outer_off, int li, int lh) {
  if (KC) {
    const int r = outer_off + li;
    return *reinterpret_cast<const bf16x8*>(tile + (8 * r + ((2 * s + lh) ^ line_key(r))) * 16);
  }
  // read c covers k = 16s + 8lh + 4c + e: within each group of 16 lanes, lane i
  // receives element e from the 4 bf16 at the address that lane 4e + i/4
  // supplies, offset i%4; so lane j supplies row 16s + 8lh + 4c + j/4 at column
  // outer_off + 16*(li/16) + 4*(j%4), j = li % 16, and lane i ends up with
  // column outer_off + li
  const int col = outer_off + 16 * (li / 16) + 4 * (li % 4);
  bf16x4 q[2];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const int k = 16 * s + 8 * lh + 4 * c + (li % 16) / 4;
    q[c] = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                          (lds_i16x4*)(tile + ks_byte<TR>(k, col / 8) + 2 * (col % 8))));
  }
  return __builtin_shufflevector(q[0], q[1], 0, 1, 2, 3, 4, 5, 6, 7);
}

__device__ __forceinline__ float sum8(const bf16x8& v) {
  const blk_u32x4 w = __builtin_bit_cast(blk_u32x4, v);
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) s += __uint_as_float(w[i] << 16) + __uint_as_float(w[i] & 0xFFFF0000u);
  return s;
}

// One output tile of expert e: rows m0 .. mend-1 at most (DW: rows of w),
// columns from n0; pa, pb: the operands at the tile's first outer index.
template <int PROD, int TR, int WAY>
__device__ __forceinline__ void tile(const ProductArgs& g, int e, int m0, int mend, int n0, int K, const uint16_t* pa,
                                     const uint16_t* pb, float* dw, float* dbias, char* lds) {
  constexpr bool A_KC = PROD != PROD_DW, B_KC = PROD == PROD_FWD;
  using G = Geo<TR>;
  constexpr int NI = G::NI, NJ = G::NJ;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6) & 7;
  const int wm = wave >> 2, wn = wave & 3, li = lane & 31, lh = lane >> 5;
  Loader<A_KC, TR, WAY> la;
  Loader<B_KC, TR, WAY> lb;
  la.init(pa, g.lda, mend - m0, wave, lane);
  lb.init(pb, g.ldb, g.N - n0, wave, lane);
  // the bias gradient (DW, first column of tiles): wave wn sums the rows of
  // its blocks i with i % 4 = wn
  const bool sums = PROD == PROD_DW && dbias && n0 == 0;
  float bsum = 0.f;

  f32x16 acc[NI][NJ];
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  const int nk = (K + BK - 1) / BK;
  const uint32_t base = lds_off(lds);
  bf16x8 a0[NI][2], b0[NJ][2], a1[NI][2], b1[NJ][2];
  // fragment f of a half (the order in which the MFMAs take them)
  constexpr int NF = 2 * (NI + NJ);
  auto read = [&](int f, int stage, int h, bf16x8(&a)[NI][2], bf16x8(&b)[NJ][2]) {
    const char* st = lds + stage * G::STAGE;
    const int s = f / (NI + NJ), i = f % (NI + NJ);
    if (i < NJ)
      b[i][s] = slice_frag<B_KC, TR>(st + G::TILE, 2 * h + s, wn * (TR / 4) + 32 * i, li, lh);
    else
      a[i - NJ][s] = slice_frag<A_KC, TR>(st, 2 * h + s, wm * (TR / 2) + 32 * (i - NJ), li, lh);
  };
  auto start = [&](int u, int kt) {
    const uint32_t st = base + (kt & 1) * G::STAGE;
    if (u < G::IPW)
      la.start(u, st, kt, K, wave);
    else
      lb.start(u - G::IPW, st + G::TILE, kt, K, wave);
  };
  auto finish = [&](int u, int kt) {
    char* st = lds + (kt & 1) * G::STAGE;
    if (u < G::IPW)
      la.finish(u, st, kt, K, wave, lane);
    else
      lb.finish(u - G::IPW, st + G::TILE, kt, K, wave, lane);
  };
  // Half a step: MFMAs on (a, b), and between them the next half's fragments
  // into (an, bn) and, in the second half, the loads of step kt + 2.  The
  // order is fixed here: left to itself the compiler reads last, to save
  // registers, and eight loads in a row hold the wave, and the MFMAs behind
  // them, in issue until the memory pipeline has room.
  constexpr int NM = 2 * NI * NJ, NG = 2 * G::IPW, MPG = NM / NG;  // groups of MPG MFMAs and a load
  auto half = [&](auto second, int kt, const bf16x8(&a)[NI][2], const bf16x8(&b)[NJ][2], int stage, int h,
                  bf16x8(&an)[NI][2], bf16x8(&bn)[NJ][2]) {
#pragma unroll
    for (int q = 0; q < NG; ++q) {
      if constexpr (decltype(second)::value) start(q, kt + 2);
      else if constexpr (WAY != DIRECT) finish(q, kt + 1);  // (started half a step ago)
#pragma unroll
      for (int f = q * NF / NG; f < (q + 1) * NF / NG; ++f) read(f, stage, h, an, bn);
#pragma unroll
      for (int m = q * MPG; m < (q + 1) * MPG; ++m) {
        const int sl = m / (NI * NJ), i = m % (NI * NJ) / NJ, j = m % NJ;
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i][sl], b[j][sl], acc[i][j], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if (PROD == PROD_DW && sums) {
#pragma unroll
      for (int i = 0; i < NI; ++i)
        if (i == wn) bsum += sum8(a[i][0]) + sum8(a[i][1]);
    }
  };
  static_assert(NM % NG == 0, "groups of equal size");
  if (nk > 0) {
#pragma unroll
    for (int u = 0; u < NG; ++u) start(u, 0);
    if constexpr (WAY != DIRECT) {
#pragma unroll
      for (int u = 0; u < NG; ++u) finish(u, 0);
    }
#pragma unroll
    for (int u = 0; u < NG; ++u) start(u, 1);
    if constexpr (WAY == DIRECT) wait_vm<NG>();
    wait_lgkm0();
    barrier();
#pragma unroll
    for (int f = 0; f < NF; ++f) read(f, 0, 0, a0, b0);
  }
  for (int kt = 0; kt < nk; ++kt) {
    __builtin_amdgcn_sched_barrier(0);
    half(std::false_type(), kt, a0, b0, kt & 1, 1, a1, b1);
    wait_lgkm0();
    if constexpr (WAY == DIRECT) wait_vm<0>();
    barrier();
    half(std::true_type(), kt, a1, b1, (kt + 1) & 1, 0, a0, b0);  // (the reads past the last step are not used)
  }
  if constexpr (WAY == DIRECT) wait_vm<0>();
  // no load is in flight (those past the end of K read zeros), every wave is
  // done reading: the LDS is free for the epilogue, TR / 2 rows at a time
  wait_lgkm0();
  barrier();
  // A thread finishes chunks of eight columns, always the same ones; what it
  // needs from memory is loaded before the tile goes through LDS.
  float* et = reinterpret_cast<float*>(lds);
  constexpr int CPR = TR / 8, NC = (TR / 2) * CPR / NT;  // chunks a row; chunks a thread and pass
  const int cl = 8 * (tid % CPR), c = n0 + cl;
  const uint32_t step = mask_step(g.mask);
  float bias[8];
  if (PROD == PROD_FWD) load_bias(g, e, c, bias);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    Raw8<uint16_t> gate[NC];
    if (PROD == PROD_DX) {
#pragma unroll
      for (int u = 0; u < NC; ++u)
        gate[u] = load_gate<uint16_t>(g, min(m0 + (TR / 2) * h + tid / CPR + (NT / CPR) * u, mend - 1), c);
    }
    if (h == 1) __syncthreads();
    if (wm == h) {
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            et[(32 * i + 8 * (r >> 2) + 4 * lh + (r & 3)) * G::EPI_LD + wn * (TR / 4) + 32 * j + li] = acc[i][j][r];
    }
    __syncthreads();
    if (c >= g.N) continue;
    const bool whole = c + 8 <= g.N;
#pragma unroll
    for (int u = 0; u < NC; ++u) {
      const int rl = tid / CPR + (NT / CPR) * u, row = m0 + (TR / 2) * h + rl;
      if (row >= mend) continue;
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; j += 4) {
        const float4 q = *reinterpret_cast<const float4*>(et + rl * G::EPI_LD + cl + j);
        v[j] = q.x;
        v[j + 1] = q.y;
        v[j + 2] = q.z;
        v[j + 3] = q.w;
      }
      if (PROD == PROD_DW) {
        Raw8<float> o;
        narrow(v, o);
        float* out = dw + (int64_t)row * g.N + c;
        whole ? store8(out, o) : store8_part(out, o, g.N - c);
      } else {
        finish8<PROD, uint16_t>(g, step, row, c, bias, gate[u], v);
        Raw8<uint16_t> o;
        narrow(v, o);
        uint16_t* out = (uint16_t*)g.out + (int64_t)row * g.ldo + c;
        whole ? store8(out, o) : store8_part(out, o, g.N - c);
      }
    }
  }
  if (PROD == PROD_DW && sums && wn < NI) {
    // lanes lh = 0 and 1 hold the sums over the two halves of each slice
    const float tot = bsum + __shfl_xor(bsum, 32);
    const int o = m0 + wm * (TR / 2) + 32 * wn + li;
    if (lh == 0 && o < mend) dbias[o] = tot;
  }
}

// The tile of TR x TR at rows r0 .. rend-1, column n0 of expert e (FWD, DX).
template <int PROD, int TR, int WAY>
__device__ __forceinline__ void row_tile(const ProductArgs& g, int e, int r0, int rend, int n0, char* lds) {
  tile<PROD, TR, WAY>(g, e, r0, rend, n0, g.K, (const uint16_t*)g.a + r0 * g.lda,
                    (const uint16_t*)g.b + e * g.bstride + (PROD == PROD_FWD ? n0 * g.ldb : (int64_t)n0), nullptr, nullptr, lds);
}

// Workgroup `pid` of the row products (FWD, DX) in 256 x 256 tiles.  What does
// not fill the chip's last round, if that is at most half of it, goes as four
// tiles of 128 x 128 each: a small tile takes about 0.4 of a large one's
// time, so 32 tiles left over cost 0.4 of a round rather than a whole one
// (16108 rows of 8 experts, 2048 x 2048: 168 against 191 us).  Grid:
// row_blocks().
template <int PROD>
__device__ __forceinline__ void row_product(const ProductArgs& g, int pid, char* lds) {
  constexpr int TR = 256;
  RowTiles tiles;
  tiles.init(g, TR);
  const int tn = (g.N + TR - 1) / TR, total = tiles.total * tn;
  const int small = total % kCUs <= kCUs / 2 ? total % kCUs : 0;
  const int big = total - small;
  if (pid < big) {
    const int logical = xcd_remap(pid, big);
    const RowTile t = tiles.find(g, logical / tn);
    if (t.e >= 0) row_tile<PROD, TR, DIRECT>(g, t.e, t.r0, t.rend, (logical % tn) * TR, lds);
  } else if (pid < big + 4 * small) {
    const int q = xcd_remap(pid - big, 4 * small), logical = big + q / 4;
    const RowTile t = tiles.find(g, logical / tn);
    const int r0 = t.r0 + (q & 2 ? TR / 2 : 0), n0 = (logical % tn) * TR + (q & 1 ? TR / 2 : 0);
    if (t.e >= 0 && r0 < t.rend && n0 < g.N) row_tile<PROD, TR / 2, DIRECT>(g, t.e, r0, min(t.rend, r0 + TR / 2), n0, lds);
  }
}
int row_blocks(const ProductArgs& g) {
  return row_tiles_most(g, 256) * ((g.N + 255) / 256) + 3 * kCUs / 2;
}

template <int TR, int WAY>
__device__ __forceinline__ void weight_tile(const ProductArgs& g, int pid, char* lds) {
  const int tn = (g.N + TR - 1) / TR;
  const WeightTile w = weight_tile_of(g, pid, weight_tiles(g, TR, TR));
  if (w.e < 0) return;
  const int m0 = (w.t / tn) * TR, n0 = (w.t % tn) * TR;
  tile<PROD_DW, TR, WAY>(g, w.e, m0, g.M, n0, w.rows, (const uint16_t*)g.a + w.r0 * g.lda + m0,
                            (const uint16_t*)g.b + w.r0 * g.ldb + n0, w.out, w.dbias, lds);
}

template <int PROD>
__global__ __launch_bounds__(NT) void product_big_kernel(ProductArgs g) {
  __shared__ __attribute__((aligned(16))) char lds[Geo<256>::LDS];
  if (PROD == PROD_DW) return weight_tile<256, DIRECT>(g, blockIdx.x, lds);
  const int nblk = gridDim.x - kTailBlocks;
  if ((int)blockIdx.x >= nblk) return clear_rows<uint16_t, NT>(g, blockIdx.x - nblk);
  row_product<PROD>(g, blockIdx.x, lds);
}

// 128 x 128 tiles, two workgroups a CU
template <int PROD, int WAY>
__global__ __launch_bounds__(NT, 4) void product_mid_kernel(ProductArgs g) {
  constexpr int TR = 128;
  __shared__ __attribute__((aligned(16))) char lds[Geo<TR>::LDS];
  if (PROD == PROD_DW) return weight_tile<TR, WAY>(g, blockIdx.x, lds);
  const int nblk = gridDim.x - kTailBlocks;
  if ((int)blockIdx.x >= nblk) return clear_rows<uint16_t, NT>(g, blockIdx.x - nblk);
  RowTiles tiles;
  tiles.init(g, TR);
  const int tn = (g.N + TR - 1) / TR, total = tiles.total * tn;
  if ((int)blockIdx.x >= total) return;
  const int logical = xcd_remap(blockIdx.x, total);
  const RowTile t = tiles.find(g, logical / tn);
  if (t.e >= 0) row_tile<PROD, TR, WAY>(g, t.e, t.r0, t.rend, (logical % tn) * TR, lds);
}

template <int PROD, int WAY>
void launch_mid(const ProductArgs& g, hipStream_t s) {
  const int blocks = PROD == PROD_DW ? (int)weight_parts_most(g) * weight_tiles(g, 128, 128)
                                     : row_tiles_most(g, 128) * ((g.N + 127) / 128) + kTailBlocks;
  hipLaunchKernelGGL((product_mid_kernel<PROD, WAY>), dim3(blocks), dim3(NT), 0, s, g);
}

template <int PROD>
void launch(const ProductKernel& k, const ProductArgs& g, hipStream_t s) {
  if (k.way == WAY_STAGED) return launch_mid<PROD, STAGED>(g, s);
  if (k.way == WAY_TINY) return launch_mid<PROD, TINY>(g, s);
  if (k.tm == 128) return launch_mid<PROD, DIRECT>(g, s);
  const int blocks = PROD == PROD_DW ? (int)weight_parts_most(g) * weight_tiles(g, 256, 256) : row_blocks(g) + kTailBlocks;
  hipLaunchKernelGGL(product_big_kernel<PROD>, dim3(blocks), dim3(NT), 0, s, g);
}

}  // namespace

hipError_t launch_product_bf16(int prod, const ProductKernel& k, const ProductArgs& g, hipStream_t s) {
  if (prod == PROD_DW) launch<PROD_DW>(k, g, s);
  else if (prod == PROD_FWD) launch<PROD_FWD>(k, g, s);
  else launch<PROD_DX>(k, g, s);
  return hipGetLastError();
}

}  // namespace agn
