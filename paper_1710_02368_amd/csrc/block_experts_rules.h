// Which kernel an experts' product takes, by its sizes, type and operands'
// alignment, with the measurements that the rules go by.  Host arithmetic, no
// HIP.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "agn.h"

namespace agn {

enum { PROD_FWD = 0, PROD_DX = 1, PROD_DW = 2 };

struct ProductSizes {
  int rows, experts;
  int M, N, K;  // M: DW only; K: not DW
};

// How a tile's operands come: straight into LDS (bfloat16), through registers,
// or element by element where rows are shorter than a load.
enum { WAY_DIRECT, WAY_STAGED, WAY_TINY };

struct ProductKernel {
  bool few;    // the kernel for few rows (forward)
  int tm, tn;  // its tiles
  int way;
};

constexpr int kCUs = 256;

// most tiles of TR rows that the experts' rows make
inline int row_tiles_most(const ProductSizes& g, int TR) {
  return g.rows / TR + (g.experts < g.rows ? g.experts : g.rows);
}
// an expert's tiles of the weight gradient
constexpr int weight_tiles(const ProductSizes& g, int tm, int tn) {
  return ((g.M + tm - 1) / tm) * ((g.N + tn - 1) / tn);
}

// Where the few-rows kernel is taken (forward, us, it against the tiles' kernel):
//   bfloat16, up to 512 rows, where an estimate of its time is the shorter one:
//     it reads an expert's weights once for every 32 rows, at about 4.3 TB/s;
//     the 128 x 128 tiles read them once, and a tile's chain of K takes 0.8 us
//     a step of 64 however few they are.  Rows in equal parts are assumed.
//     5 rows to 5 of 18 experts, 3428 -> 1885: 16 : 46; 64 rows of 8, 2048 -> 2048
//     18 : 30, 256 rows 23 : 31, 512 rows 41 : 32; 64 rows of 4, 4096 -> 4096 34 :
//     55, 256 rows of one 67 : 56; 64 of 64, 1024 -> 1024 33 : 25; 512 of one, 1024
//     -> 512 7 : 13;
//   float32, up to 8 rows an expert (64 of 8, 2048 -> 2048: 33 : 50; 64 of 64, 1024
//     -> 1024: 63 : 96), up to 16 of at most 256 (128 of 8, 2048 -> 2048: 46 : 49; 64
//     of 4, 4096 -> 4096: 86 : 96), or where the 64 x 64 tiles are at most 96 (8
//     experts, 1024 -> 512: 256 rows 13 : 17; one, 1024 rows, 136 tiles, 25 : 17).
inline bool few_rows(int prod, int dtype, const ProductSizes& g) {
  // (a launch has fewer than 2^32 threads)
  if (prod != PROD_FWD || row_tiles_most(g, 16) * (int64_t)((g.N + 15) / 16) > 1 << 22) return false;
  if (dtype == AGN_BF16) {
    if (g.rows > 512) return false;
    // estimated us of this kernel and of the 128 x 128 tiles', two a CU
    const double used = std::min(g.experts, g.rows), weights = 2.0 * g.N * g.K;
    const double here = 4 + used * ((g.rows / g.experts + 31) / 32 + (g.rows < g.experts)) * weights / 4.3e6;
    const double rounds = std::ceil(row_tiles_most(g, 128) * (double)((g.N + 127) / 128) / 512);
    return here < 5 + std::max(rounds * g.K / 80, used * weights / 5.2e6);
  }
  return g.rows <= 8 * (int64_t)g.experts || (g.rows <= 16 * (int64_t)g.experts && g.rows <= 256) ||
         row_tiles_most(g, 64) * (int64_t)((g.N + 63) / 64) <= 96;
}

// every chunk of eight elements is a piece of one row (pad: rows go on with
// zeros to a multiple of eight)
inline bool whole_chunks(int prod, const ProductSizes& g, bool a_pad, bool b_pad) {
  return (a_pad || (prod == PROD_DW ? g.M : g.K) % 8 == 0) && (b_pad || (prod == PROD_FWD ? g.K : g.N) % 8 == 0);
}

// every operand's rows have eight elements
inline bool rows_of_eight(int prod, const ProductSizes& g) {
  return (prod == PROD_DW ? g.M : g.K) >= 8 && (prod == PROD_FWD || g.N >= 8);
}

// bfloat16: 256 x 256 tiles, or 128 x 128 where the matrix is narrow, rows are few for
// the number of experts (much of the larger tiles would be empty, or their
// stores outlast their sums) or tiles are few for the 256 CUs.  us, 256 against
// 128 (row products: tiles counted as row_tiles_most does):
//   forward: 16108 rows of 8 experts, 2048 -> 2048 (560 tiles) 157 : 190; 8192 of
//     8, 1536 -> 1536 (240) 48 : 56; 1024 -> 1024 (160) 34 : 34, its input gradient
//     32 : 35; 16000 of 8, 512 -> 512 (140) 24 : 17; 4096 of 8, 1024 -> 1024 (96)
//     30 : 21; 16108 of 64, 1024 -> 1024 75 : 61;
//   weight gradients: 16108 of 8, 2048 -> 2048 (512 tiles) 136 : 167; 8000 of 4,
//     2048 -> 2048 (256) 88 : 96; 4000 of 12, 1024 -> 1024 (192) 36 : 28; 4000 of 8,
//     1024 -> 512 (64) 33 : 25; 500 of 8, 256 -> 256 (8) 13 : 6; 16108 of 64, 1024 ->
//     1024 (252 rows an expert) 103 : 122; 4000 of 18 (222) 38 : 34; 4000 of 36
//     (111) 56 : 46.
inline bool big_tiles(int prod, const ProductSizes& g) {
  if (g.N < 256) return false;
  if (prod == PROD_DW)
    return g.M >= 256 && g.rows / g.experts >= 240 && g.experts * (int64_t)weight_tiles(g, 256, 256) >= kCUs;
  return g.rows / g.experts >= 512 && row_tiles_most(g, 256) * (int64_t)((g.N + 255) / 256) >= 144;
}

// float32: 128 x 128 tiles where there are many (a CU holds two: with few of
// them the last round is mostly empty)
inline bool large_tiles(int prod, const ProductSizes& g) {
  const int64_t tn = (g.N + 127) / 128;
  return (prod == PROD_DW ? (int64_t)g.experts * weight_tiles(g, 128, 128) : row_tiles_most(g, 128) * tn) >= 2048;
}

// float32: 64 x 32 rather than 64 x 64.  A half tile's step takes a little more
// than half a tile's, but more of them lie on a CU (three for two), with few
// tiles the CUs share them more evenly, and less of the edges is padding.  us,
// 64 x 64 against 64 x 32:
//   forward, input gradient: 3330 rows of 5 experts, 517 -> 259, 28.0 : 19.5;
//     2000 of 8, 1024 -> 1024, 67 : 61; 16000 of 8, 300 -> 300 (1290 tiles) 48 :
//     46; 12000 of 8, 512 -> 512 (1560 tiles) 73 : 76;
//   weight gradients, by an estimate that fits them, 20 a 64 x 64 tile a CU and
//     11 a half tile (in brackets tiles a CU, rounded up): 8192 rows of 8,
//     515 -> 515 (3 : 5 half) 80 : 69; 2048 of 2, 2048 -> 300 (2 : 3) 57 : 44; 12000
//     of 8, 512 -> 512 (2 : 4) 76 : 81; 1500 of 30, 700 -> 700 (15 : 29) 51 : 59;
//     where the 64 x 64 tiles are less than one a CU and would go in parts:
//     3330 of 5, 517 -> 259 (425 half tiles) 34 : 24; 6000 of 4, 256 -> 500 (256)
//     34 : 36.
inline bool narrow_tiles(int prod, const ProductSizes& g) {
  const int64_t t64 = prod == PROD_DW ? (int64_t)g.experts * weight_tiles(g, 64, 64)
                                      : row_tiles_most(g, 64) * (int64_t)((g.N + 63) / 64);
  if (prod != PROD_DW) return t64 < 1400;
  const int64_t t32 = (int64_t)g.experts * weight_tiles(g, 64, 32);
  return t64 < 256 ? t32 >= 320 : 11 * ((t32 + 255) / 256) < 20 * ((t64 + 255) / 256);
}

// The kernel of a product.  direct: whole_chunks, and all 16-byte aligned.
inline ProductKernel product_kernel(int prod, int dtype, const ProductSizes& g, bool direct) {
  if (few_rows(prod, dtype, g)) {
    // 16 rows x 16 columns a workgroup up to 16 rows, or 8 an expert, else 32 x 32
    const int t = g.rows <= 16 || g.rows <= 8 * (int64_t)g.experts ? 16 : 32;
    return {true, t, t, WAY_STAGED};
  }
  if (dtype == AGN_BF16) {
    const int t = direct && big_tiles(prod, g) ? 256 : 128;
    return {false, t, t, direct ? WAY_DIRECT : rows_of_eight(prod, g) ? WAY_STAGED : WAY_TINY};
  }
  const bool tiny = (prod == PROD_DW ? g.M : g.K) < 4 || (prod != PROD_FWD && g.N < 4);
  const int way = tiny ? WAY_TINY : WAY_STAGED;
  if (large_tiles(prod, g)) return {false, 128, 128, way};
  return {false, 64, narrow_tiles(prod, g) ? 32 : 64, way};
}

// Rows a part of the weight gradients' sums: none where the tiles fill the
// chip (then a part's float32 tile, written and read again, costs more than
// the better balance gives), else parts of at least 512 rows that fill it twice.
inline int weight_part_rows(const ProductSizes& g, const ProductKernel& k) {
  const int64_t per = weight_tiles(g, k.tm, k.tn), fill = k.tm == 256 || k.tn == 32 ? kCUs : 2 * kCUs;
  if (per * g.experts >= fill) return 0;
  const int64_t rows = std::max<int64_t>(512, (g.rows * per / (2 * fill) + 63) / 64 * 64);
  return g.rows > rows ? (int)rows : 0;
}

// Copies of bfloat16 operands whose width is no multiple of eight, so that the
// direct loads take them.  Without, 16-byte loads at any alignment go through
// registers into 128 x 128 tiles at 510 to 620 TFLOP/s, with them the products
// run at 800 to 1000.  They pay where the sums are long for what is copied (at
// about 4.5 TB/s); us without : with, copies included:
//   16108 rows of 8 experts, 2047 -> 2049: forward 270 : 228, input gradient 269 :
//     216, weight gradient 248 : 227 (either with its own copies); 12000 of 2,
//     4001 -> 1001: 174 : 150, 204 : 162, 175 : 181;
//   16108 of 8, 1001 -> 1003 forward 82 : 82 at the bound (not copied), 515 -> 1003
//     its gradients 55 : 55 and 70 : 73.
// Up to 1 GiB; an operand beyond is read as it is.
struct Copies {
  int64_t x, w, dy;  // bytes of each, 0: none
  int64_t total() const { return x + w + dy; }
};
inline Copies copies(bool grad, int64_t rows, int64_t experts, int64_t inputs, int64_t outputs, int dtype) {
  Copies c{};
  if (dtype != AGN_BF16 || rows / experts < 512 || inputs < 256 || outputs < 256) return c;
  const bool xw = inputs % 8, y = grad && outputs % 8;
  const int64_t ip = (inputs + 7) / 8 * 8, op = (outputs + 7) / 8 * 8;
  const double moved = (xw ? (double)(rows + experts * outputs) * inputs : 0) + (y ? (double)rows * outputs : 0);
  if (moved == 0 || (double)rows * inputs * outputs < (grad ? 400 : 800) * moved) return c;
  if (xw) {
    c.x = rows * ip * 2;
    c.w = experts * outputs * ip * 2;
  }
  if (y) c.dy = rows * op * 2;
  if (c.total() > (INT64_C(1) << 30)) return Copies{};
  return c;
}

}  // namespace agn
