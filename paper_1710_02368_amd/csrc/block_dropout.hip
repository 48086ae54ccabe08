// Dropout with a mask that is drawn from (seed, step, row, column) and stored
// nowhere (agn_dropout), and the error text of the block operators.
#include <stdio.h>

#include <algorithm>

#include "block_common.h"

namespace agn {

static thread_local char g_block_err[512] = "";

int block_fail(int code, const char* fn, const char* what, const char* name) {
  snprintf(g_block_err, sizeof g_block_err, "%s: %s%s%s", fn, name ? name : "", name ? ": " : "", what);
  return code;
}
int block_launched(const char* fn) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? AGN_OK : block_fail(AGN_EHIP, fn, hipGetErrorString(e));
}

namespace {

// One Philox block gives the draws of eight elements, so a thread takes a
// chunk of eight columns of one row: one 16-byte load and store in bfloat16,
// two in float32.  `items` = rows of this launch x chunks a row < 2^31.
template <class T>
__global__ __launch_bounds__(256) void dropout_kernel(const T* x, int64_t ldx, T* out, int64_t ldo, int64_t row0,
                                                      uint32_t items, FastDiv chunks, int cols, MaskArgs m) {
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  if (i >= items) return;
  const uint32_t r = div_by(i, chunks), c8 = i - r * chunks.d;
  const int64_t row = row0 + r;
  const int c = (int)c8 * 8;
  Raw8<T> raw = load8_row(x + row * ldx, c, cols);
  if (m.thr) {
    float v[8];
    widen(raw, v);
    mask_apply(m, mask_step(m), row, c8, v);
    narrow(v, raw);
  }
  store8_row(out + row * ldo, c, cols, raw);
}

template <class T>
void launch(const agn_dropout_args& a, hipStream_t s) {
  const MaskArgs m = mask_args(a.mask);
  const uint32_t n8 = chunks_of(a.cols);
  const int64_t slab = std::max<int64_t>(1, ((INT64_C(1) << 31) - 1) / n8);  // rows a launch
  for (int64_t r = 0; r < a.rows; r += slab) {
    const uint32_t items = (uint32_t)(std::min(slab, a.rows - r) * n8);
    hipLaunchKernelGGL(dropout_kernel<T>, dim3((items + 255) / 256), dim3(256), 0, s, (const T*)a.x.p, a.x.ld,
                       (T*)a.out.p, a.out.ld, r, items, fast_div(n8), a.cols, m);
  }
}

}  // namespace
}  // namespace agn

using namespace agn;

extern "C" const char* agn_block_error(void) { return g_block_err; }

extern "C" int agn_dropout(const agn_dropout_args* a, void* stream) {
  const char* fn = "agn_dropout";
  AGN_BLOCK_REQUIRE(a, fn, "null arguments");
  AGN_BLOCK_REQUIRE(block_dtype_ok(a->dtype), fn, "dtype must be AGN_FP32 or AGN_BF16");
  AGN_BLOCK_REQUIRE(a->rows >= 0 && a->cols >= 0, fn, "negative size");
  AGN_BLOCK_REQUIRE(mask_threshold(a->mask.rate) >= 0, fn, "rate must be in [0, 1), below 1 - 2^-17");
  AGN_BLOCK_VECTOR(a->mask.step_dev, fn, "step_dev");
  AGN_BLOCK_ROWS(a->x, a->rows, a->cols, a->dtype, fn, "x");
  AGN_BLOCK_ROWS(a->out, a->rows, a->cols, a->dtype, fn, "out");
  if (a->rows == 0 || a->cols == 0) return AGN_OK;
  if (a->dtype == AGN_BF16)
    launch<uint16_t>(*a, (hipStream_t)stream);
  else
    launch<float>(*a, (hipStream_t)stream);
  return block_launched(fn);
}
