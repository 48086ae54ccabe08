// The experts' products (agn_experts, agn_experts_backward): arguments,
// launches and the bias gradients.
#include <algorithm>

#include "block_experts.h"

namespace agn {
namespace {

// dbias alone (where dw is wanted too, its product's first column of tiles
// sums what it reads): a workgroup takes 64 columns of one expert, a thread
// eight columns of every 32nd row, and the 32 sums are added in order.
template <class T>
__global__ __launch_bounds__(256) void bias_grad_kernel(ProductArgs g) {
  __shared__ float sh[32][65];
  const int tn = (g.M + 63) / 64;
  const int e = blockIdx.x / tn, x = threadIdx.x & 7, y = threadIdx.x >> 3, c0 = (blockIdx.x % tn) * 64, c = c0 + 8 * x;
  const int b = clamped_offset(g, e), end = clamped_offset(g, e + 1);
  float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (c < g.M) {
#pragma unroll 4
    for (int r = b + y; r < end; r += 32) {
      float v[8];
      widen(load8_row((const T*)g.a + r * g.lda, c, g.M), v);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] += v[j];
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) sh[y][8 * x + j] = s[j];
  __syncthreads();
  if (threadIdx.x < 64 && c0 + (int)threadIdx.x < g.M) {
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) v += sh[i][threadIdx.x];
    g.dbias[(int64_t)e * g.M + c0 + threadIdx.x] = v;
  }
}

// dw (and dbias) of the experts whose rows were summed in several parts, or
// that have none: the parts' sums added in order, or zeros.  A workgroup
// takes 1024 elements of one expert.
__global__ __launch_bounds__(256) void sum_weight_parts_kernel(ProductArgs g, int per) {
  const int e = blockIdx.x / per;
  const int64_t size = (int64_t)g.M * g.N;
  // the expert's parts: q .. q + n - 1
  const int lane = threadIdx.x & 63;
  int q = 0, n = 0;
  for (int e0 = 0; e0 < g.experts; e0 += 64) {
    const int i = e0 + lane;
    int c = 0;
    if (i < g.experts) c = (max(0, clamped_offset(g, i + 1) - clamped_offset(g, i)) + g.part_rows - 1) / g.part_rows;
    int before = i < e ? c : 0;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) before += __shfl_xor(before, d);
    q += before;
    if (e >= e0 && e < e0 + 64) n = __shfl(c, e - e0);
  }
  if (n == 1 || q + n > g.parts_most) return;  // (the latter: offsets that do not rise)
  const float* parts = g.parts + q * size;
  float* out = (float*)g.out + e * size;
  for (int64_t i = (int64_t)(blockIdx.x % per) * 1024 + threadIdx.x, end = min(i + 1024, size); i < end; i += 256) {
    float s = 0.f;
#pragma unroll 4
    for (int p = 0; p < n; ++p) s += parts[p * size + i];
    out[i] = s;
  }
  if (g.dbias)
    for (int i = (blockIdx.x % per) * 256 + threadIdx.x; i < g.M; i += per * 256) {
      float s = 0.f;
      for (int p = 0; p < n; ++p) s += g.parts_bias[(int64_t)(q + p) * g.M + i];
      g.dbias[(int64_t)e * g.M + i] = s;
    }
}

// Rows copied with zeros up to a multiple of eight columns, a wave a row.
__global__ __launch_bounds__(256) void pad_rows_kernel(const uint16_t* src, int64_t ld, int64_t rows, int cols,
                                                       uint16_t* dst, int64_t ldp) {
  for (int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); r < rows; r += (int64_t)gridDim.x * 4)
    for (int c = 8 * (threadIdx.x & 63); c < cols; c += 512) store8(dst + r * ldp + c, load8_row(src + r * ld, c, cols));
}
void pad_rows(const agn_rows& m, int64_t rows, int cols, const agn_rows& out, hipStream_t s) {
  hipLaunchKernelGGL(pad_rows_kernel, dim3((uint32_t)std::min<int64_t>((rows + 3) / 4, 16384)), dim3(256), 0, s,
                     (const uint16_t*)m.p, m.ld, rows, cols, (uint16_t*)out.p, out.ld);
}

// what a product reads: the operand, or its copy at `at` of so many bytes
agn_rows operand(const agn_rows& m, int64_t bytes, int cols, char* at) {
  return bytes ? agn_rows{at, (cols + 7) / 8 * 8} : m;
}

const char* sizes_error(int64_t rows, int32_t experts, int32_t inputs, int32_t outputs, int32_t dtype) {
  if (!block_dtype_ok(dtype)) return "dtype must be AGN_FP32 or AGN_BF16";
  if (rows < 0 || rows >= (INT64_C(1) << 31)) return "rows must be in [0, 2^31)";
  if (experts < 1 || experts > AGN_EXPERTS_MAX) return "experts must be in [1, AGN_EXPERTS_MAX]";
  if (inputs < 1 || outputs < 1 || inputs > (1 << 24) || outputs > (1 << 24)) return "inputs and outputs must be in [1, 2^24]";
  // A launch has fewer than 2^32 threads: at most 2^22 tiles of 128 x 128,
  // 512 threads each (64 x 64 ones are taken for fewer than 2^13 of these).
  // 2^22 tiles of bfloat16 outputs are 128 GiB.
  const int64_t ti = inputs / 128 + 1, to = outputs / 128 + 1;
  if ((rows / 128 + experts) * std::max(ti, to) > (1 << 22) || ti * to * experts > (1 << 22)) return "problem too large";
  return nullptr;
}

const char* weights_error(const agn_rows& w, int32_t experts, int32_t inputs, int32_t outputs, int32_t dtype) {
  return rows_error(w, (int64_t)experts * outputs, inputs, dtype);
}

hipError_t product(int prod, const ProductKernel& k, int dtype, const ProductArgs& g, hipStream_t s) {
  if (k.few) return launch_product_few(k, dtype, g, s);
  return dtype == AGN_BF16 ? launch_product_bf16(prod, k, g, s) : launch_product_f32(prod, k, g, s);
}
ProductKernel kernel_of(int prod, int dtype, const ProductArgs& g) {
  return product_kernel(prod, dtype, g, direct_ok(prod, g));
}

}  // namespace
}  // namespace agn

using namespace agn;

extern "C" int64_t agn_experts_workspace(int64_t rows, int32_t experts, int32_t inputs, int32_t outputs, int32_t dtype) {
  if (const char* e = sizes_error(rows, experts, inputs, outputs, dtype)) {
    block_fail(AGN_EINVAL, "agn_experts_workspace", e);
    return -1;
  }
  return copies(false, rows, experts, inputs, outputs, dtype).total();
}

extern "C" int64_t agn_experts_backward_workspace(int64_t rows, int32_t experts, int32_t inputs, int32_t outputs,
                                                  int32_t dtype) {
  if (const char* e = sizes_error(rows, experts, inputs, outputs, dtype)) {
    block_fail(AGN_EINVAL, "agn_experts_backward_workspace", e);
    return -1;
  }
  // (whatever the operands' alignment: the larger of both kinds of tiles' needs)
  const Copies c = copies(true, rows, experts, inputs, outputs, dtype);
  int64_t need = 0;
  for (int aligned = 0; aligned < 2; ++aligned) {
    ProductArgs g{};
    g.rows = (int)rows;
    g.experts = experts;
    g.M = outputs;
    g.N = inputs;
    const bool direct = aligned && whole_chunks(PROD_DW, g, c.dy > 0, c.x > 0);
    g.part_rows = weight_part_rows(g, product_kernel(PROD_DW, dtype, g, direct));
    if (g.part_rows) need = std::max(need, weight_parts_most(g) * ((int64_t)outputs * inputs + outputs) * (int64_t)sizeof(float));
  }
  return c.total() + need;
}

extern "C" int agn_experts(const agn_experts_args* a, void* stream) {
  const char* fn = "agn_experts";
  AGN_BLOCK_REQUIRE(a, fn, "null arguments");
  if (const char* e = sizes_error(a->rows, a->experts, a->inputs, a->outputs, a->dtype)) return block_fail(AGN_EINVAL, fn, e);
  AGN_BLOCK_REQUIRE(a->relu == 0 || a->relu == 1, fn, "relu must be 0 or 1");
  AGN_BLOCK_REQUIRE(mask_threshold(a->mask.rate) >= 0, fn, "rate must be in [0, 1), below 1 - 2^-17");
  AGN_BLOCK_REQUIRE(element_aligned(a->bias, AGN_FP32), fn, "bias not aligned to its element");
  AGN_BLOCK_VECTOR(a->mask.step_dev, fn, "step_dev");
  AGN_BLOCK_VECTOR(a->offsets, fn, "offsets");
  AGN_BLOCK_ROWS(a->x, a->rows, a->inputs, a->dtype, fn, "x");
  AGN_BLOCK_ROWS(a->out, a->rows, a->outputs, a->dtype, fn, "out");
  if (a->rows == 0) return AGN_OK;
  AGN_BLOCK_REQUIRE(a->offsets, fn, "null offsets");
  if (const char* e = weights_error(a->w, a->experts, a->inputs, a->outputs, a->dtype))
    return block_fail(AGN_EINVAL, fn, e, "w");
  const Copies cp = copies(false, a->rows, a->experts, a->inputs, a->outputs, a->dtype);
  AGN_BLOCK_REQUIRE(!cp.total() || (a->workspace && ((uintptr_t)a->workspace & 15) == 0 && a->workspace_bytes >= cp.total()),
                    fn, "workspace missing, unaligned or too small");
  char* ws = (char*)a->workspace;
  const agn_rows x = operand(a->x, cp.x, a->inputs, ws), w = operand(a->w, cp.w, a->inputs, ws + cp.x);
  if (cp.x) pad_rows(a->x, a->rows, a->inputs, x, (hipStream_t)stream);
  if (cp.w) pad_rows(a->w, (int64_t)a->experts * a->outputs, a->inputs, w, (hipStream_t)stream);
  ProductArgs g{};
  g.a_pad = cp.x > 0;
  g.b_pad = cp.w > 0;
  g.a = x.p;
  g.lda = x.ld;
  g.b = w.p;
  g.ldb = w.ld;
  g.bstride = a->outputs * w.ld;
  g.rows = (int)a->rows;
  g.experts = a->experts;
  g.N = a->outputs;
  g.K = a->inputs;
  g.offsets = a->offsets;
  g.out = a->out.p;
  g.ldo = a->out.ld;
  g.bias = a->bias;
  g.relu = a->relu;
  g.mask = mask_args(a->mask);
  const hipError_t e = product(PROD_FWD, kernel_of(PROD_FWD, a->dtype, g), a->dtype, g, (hipStream_t)stream);
  return e == hipSuccess ? AGN_OK : block_fail(AGN_EHIP, fn, hipGetErrorString(e));
}

extern "C" int agn_experts_backward(const agn_experts_grad_args* a, void* stream) {
  const char* fn = "agn_experts_backward";
  AGN_BLOCK_REQUIRE(a, fn, "null arguments");
  if (const char* e = sizes_error(a->rows, a->experts, a->inputs, a->outputs, a->dtype)) return block_fail(AGN_EINVAL, fn, e);
  AGN_BLOCK_REQUIRE(a->relu_input == 0 || a->relu_input == 1, fn, "relu_input must be 0 or 1");
  AGN_BLOCK_REQUIRE(mask_threshold(a->input_rate) >= 0, fn, "input_rate must be in [0, 1), below 1 - 2^-17");
  AGN_BLOCK_REQUIRE(element_aligned(a->dw, AGN_FP32) && element_aligned(a->dbias, AGN_FP32), fn,
                    "dw or dbias not aligned to its element");
  AGN_BLOCK_REQUIRE(a->offsets, fn, "null offsets");
  AGN_BLOCK_VECTOR(a->offsets, fn, "offsets");
  AGN_BLOCK_ROWS(a->dy, a->rows, a->outputs, a->dtype, fn, "dy");
  if (a->dw || a->relu_input) AGN_BLOCK_ROWS(a->x, a->rows, a->inputs, a->dtype, fn, "x");
  if (a->dx.p && a->rows > 0) {
    AGN_BLOCK_ROWS(a->dx, a->rows, a->inputs, a->dtype, fn, "dx");
    if (const char* e = weights_error(a->w, a->experts, a->inputs, a->outputs, a->dtype))
      return block_fail(AGN_EINVAL, fn, e, "w");
  }
  const hipStream_t s = (hipStream_t)stream;
  const bool want_dx = a->dx.p && a->rows > 0;
  // which operands are copied goes by the sizes alone, so that the bits of dx
  // and dw do not depend on which others are wanted (dbias has an order of
  // summation of its own where dw is not)
  const Copies cp = copies(true, a->rows, a->experts, a->inputs, a->outputs, a->dtype);
  char* ws = (char*)a->workspace;  // the copies of dy, x and w, then the parts
  const agn_rows dy = operand(a->dy, cp.dy, a->outputs, ws), x = operand(a->x, cp.x, a->inputs, ws + cp.dy),
                 w = operand(a->w, cp.w, a->inputs, ws + cp.dy + cp.x);
  ProductArgs g{};
  g.a = dy.p;
  g.lda = dy.ld;
  g.a_pad = cp.dy > 0;
  g.rows = (int)a->rows;
  g.experts = a->experts;
  g.offsets = a->offsets;
  ProductArgs dx = g, dw = g;
  dx.b = w.p;
  dx.ldb = w.ld;
  dx.b_pad = cp.w > 0;
  dx.bstride = a->outputs * w.ld;
  dx.N = a->inputs;
  dx.K = a->outputs;
  dx.out = a->dx.p;
  dx.ldo = a->dx.ld;
  if (a->relu_input) {
    dx.gate = a->x.p;
    dx.ldgate = a->x.ld;
    dx.gate_scale = 65536.f / (float)(65536 - mask_threshold(a->input_rate));
  }
  dw.b = x.p;
  dw.ldb = x.ld;
  dw.b_pad = cp.x > 0;
  dw.M = a->outputs;
  dw.N = a->inputs;
  dw.out = a->dw;
  dw.ldo = a->inputs;
  dw.dbias = a->dbias;
  int64_t need = want_dx || a->dw ? cp.total() : 0;
  const ProductKernel dw_kernel = kernel_of(PROD_DW, a->dtype, dw);
  if (a->dw) {
    dw.part_rows = weight_part_rows(dw, dw_kernel);
    if (dw.part_rows) {
      const int64_t parts = weight_parts_most(dw);
      need += parts * ((int64_t)dw.M * dw.N + dw.M) * (int64_t)sizeof(float);
      dw.parts_most = (int)parts;
      dw.parts = (float*)(ws + cp.total());
      dw.parts_bias = dw.parts + parts * dw.M * dw.N;
    }
  }
  AGN_BLOCK_REQUIRE(need == 0 || (ws && ((uintptr_t)ws & 15) == 0 && a->workspace_bytes >= need), fn,
                    "workspace missing, unaligned or too small");
  if (cp.dy && need) pad_rows(a->dy, a->rows, a->outputs, dy, s);
  if (cp.x && a->dw) pad_rows(a->x, a->rows, a->inputs, x, s);
  if (cp.w && want_dx) pad_rows(a->w, (int64_t)a->experts * a->outputs, a->inputs, w, s);
  hipError_t e = hipSuccess;
  if (want_dx) e = product(PROD_DX, kernel_of(PROD_DX, a->dtype, dx), a->dtype, dx, s);
  if (e == hipSuccess && a->dw) e = product(PROD_DW, dw_kernel, a->dtype, dw, s);
  if (e == hipSuccess && a->dw && dw.part_rows) {
    const int per = (int)(((int64_t)dw.M * dw.N + 1023) / 1024);
    hipLaunchKernelGGL(sum_weight_parts_kernel, dim3(dw.experts * per), dim3(256), 0, s, dw, per);
    e = hipGetLastError();
  }
  if (e == hipSuccess && a->dbias && !a->dw) {
    g.a = a->dy.p;
    g.lda = a->dy.ld;
    g.M = a->outputs;
    g.dbias = a->dbias;
    const dim3 grid(a->experts * ((a->outputs + 63) / 64));
    if (a->dtype == AGN_BF16)
      hipLaunchKernelGGL(bias_grad_kernel<uint16_t>, grid, dim3(256), 0, s, g);
    else
      hipLaunchKernelGGL(bias_grad_kernel<float>, grid, dim3(256), 0, s, g);
    e = hipGetLastError();
  }
  return e == hipSuccess ? AGN_OK : block_fail(AGN_EHIP, fn, hipGetErrorString(e));
}
