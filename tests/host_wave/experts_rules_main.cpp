// Prints the kernels that the experts' products of contiguous operands take
// (block_experts_rules.h).  Reads lines of "dtype rows experts inputs outputs";
// writes "forward | input gradient | weight gradient" for each.
#include <cstdio>

#include "block_experts_rules.h"

using namespace agn;

static void print(int prod, int dtype, ProductSizes g, bool direct) {
  const ProductKernel k = product_kernel(prod, dtype, g, direct);
  const bool parts = prod == PROD_DW && weight_part_rows(g, k) > 0;
  std::printf("%s%dx%d %s%s%s", k.few ? "few " : "", k.tm, k.tn,
              k.way == WAY_DIRECT ? "direct" : k.way == WAY_STAGED ? "staged" : "tiny", parts ? " parts" : "",
              prod == PROD_DW ? "\n" : "|");
}

int main() {
  int dtype, rows, experts, inputs, outputs;
  while (std::scanf("%d %d %d %d %d", &dtype, &rows, &experts, &inputs, &outputs) == 5) {
    const Copies f = copies(false, rows, experts, inputs, outputs, dtype), b = copies(true, rows, experts, inputs, outputs, dtype);
    const ProductSizes fwd{rows, experts, 0, outputs, inputs}, dx{rows, experts, 0, inputs, outputs},
        dw{rows, experts, outputs, inputs, 0};
    print(PROD_FWD, dtype, fwd, whole_chunks(PROD_FWD, fwd, f.x > 0, f.w > 0));
    print(PROD_DX, dtype, dx, whole_chunks(PROD_DX, dx, b.dy > 0, b.w > 0));
    print(PROD_DW, dtype, dw, whole_chunks(PROD_DW, dw, b.dy > 0, b.x > 0));
  }
  return 0;
}
