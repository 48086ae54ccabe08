/*
 * agn_block.h -- operators of a residual block of experts on MI355X, next to
 * the MLP rounds of agn.h: dropout, the norms around a block with its gate
 * and residual scale, routing of rows to experts, the rows' way to their
 * experts and back, and the experts' products, each with its gradient.
 *
 * Conventions shared by every entry point:
 *   - Status codes and AGN_FP32 / AGN_BF16 are agn.h's.  Arguments are
 *     checked on the host before anything is enqueued (AGN_EINVAL, nothing
 *     written); agn_block_error() gives the message of the calling thread's
 *     last failure.  No C++ exception crosses the ABI.
 *   - The calls keep no state: no context, nothing kept from one call to the
 *     next.  They allocate nothing; where a call needs scratch memory, its
 *     _workspace function says how many bytes (-1 for bad arguments) and the
 *     caller passes a DEVICE buffer of at least that size, 16-byte aligned,
 *     whose contents before the call do not matter.
 *   - Work is enqueued on `stream` (a hipStream_t; NULL = null stream) of the
 *     current device; nothing waits for it, and every call can be captured
 *     into a graph.  The buffers must stay alive until the work has run.
 *   - DEVICE pointers throughout, except the argument structs themselves
 *     (HOST, read during the call).  Pointers are aligned to their element;
 *     more alignment is not needed.
 *   - agn_rows is a matrix of rows: element (r, c) at p[r * ld + c], of the
 *     call's `dtype` (float32 or bfloat16), ld >= columns.  ld is not looked
 *     at where a matrix has at most one row.  Sums, statistics and products
 *     are accumulated in float32; a bfloat16 output is rounded once, to
 *     nearest even.  Outputs must not overlap inputs unless a call says so.
 *   - Results do not depend on timing: the same inputs give the same bits
 *     (of the experts' products: with operands of the same alignment, which
 *     has a part in the choice of kernel).
 */
#ifndef AGN_BLOCK_H
#define AGN_BLOCK_H

#include "agn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  void* p;    /* DEVICE */
  int64_t ld; /* elements from one row to the next */
} agn_rows;

/* Message of the last failed call of this thread ("" if none).  Valid until
 * the thread's next failing call. */
const char* agn_block_error(void);

/* ---- dropout ------------------------------------------------------------ */

/* A random mask that is a function of its arguments and stored nowhere.
 * Element (r, c) belongs to the Philox4x32-10 block (Salmon, Moraes, Dror,
 * Shaw 2011) with counter (c / 8, r mod 2^32, r / 2^32, step) and key
 * (seed mod 2^32, seed / 2^32); its draw is the low (c even) or high (c odd)
 * 16 bits of output word (c mod 8) / 2.  The element is kept when the draw
 * is at least t = round(65536 rate), and multiplied by 65536 / (65536 - t):
 * the rate is held in steps of 1/65536 and the expectation is exact.  A
 * dropped element is 0 whatever it was (also an infinity or NaN).  `step`
 * counts the masks of one seed; where step_dev is not NULL its value at the
 * time the kernels run is added (mod 2^32), so that a captured graph draws
 * another mask in every replay.  rate in [0, 1) with t <= 65535; with t = 0
 * nothing is drawn. */
typedef struct {
  float rate;
  uint32_t step;
  uint64_t seed;
  const uint32_t* step_dev; /* DEVICE, or NULL */
} agn_mask;

typedef struct {
  int64_t rows;
  int32_t cols;
  int32_t dtype;
  agn_rows x;
  agn_rows out; /* may be x itself (the same p and ld) */
  agn_mask mask;
} agn_dropout_args;

/* out = mask * x.  The gradient is the same call on the output's gradient. */
int agn_dropout(const agn_dropout_args* a, void* stream);

/* ---- norms around a block ------------------------------------------------ */

#define AGN_GATE_NONE 0
#define AGN_GATE_CHANNEL 1 /* one float32 for each column                    */
#define AGN_GATE_FULL 2    /* rows x cols, of the call's dtype               */

#define AGN_NORMS_MAX_COLS 8192

/* What follows a block whose output is f, up to the next block's input h:
 *   u = norm(f) * w_post                 (u = f where w_post is NULL)
 *   residual' = residual + alpha * gate * mask * u
 *   h = norm(residual') * w_pre          (no h where w_pre is NULL)
 * row by row, with norm(v) = v / sqrt(mean(v^2) + eps), the squares summed in
 * float32 (a row whose sum passes its range has norm 0).  A dropped element
 * adds 0 whatever its gate and weight are, also in the gradients.  f.p NULL: there is
 * no block before (residual' = residual, and residual_out is not written);
 * then w_pre must be given.  h is computed from the float32 residual'. */
typedef struct {
  int64_t rows;
  int32_t cols; /* 1 .. AGN_NORMS_MAX_COLS                                   */
  int32_t dtype;
  float eps;   /* >= 0, finite                                               */
  float alpha; /* finite                                                     */
  int32_t gate_kind;
  agn_rows residual;
  agn_rows f;
  agn_rows gate;       /* AGN_GATE_CHANNEL: p is cols floats, ld not used    */
  const float* w_post; /* cols floats or NULL                                */
  const float* w_pre;  /* cols floats or NULL                                */
  agn_mask mask;
  agn_rows residual_out; /* may be `residual` itself                         */
  agn_rows h;
  float* rstd_post; /* rows floats or NULL: 1 / sqrt(mean(f^2) + eps)        */
  float* rstd_pre;  /* rows floats or NULL: the same of residual'            */
} agn_norms_args;

int agn_norms(const agn_norms_args* a, void* stream);

/* Gradient of agn_norms.  `fwd` holds the forward call's f, gate, weights,
 * mask and numbers, and both rstd of the forward call as inputs here
 * (rstd_post only with w_post, rstd_pre only with w_pre; h is not looked
 * at).  With w_pre it also holds one of
 *   residual: the forward call's; residual' is computed again in float32;
 *   residual_out, with residual.p NULL: what the forward call stored, for
 *     callers that overwrote residual.  In bfloat16 that is residual'
 *     rounded, and so off by up to 2^-9 of it in the gradients.
 * (Without f the two are the same, and `residual` is given.)
 *   dresidual_out: gradient of residual' from above, p NULL = 0
 *   dh:            gradient of h (only with w_pre)
 *   dresidual:     out: gradient of residual; may be dresidual_out itself
 *   df:            out: gradient of f (only with f)
 *   dgate:         out: AGN_GATE_CHANNEL: cols floats; AGN_GATE_FULL: rows of
 *                  the call's dtype
 *   dw_post, dw_pre: out, cols floats (only with the weight)
 * The sums over rows (dw_post, dw_pre, a channel gate's dgate) are taken in
 * a fixed order; with rows = 0 they are zero. */
typedef struct {
  agn_norms_args fwd;
  agn_rows dresidual_out;
  agn_rows dh;
  agn_rows dresidual;
  agn_rows df;
  agn_rows dgate;
  float* dw_post;
  float* dw_pre;
  void* workspace;
  int64_t workspace_bytes;
} agn_norms_grad_args;

int64_t agn_norms_backward_workspace(int64_t rows, int32_t cols);
int agn_norms_backward(const agn_norms_grad_args* a, void* stream);

/* ---- routing -------------------------------------------------------------- */

#define AGN_ROUTE_MAX_EXPERTS 1024
#define AGN_ROUTE_MAX_K 16

/* Each of `rows` rows goes to up to k of `experts` experts.
 *   logits: rows x experts of `dtype`.  The k largest of a row, in falling
 *     order, ties by the lower index, a NaN above every number; -inf is never
 *     chosen, so a row may have fewer than k experts, or none.
 *   chosen: rows x k int32, the experts, -1 where there is none.
 *   weights: rows x k floats: exp(l - max) over the sum of the same over the
 *     chosen (over_all 0) or over all experts (over_all 1); 0 where there is
 *     none.
 * With logits.p NULL, `chosen` is an input (an expert outside [0, experts)
 * counts as none) and `weights` is not looked at.  Then the rows' choices are
 * sorted by expert, stably; pair p = row * k + j is choice j of a row:
 *   offsets: experts + 1 int32: expert e's pairs are sorted places
 *     offsets[e] .. offsets[e + 1] - 1;
 *   source: rows * k int32: the pair at each sorted place, -1 from
 *     offsets[experts] on;
 *   slot: rows * k int32: each pair's sorted place, -1 for none.
 * rows * k < 2^31; k <= experts. */
typedef struct {
  int64_t rows;
  int32_t experts;
  int32_t k;
  int32_t dtype;
  int32_t over_all;
  agn_rows logits;
  int32_t* chosen;
  float* weights;
  int32_t* offsets;
  int32_t* source;
  int32_t* slot;
  void* workspace;
  int64_t workspace_bytes;
} agn_route_args;

int64_t agn_route_workspace(int64_t rows, int32_t experts, int32_t k);
int agn_route(const agn_route_args* a, void* stream);

/* Gradient of the weights with respect to the logits (the choice itself is
 * taken as fixed), chosen and weights being what agn_route made of these
 * logits: with w the weights and g their gradient, s = sum_j w_j g_j,
 *   over_all 0: dlogits = w_j (g_j - s) at the chosen, 0 elsewhere;
 *   over_all 1: dlogits = p_e (g_e - s), p the softmax over all experts and
 *     g_e = 0 where e is not chosen. */
typedef struct {
  int64_t rows;
  int32_t experts;
  int32_t k;
  int32_t dtype; /* of logits and dlogits */
  int32_t over_all;
  agn_rows logits; /* looked at only with over_all 1 */
  const int32_t* chosen;
  const float* weights;
  const float* dweights; /* rows x k floats */
  agn_rows dlogits;      /* out, rows x experts; every element is written */
} agn_route_grad_args;

int agn_route_backward(const agn_route_grad_args* a, void* stream);

/* ---- rows to their experts and back --------------------------------------- */

/* The plan is agn_route's: slot (rows * k) and its count of places in use,
 * total = &offsets[experts].  x has `rows` rows, y rows * k (sorted by
 * expert).
 *   agn_dispatch:  y[slot[t, j]] = x[t]; rows of y from *total on are zero.
 *   agn_combine:   x[t] = sum_j w[t, j] y[slot[t, j]] over the pairs that
 *     have a place, in the order of j; zero where none has.  weights NULL:
 *     all 1, the gradient of agn_dispatch.
 *   agn_combine_backward: from x = the gradient of agn_combine's output,
 *     dy[slot[t, j]] = w[t, j] x[t] (rows from *total on are zero) and
 *     dweights[t, j] = sum_c x[t, c] y[slot[t, j], c], 0 without a place.
 * A slot outside [0, rows * k) counts as none. */
typedef struct {
  int64_t rows;
  int32_t cols;
  int32_t k;
  int32_t dtype;
  const int32_t* slot;
  const int32_t* total;
  const float* weights; /* rows x k floats (agn_combine: or NULL; agn_dispatch: not looked at) */
  agn_rows x;
  agn_rows y;
  agn_rows dy;     /* agn_combine_backward only */
  float* dweights; /* agn_combine_backward only */
} agn_tokens_args;

int agn_dispatch(const agn_tokens_args* a, void* stream);
int agn_combine(const agn_tokens_args* a, void* stream);
int agn_combine_backward(const agn_tokens_args* a, void* stream);

/* ---- the experts' products ------------------------------------------------- */

#define AGN_EXPERTS_MAX 1024

/* Rows sorted by expert times their expert's weights.  Expert e's rows are
 * offsets[e] .. offsets[e + 1] - 1 (DEVICE; the offsets rise from 0 to at
 * most `rows`), w_e is outputs x inputs at w.p + e * outputs * w.ld with row
 * stride w.ld, bias (experts x outputs floats, or NULL).
 *   out[r] = mask * act(x[r] w_e^T + bias_e), act = relu or none; rows from
 *   offsets[experts] on are zero.  The mask is that of `out`'s elements
 *   (r, c).  float32 products are float32 MFMAs, bfloat16 ones accumulate
 *   in float32. */
typedef struct {
  int64_t rows; /* (rows / 128 + experts) (columns / 128 + 1) <= 2^22, columns
                   the larger of inputs and outputs, and experts (inputs / 128
                   + 1) (outputs / 128 + 1) <= 2^22, each / rounded down */
  int32_t experts;
  int32_t inputs;
  int32_t outputs;
  int32_t dtype; /* of x, w, out */
  int32_t relu;
  const int32_t* offsets;
  agn_rows x;
  agn_rows w;
  const float* bias;
  agn_mask mask;
  agn_rows out;
  void* workspace;
  int64_t workspace_bytes;
} agn_experts_args;

int64_t agn_experts_workspace(int64_t rows, int32_t experts, int32_t inputs, int32_t outputs, int32_t dtype);
int agn_experts(const agn_experts_args* a, void* stream);

/* Gradient of agn_experts, dy being the gradient of x w_e^T + bias_e (of the
 * output with its ReLU and mask taken off: where the next layer's call below
 * gave dx with relu_input, that is dx itself).
 *   dx[r] = dy[r] w_e, rows from offsets[experts] on zero.  relu_input 1: x
 *     is the output of a ReLU with a mask of rate input_rate, and dx is
 *     multiplied by [x > 0] * 65536 / (65536 - t), t = round(65536
 *     input_rate): the gradient of the sums before that ReLU.
 *   dw (experts x outputs x inputs floats, contiguous) = dy^T x over the
 *     expert's rows, zero for an expert without rows; dbias (experts x
 *     outputs floats) = the sums of dy over the expert's rows (in an order that
 *     depends on whether dw is wanted too).
 * Each of dx.p, dw, dbias may be NULL: not wanted. */
typedef struct {
  int64_t rows;
  int32_t experts;
  int32_t inputs;
  int32_t outputs;
  int32_t dtype;
  int32_t relu_input;
  float input_rate;
  const int32_t* offsets;
  agn_rows x;
  agn_rows dy;
  agn_rows w;
  agn_rows dx;
  float* dw;
  float* dbias;
  void* workspace;
  int64_t workspace_bytes;
} agn_experts_grad_args;

int64_t agn_experts_backward_workspace(int64_t rows, int32_t experts, int32_t inputs, int32_t outputs, int32_t dtype);
int agn_experts_backward(const agn_experts_grad_args* a, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* AGN_BLOCK_H */
