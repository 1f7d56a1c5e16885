/*
 * cada_ops.h - C ABI of libcada's operators for networks of one's own: a layer's product with
 *              bias, activation and residual, its gradients, layer norm with its gradients, the
 *              embedding lookup with its gradient, the softmax cross-entropy with its gradient, of
 *              given logits or of a last layer's product, and the AdamW step over many tensors.
 *
 * The engine of cada.h trains the models that it knows.  With these a program trains and serves
 * any network of such layers by the plain (everybody uploads) Adam baseline, on the same device
 * memory and streams, and with the same parameter layout: a weight matrix is row-major [in, out].
 *
 * Conventions, as in cada.h
 *   - Pointers are DEVICE memory owned by the caller unless marked HOST.  The library allocates no
 *     device memory; what a call needs beyond its operands is a workspace (256-byte aligned).  The
 *     operator's ..._workspace() function checks the arguments that it names and writes the size
 *     into workspace_bytes; 0 means that none is needed (workspace may be NULL).  A workspace holds
 *     nothing between calls, and calls that may overlap (different streams) need one each.
 *   - Calls enqueue work on the given stream and never synchronise the host; operands and
 *     workspace must stay valid until that work has completed.  They record no memset or copy node
 *     and may be captured into a HIP graph (cada_adamw_init copies a table from the host and may
 *     not; a captured cada_adamw_step repeats its t and lr).
 *   - Tables have rows of contiguous elements, ld... elements apart (ld >= the row's length).
 *     Element alignment is enough; rows that start on 16-byte boundaries and have a multiple of 16
 *     bytes are faster.  Outputs share memory with no operand except where it says so, and the
 *     workspace with neither (CADA_EINVAL; columns side by side in one wider table are apart, and a
 *     single row is beside a wider table's columns).
 *   - Sums, statistics and moments are formed in float32 or more; values are rounded to nearest
 *     even where they are written as bf16.
 *   - Results do not depend on timing: the same call on the same operands gives the same bits.
 *   - Every function returns 0 or a negative CADA_E* code with the text in cada_last_error().
 */
#ifndef CADA_OPS_H
#define CADA_OPS_H

#include "cada.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { CADA_F32 = 0, CADA_BF16 = 1 }; /* element types */
enum {
  CADA_ACT_NONE = 0,
  CADA_ACT_RELU = 1, /* derivative 0 at 0 */
  CADA_ACT_GELU = 2, /* z Phi(z), Phi the normal distribution function */
  CADA_ACT_SILU = 3  /* z / (1 + exp(-z)) */
};

/* y = act(x w + bias) + residual, and on request pre = x w + bias, which the gradient of every
 * activation but CADA_ACT_NONE reads.  All tables and the bias are of one type; each output element is
 * formed in float32 and rounded once. */
typedef struct cada_linear {
  int64_t rows;         /* >= 0 (0: nothing to do) */
  int64_t in, out;      /* 1 .. CADA_MAX_WIDTH; of the tables' products, at most 2^23 - 8 tiles of 64 x 64 */
  int32_t type;         /* CADA_F32 or CADA_BF16 */
  int32_t act;          /* CADA_ACT_* */
  const void *x;        /* [rows, in] */
  int64_t ldx;
  const void *w;        /* [in, out] */
  int64_t ldw;
  const void *bias;     /* [out] or NULL */
  const void *residual; /* [rows, out] or NULL; may be y itself */
  int64_t ldr;
  void *y;              /* [rows, out] */
  int64_t ldy;
  void *pre;            /* [rows, out] or NULL */
  int64_t ldpre;
  void *workspace;
  size_t workspace_bytes;
  void *stream;         /* hipStream_t; NULL = the default stream */
} cada_linear;
#define CADA_MAX_WIDTH (1 << 24)

int cada_linear_forward_workspace(cada_linear *a); /* all but the pointers' contents, y, pre and stream is read */
int cada_linear_forward(const cada_linear *a);

/* Gradients of a layer: with dz = dy * act'(pre), dx = dz w^T, dw = x^T dz, db = column sums of
 * dz; the residual's gradient is dy.  Outputs that are NULL are not formed.  With bf16 tables dz is rounded to bf16
 * before the two products (their operands are bf16), not for db. */
typedef struct cada_linear_grad {
  int64_t rows, in, out; /* as above; rows == 0 clears dw and db */
  int32_t type, act;
  const void *dy;        /* [rows, out] */
  int64_t lddy;
  const void *x;         /* [rows, in]; not read unless dw is wanted */
  int64_t ldx;
  const void *w;         /* [in, out]; not read unless dx is wanted */
  int64_t ldw;
  const void *pre;       /* [rows, out]; not read with CADA_ACT_NONE */
  int64_t ldpre;
  void *dx;              /* [rows, in] or NULL */
  int64_t lddx;
  void *dw;              /* [in, out] or NULL */
  int64_t lddw;
  void *db;              /* [out] or NULL */
  void *workspace;
  size_t workspace_bytes;
  void *stream;
} cada_linear_grad;

int cada_linear_backward_workspace(cada_linear_grad *a); /* all but the pointers' contents and stream is read */
int cada_linear_backward(const cada_linear_grad *a);

/* Layer norm of the rows of a table.
 *   mean = sum x / width,  rstd = 1 / sqrt(sum (x - mean)^2 / width + eps),  y = (x - mean) rstd weight + bias
 * mean and rstd are in float32; y is formed in float32 and rounded once. */
typedef struct cada_norm {
  int64_t rows;         /* 0 .. 2^40 */
  int64_t width;        /* 1 .. CADA_MAX_WIDTH */
  int32_t type;         /* of all but the statistics */
  double eps;           /* positive, also in float32 */
  const void *x;        /* [rows, width] */
  int64_t ldx;
  const void *weight;   /* [width] or NULL (1) */
  const void *bias;     /* [width] or NULL (0) */
  void *y;              /* [rows, width]; may be x itself (then with its ld) */
  int64_t ldy;
  float *mean, *rstd;   /* [rows] or NULL: what the gradient reads */
  void *stream;
} cada_norm;

int cada_layer_norm_forward(const cada_norm *a); /* needs no workspace */

/* Its gradients.  With u = (x - mean) rstd and g = dy weight:
 *   dx = rstd (g - sum g / width - u (sum g u) / width) + residual,  dw = sum over the rows of dy u,  db = of dy
 * (residual: a gradient that comes around the layer).  Outputs that are NULL are not formed. */
typedef struct cada_norm_grad {
  int64_t rows, width;  /* as above; rows == 0 clears dw and db */
  int32_t type;
  const void *dy;       /* [rows, width] */
  int64_t lddy;
  const void *x;        /* [rows, width] */
  int64_t ldx;
  const float *mean, *rstd; /* [rows] */
  const void *weight;   /* [width] or NULL (1) */
  const void *residual; /* [rows, width] or NULL; not read unless dx is wanted */
  int64_t ldr;
  void *dx;             /* [rows, width] or NULL; may be dy or residual itself (then with its ld) */
  int64_t lddx;
  void *dw, *db;        /* [width] or NULL */
  void *workspace;
  size_t workspace_bytes;
  void *stream;
} cada_norm_grad;

int cada_layer_norm_backward_workspace(cada_norm_grad *a); /* rows, width, type, and whether dw and db are wanted */
int cada_layer_norm_backward(const cada_norm_grad *a);

/* Rows of a table by integer tokens: y[i] = scale w[token i], in float32, rounded once.  The row of a token that is ignore_index is zero
 * (also where ignore_index is in [0, vocab)); that of any other token outside [0, vocab) is NaN. */
typedef struct cada_embedding {
  int64_t rows;         /* 0 .. 2^30 */
  int64_t vocab;        /* 1 .. 2^24 */
  int64_t width;        /* 1 .. CADA_MAX_WIDTH */
  int32_t type;         /* of w and y */
  int32_t token_bytes;  /* 4 or 8: int32 or int64 tokens */
  const void *tokens;   /* [rows] */
  int64_t ignore_index;
  const void *w;        /* [vocab, width] */
  int64_t ldw;
  double scale;         /* finite, also in float32 */
  void *y;              /* [rows, width] */
  int64_t ldy;
  void *stream;
} cada_embedding;

int cada_embedding_forward(const cada_embedding *a); /* needs no workspace */

/* Its gradient: dw[v] = scale times the sum of dy[i] over the tokens i that are v, in float32, rounded once.  The additions have one order, which
 * depends on the sizes, the type and the tokens only: that of the tokens within a few of them, whose sums are then joined.  All of dw is written:
 * a row whose token does not occur is zero.  Tokens that are ignore_index or outside [0, vocab) add nothing. */
typedef struct cada_embedding_grad {
  int64_t rows, vocab, width; /* as above */
  int32_t type;
  int32_t token_bytes;
  const void *tokens;   /* [rows] */
  int64_t ignore_index;
  const void *dy;       /* [rows, width] */
  int64_t lddy;
  double scale;
  void *dw;             /* [vocab, width] */
  int64_t lddw;
  void *workspace;
  size_t workspace_bytes;
  void *stream;
} cada_embedding_grad;

int cada_embedding_backward_workspace(cada_embedding_grad *a); /* rows, vocab, width, type, token_bytes, scale */
int cada_embedding_backward(const cada_embedding_grad *a);

/* Softmax cross-entropy of rows of logits with integer labels, and its gradient, in one pass.
 * A class whose logit is -inf is ruled out: its probability and gradient are zero.  The target of a row is
 * (1 - smoothing) on its label plus smoothing spread evenly over the classes that are not ruled out.
 *   loss[i] = log(sum_c exp z_c) - sum_c target_c z_c        (0 for an ignored row)
 *   mean    = sum_i loss[i] / max(1, number of rows that are not ignored)
 *   grad[i] = (softmax(z) - target) * scale / max(1, that number)
 * A row whose label is ruled out has loss +inf and a finite gradient; one with no class left has loss +inf and
 * gradient zero.  NaN and +inf among the logits give NaN.  A label that is neither ignore_index nor in [0, classes) gives loss NaN
 * and gradient zero. */
typedef struct cada_xent {
  int64_t rows;          /* 0 .. 2^30, and no more than one launch takes (2^22 - 1 of the longest rows) */
  int64_t classes;       /* 1 .. 2^31 - 1 - 2^20 */
  int32_t type;          /* of logits and grad */
  int32_t label_bytes;   /* 4 or 8: int32 or int64 labels */
  const void *logits;    /* [rows, classes] */
  int64_t ldz;
  const void *labels;    /* [rows] */
  int64_t ignore_index;
  double smoothing;      /* [0, 1) */
  double scale;          /* factor of the gradient (loss scaling) */
  float *mean;           /* [1] or NULL */
  float *loss;           /* [rows] or NULL */
  void *grad;            /* [rows, classes] or NULL; may be the logits themselves (then with their ld) */
  int64_t ldg;
  void *workspace;
  size_t workspace_bytes;
  void *stream;
} cada_xent;

int cada_xent_workspace(cada_xent *a); /* rows, classes, type, mean and loss are read */
int cada_cross_entropy(const cada_xent *a);

/* The same loss of the logits z = x w + bias of a last layer, and its gradients, without the logits in memory:
 *   dx = g w^T,  dw = x^T g,  db = column sums of g,  g = (softmax(z) - target) * scale / max(1, number of rows that are not ignored)
 * z is formed in float32 for each row's statistics and, for the gradients, again in pieces of the classes, whose softmax - target
 * lies in the workspace in the operands' type (db is summed before that rounding).  Logits of less than a piece are kept in
 * the workspace in between.  Outputs that are NULL are not formed.
 * A class is ruled out by a bias of -inf; w is read there all the same.  An ignored row counts nowhere.  One whose label is neither
 * ignore_index nor in [0, classes) has loss NaN, and so has the mean; it is one of the rows that are not ignored.  Either has
 * dx = 0 and no part in dw and db, whatever x holds there. */
typedef struct cada_linear_xent {
  int64_t rows;          /* 0 .. 2^30 */
  int64_t in, classes;   /* 1 .. CADA_MAX_WIDTH; of the tables' products, at most 2^23 - 8 tiles of 64 x 64 */
  int32_t type;          /* of all tables and the bias */
  int32_t label_bytes;   /* 4 or 8: int32 or int64 labels */
  const void *x;         /* [rows, in] */
  int64_t ldx;
  const void *w;         /* [in, classes] */
  int64_t ldw;
  const void *bias;      /* [classes] or NULL */
  const void *labels;    /* [rows] */
  int64_t ignore_index;
  double smoothing;      /* [0, 1) */
  double scale;          /* factor of the gradients (loss scaling) */
  float *mean;           /* [1] or NULL */
  float *loss;           /* [rows] or NULL */
  void *dx;              /* [rows, in] or NULL */
  int64_t lddx;
  void *dw;              /* [in, classes] or NULL */
  int64_t lddw;
  void *db;              /* [classes] or NULL */
  void *workspace;
  size_t workspace_bytes;
  void *stream;
} cada_linear_xent;

int cada_linear_xent_workspace(cada_linear_xent *a); /* all but the pointers' contents, mean, scale, ignore_index and stream is read */
int cada_linear_cross_entropy(const cada_linear_xent *a);

/* AdamW over many tensors in one launch (two with clipping).  Step t = 1, 2, ... of tensor p with gradient g:
 *   g <- g * grad_scale * min(1, max_norm / norm)                 (norm: over grad_scale * all gradients; max_norm 0: no clipping;
 *                                                                  a norm past float32 counts as infinite and leaves zeros)
 *   m <- beta1 m + (1 - beta1) g,   v <- beta2 v + (1 - beta2) g^2
 *   p <- (p - lr weight_decay p) - lr/(1 - beta1^t) m / (sqrt(v)/sqrt(1 - beta2^t) + eps)
 * in float32, each operation rounded by itself; p is rounded once if it is bf16.
 *
 * The moments of all tensors lie in two flat arrays, each tensor's part filled up to whole blocks of
 * CADA_MOMENT_BLOCK elements (cada_adamw_moment_elements() in all; the fill keeps its zeros).
 * CADA_MOMENTS_32: float32.  CADA_MOMENTS_8: one byte per element and a float32 scale per block,
 *   m = q |q| s / 127^2,        q int8 in [-127, 127],  s = the block's largest |m|
 *   sqrt(v) = c^2 s / 255^2,    c uint8,                s = the block's largest sqrt(v)
 * The codes grow with the root, so that small values keep a relative precision; sqrt(v) is rounded to the nearest code but
 * never from something to zero, since it divides.  A block whose scale is below 1e-30 keeps no codes (but the 1 of a sqrt(v)
 * that is not zero); NaN or an infinity in a block makes the block NaN.  The update itself uses the moments before they are
 * rounded to codes. */
enum { CADA_MOMENTS_32 = 32, CADA_MOMENTS_8 = 8 };
#define CADA_MOMENT_BLOCK 256
typedef struct cada_adamw_tensor {
  void *param;          /* [n] contiguous, updated in place; no tensor of a plan may be listed twice (gradients may) */
  const void *grad;     /* [n] contiguous */
  void *copy;           /* [n] bf16 or NULL: the new value rounded to bf16 (for float32 masters) */
  int64_t n;            /* >= 0; all tensors' together at most 2^34, each filled up to 2048 */
  int32_t param_type, grad_type; /* CADA_F32 or CADA_BF16 */
  double weight_decay;
} cada_adamw_tensor;
typedef struct cada_adamw_config {
  const cada_adamw_tensor *tensors; /* HOST [n_tensors] */
  int32_t n_tensors;                /* 1 .. 2^20 */
  int32_t moment_bits;              /* CADA_MOMENTS_* */
  void *m, *v;                      /* float32, or int8 and uint8, [cada_adamw_moment_elements()]; 16-byte aligned */
  float *m_scale, *v_scale;         /* CADA_MOMENTS_8: [that / CADA_MOMENT_BLOCK]; else ignored */
  float *norm;                      /* [1] or NULL: where a clipped step leaves the gradients' norm */
  double beta1, beta2, eps;
  double max_norm;                  /* 0: no clipping */
  void *workspace;                  /* the plan: kept by the caller until cada_adamw_destroy */
  size_t workspace_bytes;
  void *stream;
} cada_adamw_config;
typedef struct cada_adamw cada_adamw; /* opaque, host memory owned by the library */

int64_t cada_adamw_moment_elements(const cada_adamw_config *cfg); /* the tensors' n are read; -1 and an error text if invalid */
int cada_adamw_workspace(cada_adamw_config *cfg); /* the tensors' n are read */
/* Lays the plan out in the workspace.  Does not touch the moments: a new run starts from zeros (zero bytes: also
 * CADA_MOMENTS_8), a resumed one from what was saved. */
int cada_adamw_init(const cada_adamw_config *cfg, cada_adamw **out);
/* One step, on the stream of the plan's config; t >= 1.  grad_scale: DEVICE [1] or NULL (1), read when the step runs, in nothing
 * that the plan writes. */
int cada_adamw_step(cada_adamw *plan, int64_t t, double lr, const float *grad_scale);
/* The moments as float32 values, [cada_adamw_moment_elements()] each, on the plan's stream; either may be NULL. */
int cada_adamw_moments(cada_adamw *plan, float *m, float *v);
void cada_adamw_destroy(cada_adamw *plan);

#ifdef __cplusplus
}
#endif
#endif /* CADA_OPS_H */
