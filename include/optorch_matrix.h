/*
 * optorch_matrix -- matrix operators on the device, for AMD MI355X (gfx950): linear layers with bias,
 * activation and skip connection in the product's epilogue, their gradients, and the orthogonalised
 * update of weight matrices.  C ABI; part of liboptorch_seq.so.
 *
 * Matrices are row-major: element (r, c) at r * ld + c, ld >= columns, any alignment of the element
 * type.  Pointers are DEVICE pointers unless named *_host.  Matrices and vectors that are written must not share an
 * element with any other of the call unless stated otherwise (refused; rows that lie between each other's are apart).
 *
 * Execution: every call only enqueues kernels on the stream it is given (NULL = the default stream) and
 * returns; it neither allocates nor synchronises and may be captured into a HIP graph.  The caller owns
 * all buffers, workspaces included, and keeps them alive until the stream has passed the call; calls that
 * share a workspace have to follow one another on the device.  Results do not depend on the launch: no
 * sum is made with atomics.
 *
 * Errors: OPTORCH_OK or a negative code of optorch_seq.h; optorch_matrix_last_error gives the message of
 * the calling thread's most recent failure.  A call that fails a check has launched nothing.
 */
#ifndef OPTORCH_MATRIX_H
#define OPTORCH_MATRIX_H

#include <stdint.h>

#include "optorch_seq.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- linear layers ------------------------------------------------------------------------------- */

typedef enum {
  OPTORCH_ACT_NONE = 0, OPTORCH_ACT_RELU = 1,
  OPTORCH_ACT_GELU = 2, /* z * Phi(z), Phi the normal distribution function */
  OPTORCH_ACT_SILU = 3  /* z / (1 + exp(-z)) */
} optorch_activation_t;

/* Arguments of both directions.  `precision` (optorch_precision_t) is the type of x, w, residual, y, z, dy, dx
 * and dw; bias and dbias are fp32.  Products are summed in fp32 (fp32 operands as three bf16 planes, which keep
 * all 24 bits), everything up to the stored result is fp32, and a result is rounded once. */
typedef struct {
  int32_t precision, activation;
  int64_t rows;                       /* samples; 0 is allowed */
  int32_t in_features, out_features;  /* 1 .. 2^22 - 8, leading dimensions too; fp32: 1 .. 2^20 - 16 */
  const void* x; int64_t ldx;         /* rows x in */
  const void* w; int64_t ldw;         /* out x in */
  const float* bias;                  /* out, or NULL */
  const void* residual; int64_t ldr;  /* forward: rows x out, or NULL; may be y itself */
  void* y; int64_t ldy;               /* forward: rows x out */
  void* z; int64_t ldz;               /* rows x out: x w^T + bias before the activation.  Forward: written, or NULL;
                                         backward: read, NULL allowed without an activation */
  const void* dy; int64_t lddy;       /* backward: rows x out */
  void* dx; int64_t lddx;             /* backward: rows x in, or NULL */
  void* dw; int64_t lddw;             /* backward: out x in, or NULL */
  float* dbias;                       /* backward: out, or NULL */
  void* workspace; uint64_t workspace_bytes; /* 256-byte aligned */
  void* hip_stream;
} optorch_linear_t;

/* Bytes of workspace that the forward (backward = 0) or backward call needs with these arguments (the workspace
 * fields are ignored); negative code on invalid arguments. */
int64_t optorch_linear_workspace(const optorch_linear_t* a, int32_t backward);

/* y = activation(x w^T + bias) + residual */
int optorch_linear_forward(const optorch_linear_t* a);

/* dz = dy * activation'(z);  dx = dz w,  dw = dz^T x,  dbias = column sums of dz.  In 16-bit precision dz is held as two
 * values of the storage type for the two products, which keeps 16 (bf16) or 22 (fp16) of its bits; dbias sums it unrounded.
 * ReLU's dz is 0 where z is not above 0, whatever dy is there.  The gradient of the skip connection is dy itself.  With
 * rows = 0, dw and dbias are zero. */
int optorch_linear_backward(const optorch_linear_t* a);

/* ---- orthogonalised updates ------------------------------------------------------------------------ */

/* A matrix inside a flat vector: element (r, c) at offset + r * ld + c. */
typedef struct {
  int64_t offset;
  int32_t rows, cols;
  int64_t ld;
} optorch_matrix_t;

typedef struct {
  int32_t steps;             /* Newton-Schulz steps, 1 .. 16; <= 0 selects 5 */
  const float* coefficients; /* host: a, b, c of every step (3 * steps values), or NULL: 3.4445, -4.7750, 2.0315 in each */
  float eps;                 /* a matrix of a smaller 2-norm is divided by eps instead; <= 0 selects 1e-7 */
  int32_t reserved;
} optorch_ortho_config_t;

typedef struct optorch_ortho optorch_ortho_t; /* opaque: the plan for one list of matrices */

/* Plans the launches for a list of matrices (host only): sizes from 1 x 1 on, any mixture; the matrices must not
 * overlap.  Steps whose polynomial would let a singular value in [0, 1] grow beyond 64 are refused. */
int optorch_ortho_create(const optorch_matrix_t* matrices, int32_t n, const optorch_ortho_config_t* cfg, optorch_ortho_t** out);

/* workspace_bytes: device memory the plan needs; span: 1 + the largest element index of any matrix (the length a flat
 * vector must have).  Either may be NULL. */
int optorch_ortho_query(const optorch_ortho_t* h, uint64_t* workspace_bytes, int64_t* span);

/* Lends the workspace (256-byte aligned) to the plan and copies its tables there; returns when they have arrived (not to be
 * captured into a graph).  Borrowed until the next bind or destroy. */
int optorch_ortho_bind(optorch_ortho_t* h, void* workspace_dev, uint64_t workspace_bytes);

/* For every matrix G of the list: X = G / max(|G|, eps) (2-norm of its elements), then `steps` times
 * X <- a X + (b X X^T + c (X X^T)^2) X, towards the orthogonal factor of G.  g and o are flat vectors of the given
 * precisions, elements of o outside the matrices are left alone; o may be g.  Whatever the precision of g, the result is off by
 * what fp32 arithmetic makes of the steps (in the 2-norm about 1e-6, up to 1e-4 where all but a few singular values are below 1e-3
 * of the largest) and 7e-6 more, 1e-4 more where o is bf16, before it is rounded.
 * A zero matrix gives zeros, one with an infinity or NaN gives NaN throughout; the others are not touched by it. */
int optorch_orthogonalize(optorch_ortho_t* h, int32_t g_precision, const void* g, int32_t o_precision, void* o, void* hip_stream);

typedef enum {
  OPTORCH_SCALE_NONE = 0,
  OPTORCH_SCALE_ASPECT = 1, /* sqrt(max(1, rows / cols)) */
  OPTORCH_SCALE_RMS = 2     /* 0.2 * sqrt(max(rows, cols)): the update's root mean square is about 0.2 */
} optorch_update_scale_t;

/* One update of every matrix of the list; all vectors are flat and share the list's offsets:
 *   v <- momentum * v + grad_scale * g;   u = nesterov ? grad_scale * g + momentum * v : v
 *   w <- (1 - lr * weight_decay) * w - lr * scale(rows, cols) * orthogonalised(u);   w16 <- w rounded */
typedef struct {
  int32_t g_precision; const void* g;
  float* w; float* v;                  /* fp32 master weights and momentum */
  int32_t w16_precision; void* w16;    /* bf16 or fp16 copy of w, or NULL */
  float lr, momentum, weight_decay, grad_scale; /* grad_scale: 1 / loss scale */
  int32_t nesterov, scale_mode;        /* optorch_update_scale_t */
  int32_t* skipped;                    /* device or NULL: 1 if any matrix holds an element of u that is not finite, else 0;
                                          then w, v and w16 are left as they were */
} optorch_muon_t;
int optorch_muon_update(optorch_ortho_t* h, const optorch_muon_t* a, void* hip_stream);

void optorch_ortho_destroy(optorch_ortho_t* h);

const char* optorch_matrix_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* OPTORCH_MATRIX_H */
