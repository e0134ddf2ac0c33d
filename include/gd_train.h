/*
 * gd_train.h - the operators of a training step around the gradient exchange of gd.h (libgd.so, CUDA, sm_100a).
 *
 * gd.h drops, packs and applies gradients.  These calls make the gradient and use the summed one:
 *   gd_linear_forward / gd_linear_backward   a linear layer with bias, activation and residual, and its gradients
 *   gd_cross_entropy                         the softmax cross-entropy of a batch and the gradient of its logits
 *   gd_adamw_step                            one AdamW update of many tensors, the moments in 32 or in 8 bits
 *
 * The conventions of gd.h hold: device pointers unless marked HOST, a stream as void*, calls only enqueue and never
 * allocate, argument errors are found on the host before anything is enqueued and returned as a gd_status_t.  All sums,
 * softmax statistics and moments are fp32 (or the 8-bit form stated below); a result is rounded once, to the type of its buffer.
 * Leading dimensions ("ld...") are in elements, rows may lie further apart than their length and start at any address that is a
 * multiple of the element's size; inputs and outputs of one call must not overlap unless it says so.
 */
#ifndef GD_TRAIN_H
#define GD_TRAIN_H

#include "gd.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { GD_DTYPE_FP32 = 0, GD_DTYPE_BF16 = 1, GD_DTYPE_FP16 = 2 };
enum { GD_ACT_NONE = 0, GD_ACT_RELU = 1, GD_ACT_GELU = 2 /* x Phi(x), with erf */, GD_ACT_SILU = 3 };
enum { GD_W_IN_OUT = 0 /* w is [k, n], as the matrices of gd.h's workloads are */, GD_W_OUT_IN = 1 /* w is [n, k] */ };

/* gd_linear_backward_args.flags */
enum { GD_LINEAR_ACCUMULATE = 1u /* dw and db are added to what their buffers hold (dw_dtype must then be GD_DTYPE_FP32) */ };

/*
 * gd_linear_forward
 *     z = x W + bias              x [m, k], W given as w [k, n] or [n, k] (w_layout); fp32 accumulation
 *     y = act(z) + residual       both terms in fp32, one rounding to y_dtype
 *     pre = z                     rounded to dtype; what gd_linear_backward takes (activations other than GD_ACT_NONE)
 * m, n, k may be 0 (an empty sum is 0).  y may be the same buffer as residual when the types, addresses and leading dimensions agree.
 */
typedef struct gd_linear_forward_args {
  uint64_t m, n, k;           /* each < 2^31 */
  int32_t dtype;              /* of x, w, residual and pre: GD_DTYPE_BF16 or GD_DTYPE_FP16 */
  int32_t activation;         /* GD_ACT_* */
  int32_t w_layout;           /* GD_W_* */
  int32_t bias_dtype;         /* GD_DTYPE_FP32, or dtype */
  int32_t y_dtype;            /* dtype, or GD_DTYPE_FP32 */
  int32_t reserved;           /* 0 */
  const void* x;              /* [m, k] */
  uint64_t ldx;
  const void* w;              /* [k, n] or [n, k] */
  uint64_t ldw;
  const void* bias;           /* n, or NULL */
  const void* residual;       /* [m, n], or NULL */
  uint64_t ld_residual;
  void* y;                    /* [m, n] */
  uint64_t ldy;
  void* pre;                  /* [m, n], or NULL */
  uint64_t ld_pre;
  void* workspace;            /* 256-byte aligned, >= gd_linear_workspace_bytes(); zeroed once before its first use */
  size_t workspace_bytes;
} gd_linear_forward_args;

int gd_linear_forward(const gd_linear_forward_args* args, void* stream);

/*
 * gd_linear_backward - gradients of the above for dy, the gradient of y (that of residual is dy itself):
 *     dz = dy * act'(pre)         (GD_ACT_NONE: dz = dy, pre is not read)
 *     dx = dz W^T    [m, k], dtype
 *     dw = x^T dz    in w's layout, dw_dtype
 *     db = column sums of dz, fp32
 * Any of dx, dw, db may be NULL.  The products take dz rounded to dtype: exact for GD_ACT_NONE and GD_ACT_RELU (the slope
 * is 0 or 1; 0 at pre = 0), one rounding of at most 2^-8 (bf16) or 2^-11 (fp16) of an entry for GELU and SiLU; db sums the unrounded dz.
 *
 * In both calls the tensor cores' fp32 accumulator truncates: a 16-bit result is off by about 1.1e-9 of its size per step of the contraction
 * before its own rounding (9e-5 over 85000), an fp32 result, summed in chains of 512, by 5e-7 at any depth.
 */
typedef struct gd_linear_backward_args {
  uint64_t m, n, k;
  int32_t dtype, activation, w_layout;
  int32_t dw_dtype;           /* dtype, or GD_DTYPE_FP32 */
  uint32_t flags;             /* GD_LINEAR_ACCUMULATE or 0 */
  int32_t reserved;           /* 0 */
  const void* dy;             /* [m, n] */
  uint64_t ld_dy;
  const void* pre;            /* [m, n]; may be NULL with GD_ACT_NONE */
  uint64_t ld_pre;
  const void* x;              /* [m, k]; may be NULL without dw */
  uint64_t ldx;
  const void* w;              /* as in the forward call; may be NULL without dx */
  uint64_t ldw;
  void* dx;
  uint64_t ld_dx;
  void* dw;
  uint64_t ld_dw;
  float* db;
  void* workspace;
  size_t workspace_bytes;
} gd_linear_backward_args;

int gd_linear_backward(const gd_linear_backward_args* args, void* stream);

/*
 * Workspace of the two calls above for up to m rows.  The products read their operands with tiled copies that want 16-byte
 * aligned rows; others are first laid out in the workspace.  any_layout = 0: x, w, dy and pre are contiguous and
 * start at multiples of 16 bytes (space is then set aside only for what m, n, k themselves make ragged); 1: anything.
 * The first 256 bytes hold the status word: zero them once; gd_linear_status() reads it (GD_OK or GD_ERR_DEVICE_TIMEOUT,
 * which stays until the word is zeroed again) and synchronises the stream.
 */
int gd_linear_workspace_bytes(uint64_t m, uint64_t n, uint64_t k, int any_layout, size_t* bytes_out);
int gd_linear_status(const void* workspace, void* stream);

/*
 * Self-test of a bounded wait, as gd_selftest_bounded_wait is in gd.h: zeroes the workspace (256-byte aligned, at least 16896 bytes) and runs the
 * sum of a bias gradient by two CTAs, of which one waits at most budget_ns for eight bytes more than the other sends.  Afterwards
 * gd_linear_status(workspace) is GD_ERR_DEVICE_TIMEOUT and the 32 fp32 sums at its byte 256 are NaN.  The context stays usable.
 */
int gd_selftest_linear_wait(void* workspace, size_t workspace_bytes, uint64_t budget_ns, void* stream);

/*
 * gd_cross_entropy - for every row i of logits [rows, classes] with target t = targets[i]:
 *     lse[i]    = log sum_j exp(logits[i, j])
 *     loss[i]   = lse[i] - logits[i, t]
 *     grad[i,j] = (exp(logits[i, j] - lse[i]) - (j == t)) * grad_scale * (*grad_scale_dev)
 * A row whose target is ignore_index has loss 0 and gradient 0 whatever its logits are (its lse is theirs).  Logits of -inf are masked classes:
 * they take no part and their gradient is 0, unless the target is one: the row's loss is then +inf, and the gradient as the formula
 * says, -grad_scale * (*grad_scale_dev) at the target.  In a row with a target, where every class is masked, or with +inf or NaN among
 * the logits, loss and gradient are NaN; so are those of a row whose target is neither ignore_index nor in [0, classes).
 * grad may be logits itself (same address and leading dimension) or NULL; loss and lse may be NULL.  The call has no workspace and
 * so no status word: a device-side wait that gives up leaves NaN in its row's results.
 */
typedef struct gd_cross_entropy_args {
  uint64_t rows, classes;     /* classes >= 1, each < 2^31 */
  int32_t dtype;              /* of logits and grad: GD_DTYPE_* */
  int32_t target_bits;        /* 32 or 64: signed integers */
  const void* logits;         /* [rows, classes] */
  uint64_t ld_logits;
  const void* targets;        /* rows */
  int64_t ignore_index;
  float grad_scale;
  int32_t reserved;           /* 0 */
  const float* grad_scale_dev;/* one fp32, or NULL (1) */
  float* loss;                /* rows, or NULL */
  float* lse;                 /* rows, or NULL */
  void* grad;                 /* [rows, classes], or NULL */
  uint64_t ld_grad;
} gd_cross_entropy_args;

int gd_cross_entropy(const gd_cross_entropy_args* args, void* stream);

/*
 * gd_adamw_step - one update of n_tensors tensors, element by element, every operation one fp32 rounding in this order
 * (constants are computed in double on the host and rounded to fp32):
 *     s = grad_scale * (*grad_scale_dev)              g = grad * s
 *     m = m * beta1 + g * (1 - beta1)                 v = v * beta2 + (g * (1 - beta2)) * g
 *     d = sqrt(v) * (1 / sqrt(1 - beta2^step)) + eps
 *     p = p * (1 - lr * weight_decay) - (m / d) * (lr / (1 - beta1^step))
 * so that fp32 results are the same bits whatever the tensors' alignment.  p is rounded once to param_dtype; copy, if given, receives p
 * rounded once to copy_dtype (the 16-bit weights the next forward pass reads).
 *
 * state_bits = 8: m and the ROOT of v are held as fp8 (1 sign, 4 exponent, 3 mantissa bits, bias 7) times a scale that a block of
 * 128 consecutive elements of a tensor shares: m_scale and v_scale, ceil(n / 128) fp32 powers of two, 2^(E - 7) with 2^E
 * <= the block's largest finite magnitude < 2^(E + 1) (at least 2^-126).  v is the square of its held root.  A magnitude is rounded up
 * to its upper neighbour with a probability of 1 in 2^16 for every 2^-16 of the way it lies past the lower one, so that
 * moments that change by less than a step still change on average; the 16 random bits are the upper (m) and lower (v) half of
 * mix(i * 0x9E3779B9 + seed + t * 0x85EBCA77) mod 2^32 for element i of tensor t, with mix as in gd.h's sampled-threshold mode.
 * Pass another seed every step.  A positive root is held as at least the smallest positive code, so no divisor
 * vanishes that should not; a moment that is not finite is held as NaN.
 */
typedef struct gd_adamw_tensor {
  void* param;                /* n, param_dtype */
  const void* grad;           /* n, grad_dtype */
  void* m;                    /* n fp32, or n bytes */
  void* v;                    /* n fp32, or n bytes */
  float* m_scale;             /* ceil(n / 128) fp32; state_bits = 8 only */
  float* v_scale;
  void* copy;                 /* n, copy_dtype, or NULL */
  uint64_t n;                 /* may be 0; < 2^40 */
  double weight_decay;
} gd_adamw_tensor;

typedef struct gd_adamw_args {
  const gd_adamw_tensor* tensors; /* HOST */
  uint32_t n_tensors;
  int32_t state_bits;         /* 32 or 8 */
  int32_t param_dtype, grad_dtype, copy_dtype;
  uint32_t seed;
  uint64_t step;              /* 1 for the first update */
  double lr, beta1, beta2, eps;  /* 0 <= beta < 1, eps >= 0 */
  float grad_scale;
  int32_t reserved;           /* 0 */
  const float* grad_scale_dev;/* one fp32, or NULL (1) */
} gd_adamw_args;

int gd_adamw_step(const gd_adamw_args* args, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* GD_TRAIN_H */
