/*
 * gd_layers.h - the layers of a language model around the linear layer and the loss of gd_train.h (libgd.so, CUDA, sm_100a).
 *
 *   gd_embedding_forward / _backward    lookup of scaled rows, and their gradient by sorted tokens
 *   gd_layer_norm_forward / _backward   layer norm of rows
 *   gd_recurrence_forward / _backward   a gated linear recurrence over packed sequences
 *   gd_gated_forward / _backward        the gated feed-forward block: two projections, activation and product
 *
 * The conventions of gd_train.h hold: device pointers, a stream as void*, calls only enqueue and never allocate, argument errors are
 * found on the host before anything is enqueued and returned as a gd_status_t.  All sums, statistics and states are fp32; a result is
 * rounded once, to the type of its buffer.  Leading dimensions ("ld...") are in elements, rows may lie further apart than their
 * length and start at any address that is a multiple of the element's size; inputs and outputs of one call must not overlap unless
 * it says so.  Results are the same bits every time: nothing is summed by atomics.
 */
#ifndef GD_LAYERS_H
#define GD_LAYERS_H

#include "gd_train.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * gd_embedding_forward - y[i, :] = scale * table[ids[i], :], one fp32 product, rounded to y_dtype.
 * A position whose id is ignore_index (padding) gives a row of zeros.  An id that is neither ignore_index nor in [0, vocab) gives a row
 * of NaN; nothing outside the table is read.
 * y_dtype is table_dtype, or GD_DTYPE_FP32, or, from a table in fp32, any.
 */
typedef struct gd_embedding_forward_args {
  uint64_t tokens, vocab, width;   /* tokens and vocab < 2^31, width < 2^20 */
  int32_t table_dtype, y_dtype;    /* GD_DTYPE_* */
  int32_t id_bits;                 /* 32 or 64: signed integers */
  float scale;
  int64_t ignore_index;
  const void* table;               /* [vocab, width] */
  uint64_t ld_table;
  const void* ids;                 /* tokens */
  void* y;                         /* [tokens, width] */
  uint64_t ld_y;
} gd_embedding_forward_args;

int gd_embedding_forward(const gd_embedding_forward_args* args, void* stream);

/* gd_embedding_backward_args.flags */
enum { GD_EMBEDDING_ACCUMULATE = 1u /* the sums are added to what dtable holds (GD_DTYPE_FP32 then); rows of ids that do not occur stay as they are */ };

/*
 * gd_embedding_backward - dtable[v, :] = scale * sum of dy[i, :] over the positions i with ids[i] = v, in ascending order of i within parts
 * that depend on the ids alone; rows of ids that do not occur are zeros.  Positions with ignore_index or an id out of range have no part in it.
 */
typedef struct gd_embedding_backward_args {
  uint64_t tokens, vocab, width;   /* tokens and vocab < 2^31, width < 2^20 */
  int32_t dtype;                   /* of dy: GD_DTYPE_* */
  int32_t dtable_dtype;            /* GD_DTYPE_FP32, or dtype */
  int32_t id_bits;
  float scale;
  int64_t ignore_index;
  uint32_t flags;                  /* GD_EMBEDDING_ACCUMULATE or 0 */
  int32_t reserved;                /* 0 */
  const void* dy;                  /* [tokens, width] */
  uint64_t ld_dy;
  const void* ids;
  void* dtable;                    /* [vocab, width] */
  uint64_t ld_dtable;
  void* workspace;                 /* 256-byte aligned, >= gd_embedding_workspace_bytes(); its contents do not matter */
  size_t workspace_bytes;
} gd_embedding_backward_args;

int gd_embedding_backward(const gd_embedding_backward_args* args, void* stream);
/* Workspace of the call above for up to that many tokens. */
int gd_embedding_workspace_bytes(uint64_t tokens, uint64_t vocab, uint64_t width, size_t* bytes_out);

/*
 * gd_layer_norm_forward - for every row x of [rows, width]:
 *     mean = sum(x) / width      rstd = 1 / sqrt(sum((x - mean)^2) / width + eps)      y = (x - mean) * rstd * weight + bias
 * mean and rstd are what gd_layer_norm_backward takes.  y may be x itself (same address and leading dimension).
 */
typedef struct gd_layer_norm_forward_args {
  uint64_t rows, width;            /* each < 2^31; width >= 1 */
  int32_t dtype;                   /* of x and y: GD_DTYPE_* */
  int32_t param_dtype;             /* of weight and bias: GD_DTYPE_FP32, or dtype */
  float eps;                       /* >= 0 */
  int32_t reserved;                /* 0 */
  const void* x;
  uint64_t ldx;
  const void* weight;              /* width, or NULL (1) */
  const void* bias;                /* width, or NULL (0) */
  void* y;
  uint64_t ldy;
  float* mean;                     /* rows, or NULL */
  float* rstd;                     /* rows, or NULL */
} gd_layer_norm_forward_args;

int gd_layer_norm_forward(const gd_layer_norm_forward_args* args, void* stream);

/* gd_layer_norm_backward_args.flags */
enum { GD_LAYER_NORM_ACCUMULATE = 1u /* dweight and dbias are added to what their buffers hold */ };

/*
 * gd_layer_norm_backward - gradients for dy, with n = (x - mean) * rstd and g = dy * weight:
 *     dx = (g - sum(g) / width - n * sum(g * n) / width) * rstd + add
 *     dweight = sum over rows of dy * n        dbias = sum over rows of dy
 * add is the gradient that reaches x past the norm (a skip connection's).  Any of dx, dweight and dbias may be NULL.  dx may be dy or
 * add itself (same address and leading dimension).
 */
typedef struct gd_layer_norm_backward_args {
  uint64_t rows, width;
  int32_t dtype;                   /* of dy, x, add and dx */
  int32_t param_dtype;             /* of weight */
  uint32_t flags;                  /* GD_LAYER_NORM_ACCUMULATE or 0 */
  int32_t reserved;                /* 0 */
  const void* dy;
  uint64_t ld_dy;
  const void* x;
  uint64_t ldx;
  const void* weight;              /* width, or NULL (1) */
  const float* mean;               /* rows */
  const float* rstd;               /* rows */
  const void* add;                 /* [rows, width], or NULL */
  uint64_t ld_add;
  void* dx;
  uint64_t ld_dx;
  float* dweight;                  /* width */
  float* dbias;                    /* width */
  void* workspace;                 /* 256-byte aligned, >= gd_layer_norm_workspace_bytes(); its contents do not matter */
  size_t workspace_bytes;
} gd_layer_norm_backward_args;

int gd_layer_norm_backward(const gd_layer_norm_backward_args* args, void* stream);
int gd_layer_norm_workspace_bytes(uint64_t rows, uint64_t width, size_t* bytes_out);

/*
 * gd_recurrence_forward - for every sequence and column, from the state h[-1] = h0:
 *     f = 1 / (1 + exp(-gate[t]))      h[t] = f * h[t-1] + (1 - f) * value[t]      y[t] = h[t], rounded to dtype
 * A device-side wait that runs out leaves NaN in the results (these calls have no status).
 * The state is fp32 throughout.  A gate of -inf forgets all that came before (a state that is not finite stays), one of +inf keeps the state.
 *
 * Sequences lie one behind the other in the rows of gate, value and y: sequence s is rows offsets[s] .. offsets[s + 1] - 1, offsets
 * ascending and at most `rows`; rows before the first and behind the last sequence have no part in it and are not written.  A beginning or
 * end outside 0 .. rows is cut to that, and an end before its beginning to the beginning.  Where offsets descend, sequences may come to share
 * rows or marks: the results of all of them are undefined then and need not be the same twice, but nothing outside them is touched.
 * offsets = NULL: all sequences are rows / sequences long (rows a multiple of that).  A sequence of length 0 has h_last = h0.
 * A call with one row per sequence is the step of a model that answers token by token; h_last may then, as always, be h0 itself.
 *
 * marks, if given, receive the states that gd_recurrence_backward starts from: gd_recurrence_marks_rows() rows of `width` fp32.  The backward
 * call takes the same offsets, sequences and rows.
 */
typedef struct gd_recurrence_forward_args {
  uint64_t rows, sequences, width; /* each < 2^31 */
  int32_t dtype;                   /* of gate, value and y: GD_DTYPE_* */
  int32_t offset_bits;             /* 32 or 64: signed integers */
  const void* offsets;             /* sequences + 1, or NULL */
  const void* gate;                /* [rows, width] */
  uint64_t ld_gate;
  const void* value;
  uint64_t ld_value;
  void* y;
  uint64_t ld_y;
  const float* h0;                 /* [sequences, width], contiguous, or NULL (0) */
  float* h_last;                   /* [sequences, width], contiguous, or NULL; may be h0 */
  float* marks;                    /* or NULL */
} gd_recurrence_forward_args;

int gd_recurrence_forward(const gd_recurrence_forward_args* args, void* stream);
int gd_recurrence_marks_rows(uint64_t rows, uint64_t sequences, uint64_t* rows_out);

/*
 * gd_recurrence_backward - gradients for dy and dh_last, the gradients of y and h_last, backwards in time:
 *     dh[t] = dy[t] + f[t+1] * dh[t+1]   (dh_last in place of the second term at a sequence's last row)
 *     dvalue[t] = (1 - f[t]) * dh[t]     dgate[t] = dh[t] * (h[t-1] - value[t]) * f[t] * (1 - f[t])     dh0 = f[0] * dh[0]
 * dgate may be gate or dy itself, and dvalue value (same address and leading dimension).  A sequence of length 0 has dh0 = dh_last.
 */
typedef struct gd_recurrence_backward_args {
  uint64_t rows, sequences, width;
  int32_t dtype;                   /* of dy, gate, value, dgate and dvalue */
  int32_t offset_bits;
  const void* offsets;
  const void* dy;
  uint64_t ld_dy;
  const void* gate;
  uint64_t ld_gate;
  const void* value;
  uint64_t ld_value;
  const float* marks;              /* of the forward call */
  void* dgate;
  uint64_t ld_dgate;
  void* dvalue;
  uint64_t ld_dvalue;
  const float* dh_last;            /* [sequences, width], or NULL (0) */
  float* dh0;                      /* [sequences, width], or NULL; may be dh_last */
} gd_recurrence_backward_args;

int gd_recurrence_backward(const gd_recurrence_backward_args* args, void* stream);

/*
 * Self-test of the recurrence's bounded waits, as gd_selftest_linear_wait is in gd_train.h: zeroes the workspace (256-byte aligned, at least 663552
 * bytes) and runs a call over 8192 rows of 8 columns in bf16 whose waits, for at most budget_ns, are for more than is sent.  which: 0 forward, a
 * tile's copies; 1 forward, the maps of a cluster; 2 and 3 the same of the backward call.  Afterwards y, or dgate, which begins at byte 401408, is NaN
 * throughout, and so is dvalue, 131072 bytes further on, and the context stays usable.
 */
int gd_selftest_recurrence_wait(void* workspace, size_t workspace_bytes, int which, uint64_t budget_ns, void* stream);

/*
 * gd_gated_forward - the gated feed-forward block up to its hidden layer.  x [m, k], W given as w [k, 2 n] or [2 n, k] (w_layout): the first n
 * outputs are the gate, the others are multiplied by it.
 *     z = x W + bias  [m, 2 n]        y = act(z[:, :n]) * z[:, n:]  [m, n]        pre = z, rounded to dtype
 * fp32 accumulation; y is made from the unrounded z.  m, n and k may be 0 (an empty sum is 0).
 */
typedef struct gd_gated_forward_args {
  uint64_t m, n, k;                /* each < 2^30 */
  int32_t dtype;                   /* of x, w, y and pre: GD_DTYPE_BF16 or GD_DTYPE_FP16 */
  int32_t activation;              /* GD_ACT_* */
  int32_t w_layout;                /* GD_W_* */
  int32_t bias_dtype;              /* GD_DTYPE_FP32, or dtype */
  const void* x;
  uint64_t ldx;
  const void* w;
  uint64_t ldw;
  const void* bias;                /* 2 n, or NULL */
  void* y;                         /* [m, n] */
  uint64_t ldy;
  void* pre;                       /* [m, 2 n], or NULL */
  uint64_t ld_pre;
  void* workspace;                 /* 256-byte aligned, >= gd_gated_workspace_bytes(); zeroed once before its first use */
  size_t workspace_bytes;
} gd_gated_forward_args;

int gd_gated_forward(const gd_gated_forward_args* args, void* stream);

/*
 * gd_gated_backward - gradients of the above for dy, the gradient of y, with a = pre[:, :n] and u = pre[:, n:]:
 *     dz = [dy * u * act'(a), dy * act(a)]  [m, 2 n]
 *     dx = dz W^T  [m, k], dtype      dw = x^T dz in w's layout, dw_dtype      db = column sums of dz, 2 n fp32
 * Any of dx, dw, db may be NULL.  The products take dz rounded to dtype (one rounding of at most 2^-8 (bf16) or 2^-11 (fp16) of an
 * entry); db sums the unrounded dz.  With GD_LINEAR_ACCUMULATE dw (GD_DTYPE_FP32 then) and db are added to what their buffers hold.
 */
typedef struct gd_gated_backward_args {
  uint64_t m, n, k;
  int32_t dtype, activation, w_layout;
  int32_t dw_dtype;                /* dtype, or GD_DTYPE_FP32 */
  uint32_t flags;                  /* GD_LINEAR_ACCUMULATE or 0 */
  int32_t reserved;                /* 0 */
  const void* dy;                  /* [m, n] */
  uint64_t ld_dy;
  const void* pre;                 /* [m, 2 n] */
  uint64_t ld_pre;
  const void* x;                   /* may be NULL without dw */
  uint64_t ldx;
  const void* w;                   /* may be NULL without dx */
  uint64_t ldw;
  void* dx;
  uint64_t ld_dx;
  void* dw;
  uint64_t ld_dw;
  float* db;
  void* workspace;
  size_t workspace_bytes;
} gd_gated_backward_args;

int gd_gated_backward(const gd_gated_backward_args* args, void* stream);

/*
 * Self-test of a bounded wait, as gd_selftest_linear_wait is in gd_train.h: zeroes the workspace (256-byte aligned, at least 25088 bytes) and sums the
 * bias gradient of 128 rows by two CTAs, one waiting (for at most budget_ns) for more than the other sends.  Afterwards gd_linear_status() is
 * GD_ERR_DEVICE_TIMEOUT and the 64 floats behind the status word's 256 bytes are NaN; the context stays usable.
 */
int gd_selftest_gated_wait(void* workspace, size_t workspace_bytes, uint64_t budget_ns, void* stream);

/* Workspace of the two calls above for up to m rows; any_layout and the status word as in gd_linear_workspace_bytes(), read by gd_linear_status(). */
int gd_gated_workspace_bytes(uint64_t m, uint64_t n, uint64_t k, int any_layout, size_t* bytes_out);

#ifdef __cplusplus
}
#endif
#endif /* GD_LAYERS_H */
