/*
 * moccasin_training.h -- C ABI of the operators that a rematerialisation plan
 * is run with (libmoccasin_hip.so, next to moccasin.h): activation checkpoints
 * in 8 bits, layer norm, linear layers, and their gradients; what joins the
 * layers to a training step: the residual connection with its norms and gate,
 * log probabilities and their gradient, and AdamW over many tensors; on one AMD
 * MI355X (gfx950).
 *
 * A plan says of every output of a training step whether it stays in memory or
 * is computed again.  These calls are the steps of such a plan; what stays may
 * be kept in 8 bits and used in the backward pass as it is kept (the search
 * knows one size of an output: which are kept so is up to the caller).  Every
 * call gives the same bits for the same values at the same alignments and
 * strides on one kind of device, whatever else runs (no atomics, a fixed order
 * of every sum), so an activation that is computed again from operands that lie
 * alike is the one that was dropped.  Alignment, strides and sizes choose a
 * product's kernel and with it the order of its sums: operands that lie
 * otherwise can change the last bit of a sum.
 *
 * Matrices.  moc_matrix describes rows x cols values: float32, float16 or
 * bfloat16, or a checkpoint.  Values of a row lie next to each other, rows are
 * `stride` elements apart (stride >= cols).  Every alignment to the element's
 * size is taken; the matrix products load 16 bytes at a time straight into
 * LDS where operands start on 16 bytes and strides and contiguous sizes are
 * multiples of 8 elements, and through registers otherwise.  A product of more
 * than 2^22 tiles is refused with MOC_EOVERFLOW.
 *
 * Checkpoints.  32 consecutive columns of a row share a scale 2^k, held as the
 * byte k + 127 at scales[row * scale_stride + col / 32]; one byte a value, at
 * ((uint8_t*)data)[row * stride + col], is a code of the format:
 *   MOC_E4M3   1 sign, 4 exponent, 3 fraction bits, largest 448, no infinities,
 *              0x7F and 0xFF are NaN
 *   MOC_I8     two's complement -127..127, -128 is NaN
 * and stands for code * 2^k.  Writing: k is the smallest whole number, at least
 * -111, for which the block's largest finite magnitude is at most 448 * 2^k or
 * 127 * 2^k; codes are rounded to nearest, ties to even; infinities and NaN
 * become NaN (0x7F, -128).  Magnitudes above 1.875 * 2^E (MOC_E4M3) or 1.96875 * 2^E
 * (MOC_I8) are taken for that, with E = 15 where the values are float16 and 127
 * otherwise, so that what is read back in the type it came in is finite.  A
 * value is off by at most 2^-4 of itself or 2^(k-10) (MOC_E4M3), 2^(k-1)
 * (MOC_I8).  A scale is a power of two, so a code's value is exact in float32
 * and bfloat16 (in float16 too unless it is below 2^-14 or above 65504): a
 * checkpoint that a call reads adds no rounding to the one of its writing.
 *
 * Activations (`act`): MOC_ACT_RELU  u <= 0 ? 0 : u;  MOC_ACT_GELU  u * s(2 * sqrt(2/pi) *
 * (u + 0.044715 u^3)), the tanh form;  MOC_ACT_SILU  u * s(u);  s(z) = 1 / (1 + exp(-z)).
 *
 * Memory, streams, errors: as in moccasin.h.  All pointers but the descriptors
 * are device pointers; descriptors are read before the call returns.  Calls
 * allocate nothing and are asynchronous on the given stream; those that need a
 * workspace say how many bytes (moc_*_work), 16-byte aligned; it may be used
 * again as soon as later work on the same stream may write to it.  The calls
 * can be captured into a graph.  Arguments are checked before anything is
 * queued.  An output may be the same memory as an input only where said.
 */
#ifndef MOCCASIN_TRAINING_H
#define MOCCASIN_TRAINING_H

#include <stdint.h>

#include "moccasin.h" /* error codes, moc_strerror, moc_last_hip_error */

#ifdef __cplusplus
extern "C" {
#endif

#define MOC_TRAINING_VERSION 3

#define MOC_F32  0
#define MOC_F16  1
#define MOC_BF16 2
#define MOC_E4M3 3 /* checkpoint */
#define MOC_I8   4 /* checkpoint */

#define MOC_ACT_NONE 0
#define MOC_ACT_RELU 1
#define MOC_ACT_GELU 2
#define MOC_ACT_SILU 3

#define MOC_BLOCK 32 /* columns that share a scale */

/* Largest number of rows, columns and elements from one row to the next. */
#define MOC_MAX_ROWS   2147483136ll
#define MOC_MAX_COLS   4194240ll
#define MOC_MAX_STRIDE 4194240ll

typedef struct {
  void* data;           /* value (0, 0) */
  uint8_t* scales;      /* checkpoints only */
  int64_t stride;       /* elements from one row to the next, >= cols, <= MOC_MAX_STRIDE */
  int64_t scale_stride; /* checkpoints: bytes from one row's scales to the next, >= ceil(cols / 32), <= MOC_MAX_STRIDE */
  int32_t type;         /* MOC_F32 .. MOC_I8 */
  int32_t reserved;     /* 0 */
} moc_matrix;

/*
 * Keep x [rows][cols] (float32, float16, bfloat16) as the checkpoint `kept`.
 * rows == 0 or cols == 0 is a no-op.  Errors: MOC_EINVAL, MOC_EHIP.
 */
int moc_checkpoint_write(int64_t rows, int64_t cols, const moc_matrix* x, const moc_matrix* kept, void* hip_stream);

/*
 * out = act(kept), rounded once to out's type: the values a checkpoint stands
 * for, or an activation computed again from its kept argument.
 * Errors: MOC_EINVAL, MOC_EHIP.
 */
int moc_checkpoint_read(int64_t rows, int64_t cols, const moc_matrix* kept, int32_t act, const moc_matrix* out,
                        void* hip_stream);

/*
 * Layer norm over the columns: per row, mean and variance (biased) of x, rstd =
 * 1 / sqrt(variance + eps), y = (x - mean) * rstd * gamma + beta.
 *   x           a tensor or a checkpoint
 *   gamma, beta device, [cols] of param_type (float32, float16, bfloat16);
 *               NULL: 1 and 0
 *   eps         >= 0
 *   y           float32, float16 or bfloat16; may be x's own memory (same
 *               type and stride)
 *   kept        a checkpoint that y is written to before its rounding to y's
 *               type, in the same pass (its E is that of y's type), or NULL
 *   mean, rstd  device, float [rows]
 * cols >= 1; rows == 0 is a no-op.  Sums are held in 32 bits, the variance is
 * that of the differences from the mean.  Errors: MOC_EINVAL, MOC_EHIP.
 */
int moc_norm_forward(int64_t rows, int64_t cols, const moc_matrix* x, const void* gamma, const void* beta,
                     int32_t param_type, float eps, const moc_matrix* y, const moc_matrix* kept, float* mean, float* rstd,
                     void* hip_stream);

/*
 * Layer norm's gradients, with h = (x - mean) * rstd and p = dy * gamma:
 *   dx = rstd * (p - mean(p) - h * mean(p * h)) + residual
 *   dgamma = sum over rows of dy * h,  dbeta = sum over rows of dy
 *   dy        float32, float16 or bfloat16
 *   x         as it was given to moc_norm_forward, of dy's type, or a
 *             checkpoint of it
 *   residual  of dy's type, added to dx (the gradient of a branch around the
 *             norm), or NULL
 *   dx        of dy's type; may be dy's, x's or residual's own memory (same stride)
 *   dgamma, dbeta  device, float [cols]; both or neither (NULL).  With rows ==
 *             0 they are set to zero.
 *   work      moc_norm_backward_work(rows, cols) bytes; NULL without dgamma
 * Errors: MOC_EINVAL, MOC_EHIP.
 */
int64_t moc_norm_backward_work(int64_t rows, int64_t cols);
int moc_norm_backward(int64_t rows, int64_t cols, const moc_matrix* dy, const moc_matrix* x, const void* gamma,
                      int32_t param_type, const float* mean, const float* rstd, const moc_matrix* residual,
                      const moc_matrix* dx, float* dgamma, float* dbeta, void* work, int64_t work_bytes,
                      void* hip_stream);

/*
 * y = act(u) + residual, u = x w^T + bias.
 *   x         [rows][cin], float16 or bfloat16
 *   w         [cout][cin], x's type
 *   bias      device, [cout] of bias_type (float32, float16, bfloat16), or NULL
 *   residual  [rows][cout], x's type or float32, or NULL
 *   y         [rows][cout], x's type or float32; may be the residual's own
 *             memory (same type and stride)
 *   kept      a checkpoint that u is written to (its E is that of x's type),
 *             or NULL
 *   work      moc_linear_work bytes (may be 0)
 * Products are exact, sums are held in 32 bits; u is rounded once to the
 * checkpoint, act(u) + residual once to y.  cin == 0: u = bias.
 * Errors: MOC_EINVAL, MOC_EOVERFLOW, MOC_EHIP.
 */
int moc_linear_forward(int64_t rows, int64_t cin, int64_t cout, const moc_matrix* x, const moc_matrix* w, const void* bias,
                       int32_t bias_type, int32_t act, const moc_matrix* residual, const moc_matrix* y,
                       const moc_matrix* kept, void* work, int64_t work_bytes, void* hip_stream);

/*
 * dx = (dy w) * act'(pre): the gradient with regard to the layer's input, and,
 * where that input is act(pre), on to pre.
 *   dy   [rows][cout], float16 or bfloat16;  w  [cout][cin], dy's type
 *   pre  [rows][cin], a tensor of dy's type or float32, or a checkpoint; NULL
 *        with MOC_ACT_NONE only.  Where pre is NaN, dx is NaN; act' of
 *        MOC_ACT_RELU is 0 at pre <= 0 whatever dy is.
 *   dx   [rows][cin], dy's type or float32; may be pre's own memory (same type
 *        and stride)
 * Errors: MOC_EINVAL, MOC_EOVERFLOW, MOC_EHIP.
 */
int moc_linear_backward_input(int64_t rows, int64_t cin, int64_t cout, const moc_matrix* dy, const moc_matrix* w,
                              int32_t act, const moc_matrix* pre, const moc_matrix* dx, void* work, int64_t work_bytes,
                              void* hip_stream);

/*
 * dw = dy^T x, db = sum over rows of dy.
 *   dy   [rows][cout], float16 or bfloat16
 *   x    [rows][cin], a tensor of dy's type or a checkpoint (its values are
 *        taken in dy's type)
 *   dw   [cout][cin], float32 or dy's type
 *   db   device, float [cout], or NULL
 * rows == 0 sets dw and db to zero.  Errors: MOC_EINVAL, MOC_EOVERFLOW, MOC_EHIP.
 */
int moc_linear_backward_weight(int64_t rows, int64_t cin, int64_t cout, const moc_matrix* dy, const moc_matrix* x,
                               const moc_matrix* dw, float* db, void* work, int64_t work_bytes, void* hip_stream);

/* Bytes of workspace that the three calls above need for these sizes on the
 * current device (the largest of the three), or a negative error code. */
int64_t moc_linear_work(int64_t rows, int64_t cin, int64_t cout);

/*
 * How a product is cut up, for tests and tuning: no device is used where `units` says for how many compute units (0: the
 * current device's).
 *   product  which call: MOC_LINEAR_FORWARD, MOC_LINEAR_BACKWARD_INPUT or MOC_LINEAR_BACKWARD_WEIGHT
 *   aligned  whether operands start on 16 bytes and strides are multiples of 8 elements (of a checkpoint 16, and cin too)
 *   out      host, [5]: rows and columns of the output that a workgroup computes; 1 where operands go straight into LDS, else
 *            0; the parts that the sum is cut into; terms of a part; terms of the last one
 * Errors: MOC_EINVAL, MOC_EHIP.
 */
#define MOC_LINEAR_FORWARD         0
#define MOC_LINEAR_BACKWARD_INPUT  1
#define MOC_LINEAR_BACKWARD_WEIGHT 2
int moc_linear_parts(int32_t product, int64_t rows, int64_t cin, int64_t cout, int32_t aligned, int32_t units, int64_t* out);

/*
 * The residual connection between two blocks:
 *   h = after(block), or block     the norm behind the block
 *   r = scale * x + gate h         the stream; without x: gate h
 *   n = before(r)                  the norm before the next block, of r as it is before its rounding
 * A norm is layer norm as above, or by the root of the squares alone, gamma * v /
 * sqrt(mean(v^2) + eps).
 *   x       float32, float16 or bfloat16, or NULL
 *   block   a tensor or a checkpoint
 *   gate    [gates][cols] of values: row i takes row i / (rows / gates); gates
 *           divides rows.  NULL with 0 gates
 *   after, before  NULL or of kind MOC_NORM_NONE: none
 *   r       NULL: not kept; may be x's or the block's own memory (same type and stride)
 *   n       NULL without `before`; may be x's or the block's own memory, but not r's
 *   kept    a checkpoint that n is written to before its rounding (its E is that of
 *           n's type), or NULL
 * cols 1 .. MOC_RESIDUAL_MAX_COLS; rows == 0 is a no-op; r or n is wanted.  Statistics
 * and sums are held in 32 bits.  Errors: MOC_EINVAL, MOC_EHIP.
 */
#define MOC_NORM_NONE  0
#define MOC_NORM_LAYER 1
#define MOC_NORM_RMS   2

#define MOC_RESIDUAL_MAX_COLS 16384

typedef struct {
  int32_t kind;             /* MOC_NORM_NONE .. MOC_NORM_RMS */
  int32_t param_type;       /* float32, float16, bfloat16 */
  const void *gamma, *beta; /* device, [cols]; NULL: 1 and 0; MOC_NORM_RMS has no beta */
  float *mean, *rstd;       /* device, [rows]: written by the forward, read by the backward pass; MOC_NORM_RMS has no mean */
  float eps;                /* >= 0 */
  int32_t reserved;         /* 0 */
} moc_row_norm;

int moc_residual_forward(int64_t rows, int64_t cols, const moc_matrix* x, const moc_matrix* block, const moc_matrix* gate,
                         int64_t gates, float scale, const moc_row_norm* after, const moc_row_norm* before,
                         const moc_matrix* r, const moc_matrix* n, const moc_matrix* kept, void* hip_stream);

/*
 * Its gradients.  With norm' a norm's gradient as above (without the mean's
 * part for MOC_NORM_RMS):
 *   d = dr + before'(dn),  dx = scale * d,  dgate = sum over a gate's rows of d h,
 *   dblock = after'(gate d), or gate d
 *   dr      the stream's gradient, or NULL;  dn  n's, NULL without `before`; one of them is there
 *   r       as the forward pass has left it, or a checkpoint of it; looked at with `before` only
 *   block   as it was given to the forward pass; looked at with `after` or for dgate
 *   dx, dblock  values, NULL: not wanted.  dx may be dr's or r's own memory, dblock dn's or the block's (same type and
 *           stride), but not each other's
 *   grads   the parameters' gradients, device, float [cols] (gate: [gates][cols]),
 *           or NULL; each NULL: not wanted.  With rows == 0 they are set to zero.
 *   work    moc_residual_backward_work bytes; not needed without grads
 * Errors: MOC_EINVAL, MOC_EHIP.
 */
typedef struct {
  float *before_gamma, *before_beta, *after_gamma, *after_beta, *gate;
} moc_residual_grads;

int64_t moc_residual_backward_work(int64_t rows, int64_t cols, int64_t gates);
int moc_residual_backward(int64_t rows, int64_t cols, const moc_matrix* dr, const moc_matrix* dn, const moc_matrix* r,
                          const moc_matrix* block, const moc_matrix* gate, int64_t gates, float scale,
                          const moc_row_norm* after, const moc_row_norm* before, const moc_matrix* dx,
                          const moc_matrix* dblock, const moc_residual_grads* grads, void* work, int64_t work_bytes,
                          void* hip_stream);

/*
 * Log probabilities of rows of logits, z = scale * logits:
 *   lse = log sum over the columns of exp(z),  logp = z[token] - lse,
 *   entropy = lse - sum of p z  with p = exp(z - lse),
 * and the `top` most likely columns: the largest logits in falling order, equal
 * ones by column (-0 equals 0).
 *   logits  [rows][vocab], float32, float16 or bfloat16
 *   scale   2^-64 .. 2^64 (of a temperature, its inverse)
 *   tokens  device, [rows] of token_bytes (4 or 8), signed, or NULL.  Below 0: no
 *           token, logp is 0 and has no gradient; from vocab on: logp and the
 *           row's gradient are NaN
 *   top     0 .. 64, at most vocab
 *   logp    device, float [rows], NULL without tokens;  lse, entropy  float [rows]
 *   top_logp, top_tokens  device, float and int64 [rows][top], NULL where top is 0
 *   work    moc_logprob_forward_work(rows, vocab, top) bytes (may be 0)
 * Logits of -infinity have p = 0; a p below 2^-126 may count as 0.  A row of nothing else: lse and logp
 * -infinity, entropy 0, no gradient.  A row with NaN or +infinity: all NaN, columns -1.
 * Sums are held in 32 bits.  vocab >= 1; rows == 0 is a no-op.
 * Errors: MOC_EINVAL, MOC_EHIP.
 */
int64_t moc_logprob_forward_work(int64_t rows, int64_t vocab, int32_t top);
int moc_logprob_forward(int64_t rows, int64_t vocab, const moc_matrix* logits, const void* tokens, int32_t token_bytes,
                        float scale, int32_t top, float* logp, float* lse, float* entropy, float* top_logp,
                        int64_t* top_tokens, void* work, int64_t work_bytes, void* hip_stream);

/*
 * The gradient of logp and entropy with regard to the logits:
 *   out = scale * (dlogp * ([column == token] - p) - dentropy * p * (z - lse + entropy))
 *   lse, entropy     as the forward pass has left them; entropy NULL without dentropy.  p
 *                    is off by what lse is, of itself; of rows with lse beyond 1024 either
 *                    way the sum is taken again from the logits, by one workgroup
 *   tokens, dlogp    device, float [rows]: both or neither
 *   dentropy         device, float [rows], or NULL
 *   out              [rows][vocab], the logits' type or float32; may be the logits' own
 *                    memory (same type and stride)
 * Errors: MOC_EINVAL, MOC_EHIP.
 */
int moc_logprob_backward(int64_t rows, int64_t vocab, const moc_matrix* logits, const float* lse, const float* entropy,
                         const void* tokens, int32_t token_bytes, const float* dlogp, const float* dentropy, float scale,
                         const moc_matrix* out, void* hip_stream);

/*
 * AdamW over many tensors at once, in place:
 *   g = grad_scale * grad
 *   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
 *   param -= lr * decay * param + lr / (1 - beta1^step) * m / (sqrt(v / (1 - beta2^step)) + eps)
 * computed in 32 bits from what is stored, param and `copy` rounded once from
 * the result.
 *
 * Moments are float32, or take 8 bits (moment_type MOC_E4M3): 32 consecutive
 * values of the tensor share a scale 2^k, held as the byte k + 127 at
 * scales[place / 32], with k as in a checkpoint in MOC_E4M3.  A code of m is one
 * of MOC_E4M3; a code of v has no sign, 5 exponent and 3 fraction bits, is
 * normal from 2^-22 on, 448 at its largest (254), and 255 is NaN.  Zeroed codes
 * and scales are zeros.  v changes by a thousandth a step and codes are 6 to 12 %
 * apart, so nearest codes would never fall: a value between two codes goes to
 * the upper one where its distance from the lower, in parts of 2^20 of the
 * codes' distance and rounded down, plus 16 b + 8 reaches 2^20, with b 16 random bits;
 * the mean of what is stored is the value.  A positive v takes no code below
 * 1.  What is not finite becomes NaN; magnitudes above 1.875 * 2^127 are taken for
 * that.  Random bits of the value at place i of the tensor of number t:
 *   mix(low(i) ^ mix(high(i) ^ mix(t ^ mix(low(step) ^ mix(high(seed) ^ mix(low(seed)))))))
 * with low and high halves of 32 bits, the lower 16 for m, the upper for v, and
 *   mix(h):  h ^= h >> 16, h *= 0xF704BB15, h ^= h >> 15, h *= 0x371E2E67, h ^= h >> 16.
 * t counts within a call: calls of one step (groups of parameters with rates of their
 * own) need seeds of their own, or their tensors are rounded by the same bits.
 *
 * v below 2^-126 may count as 0.  All memory that is written is apart from all
 * other memory of the call.  A tensor of no values is left out.  No tensors:
 * a no-op.  Errors: MOC_EINVAL, MOC_EHIP.
 */
typedef struct {
  void* param;          /* device, [count], contiguous, float32, float16 or bfloat16 */
  const void* grad;     /* the same of grad_type */
  void *m, *v;          /* float32, or bytes */
  uint8_t *m_scales, *v_scales; /* 8 bits: ceil(count / 32) bytes each */
  void* copy;           /* param's new values in copy_type (float16 or bfloat16), or NULL */
  int64_t count;
  int32_t param_type, grad_type;
  int32_t moment_type;  /* MOC_F32, or MOC_E4M3 for 8 bits */
  int32_t copy_type;
  float decay;          /* >= 0 */
  int32_t reserved;     /* 0 */
} moc_adamw_tensor;

typedef struct {
  double lr, beta1, beta2, eps;   /* finite in float; 0 <= beta < 1; eps >= 2^-126 */
  double grad_scale;
  int64_t step;                   /* >= 1 */
  uint64_t seed;                  /* of moments in 8 bits */
  const float* lr_at;             /* device: read instead of lr, or NULL */
  const float* grad_scale_at;     /* device: read instead of grad_scale, or NULL */
  const int64_t* step_at;         /* device: read instead of step, or NULL (a captured call finds each replay's step there) */
} moc_adamw_rule;

int moc_adamw_step(int64_t tensors, const moc_adamw_tensor* tensor, const moc_adamw_rule* rule, void* hip_stream);

/*
 * What moments stand for: m and v of each tensor as values.
 *   m, v, scales, count, moment_type  as above
 *   m_values, v_values  device, [count] of value_type (float32 or bfloat16, which
 *                       have every value of a code; float16)
 * Errors: MOC_EINVAL, MOC_EHIP.
 */
typedef struct {
  const void *m, *v;
  const uint8_t *m_scales, *v_scales;
  void *m_values, *v_values;
  int64_t count;
  int32_t moment_type, value_type;
} moc_moments_tensor;
int moc_moments_read(int64_t tensors, const moc_moments_tensor* tensor, void* hip_stream);

/* The MOC_TRAINING_VERSION that the library was built with. */
int moc_training_version(void);

#ifdef __cplusplus
}
#endif
#endif /* MOCCASIN_TRAINING_H */
