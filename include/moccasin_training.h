/*
 * moccasin_training.h -- C ABI of the operators that a rematerialisation plan
 * is run with (libmoccasin_hip.so, next to moccasin.h): activation checkpoints
 * in 8 bits, layer norm, linear layers, and their gradients, on one AMD MI355X
 * (gfx950).
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

#define MOC_TRAINING_VERSION 2

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

/* The MOC_TRAINING_VERSION that the library was built with. */
int moc_training_version(void);

#ifdef __cplusplus
}
#endif
#endif /* MOCCASIN_TRAINING_H */
