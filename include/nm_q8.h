/*
 * nm_q8.h -- C ABI of libnmconv: the operators of a feed-forward layer in 8-bit integers.
 *
 * Tensors are rows (tokens) of `width` values, one row after another at a row stride
 * that the caller gives in elements, values of a row adjacent.  A row in 8 bits is
 * whole numbers q in [-127, 127] and one fp32 scale s; it stands for the values q * s.
 * Weights in 8 bits have one scale for each output channel.
 *
 * Conventions are those of nm_conv.h: NM_OK or a negative nm_status_t, nm_last_error()
 * for the description, no exception crosses the boundary, device pointers are the
 * caller's, calls enqueue on `hip_stream` (a hipStream_t, NULL = default stream) of the
 * calling thread's current device, allocate nothing and never wait, and may be captured
 * into a graph -- except nm_q8_pack and the exports, which are synchronous.
 *
 * Rows, widths and strides: 0 <= rows <= 2^30 (a call with no rows checks its
 * arguments and enqueues nothing), 1 <= width <= NM_Q8_MAX_WIDTH.  An input's rows may
 * overlap or be one and the same (stride 0); an output's must not.  Strides are at most
 * 2^24 elements.  fp32 and bf16 pointers need the alignment of their element only.
 *
 * Not-a-number and infinity: a row whose values (or, for the norm, whose sum of
 * squares) are not finite in fp32 gets q = 0 and s = NaN, so everything computed from
 * it is NaN, and no other row is touched.  A row whose largest magnitude (for the norm:
 * that of v) is below 1.5e-36 (127 times the smallest normal fp32 number) counts as
 * zero: q = 0, s = 0.  A norm divides by sqrt(mean(h^2) + eps), held to fp32 precision down
 * to 1.5e-36 (2^-119); a row for which it is below that, as for a zero row with eps = 0,
 * has no norm: q = 0, s = NaN.
 */
#ifndef NM_Q8_H
#define NM_Q8_H

#include "nm_conv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element type of 8-bit integers, next to NM_F32 and NM_BF16; only the calls of this header know it. */
enum { NM_I8 = 3 };

/* Longest row: sums of up to this many products of 8-bit integers are exact in 32 bits. */
enum { NM_Q8_MAX_WIDTH = 65536 };

/*
 * nm_quantize_q8 -- every row rounded to 8 bits under its own scale:
 *   a = max |x_i|,  s = a / 127,  q_i = x_i * 127 / a rounded to the nearest, ties to even
 *   Of bf16 values that is exact.  Of fp32 values, a quotient not half way between two whole numbers but within 4e-6 of
 *   it may go to either.
 *   x_dev      rows of x_dtype (NM_F32 or NM_BF16) at stride ldx, only read
 *   q_dev      int8 rows at stride ldq >= width, fully overwritten (gaps between rows are not touched)
 *   scales_dev fp32 [rows]
 * Errors: NM_ERR_ARG, NM_ERR_SHAPE (width), NM_ERR_HIP.
 */
int nm_quantize_q8(const void* x_dev, nm_dtype_t x_dtype, int64_t rows, int width, int64_t ldx,
                   int8_t* q_dev, int64_t ldq, float* scales_dev, void* hip_stream);

/*
 * nm_dequantize_q8 -- the values that 8-bit rows stand for: y = q * s, in fp32, rounded
 * to nearest even once if y_dtype is NM_BF16.
 */
int nm_dequantize_q8(const int8_t* q_dev, int64_t ldq, const float* scales_dev, int64_t rows, int width,
                     void* y_dev, nm_dtype_t y_dtype, int64_t ldy, void* hip_stream);

/*
 * nm_rmsnorm_q8 -- residual addition, root-mean-square norm and rounding to 8 bits in one pass:
 *   h = x + residual                      (h = x without one), formed in fp32
 *   v_i = gamma_i * h_i / sqrt(mean_i(h_i^2) + eps)
 *   q, s = the row v rounded as by nm_quantize_q8 (q: to the nearest within the fp32 errors of v)
 *   residual_out = h rounded to x_dtype   (the residual stream that the next layer adds to)
 * The norm is taken of h before that rounding; sums are fp32.
 *   residual_dev      rows of x_dtype at stride ldr, or NULL
 *   gamma_dev         fp32 [width], or NULL for 1
 *   eps               finite, >= 0
 *   residual_out_dev  rows of x_dtype at stride ldo >= width, or NULL.  It may be x_dev or
 *                     residual_dev itself (same pointer and stride); any other overlap of an
 *                     output with an input is an error.
 */
int nm_rmsnorm_q8(const void* x_dev, nm_dtype_t x_dtype, int64_t rows, int width, int64_t ldx,
                  const void* residual_dev, int64_t ldr, const float* gamma_dev, float eps,
                  void* residual_out_dev, int64_t ldo, int8_t* q_dev, int64_t ldq, float* scales_dev,
                  void* hip_stream);

/* Weights of one product in 8 bits, laid out for the kernels.  Opaque, owned by the library, immutable
 * after creation, bound to the device that was current in nm_q8_pack. */
typedef struct nm_q8 nm_q8_t;

/*
 * nm_q8_pack -- lays out w[channels][width] (row stride ldw elements) for nm_linear_q8.
 *   w_dtype    NM_I8: w is taken as it is, with scales_dev [channels].
 *              NM_F32 or NM_BF16: each channel is rounded as a row by nm_quantize_q8; scales_dev must be NULL.
 *   gated      1: the first half of the channels are the gates of the second half (channels must be even)
 *   out        receives the handle; free it with nm_q8_free
 * Weights pruned by nm_prune keep their zeros here; they are not skipped.
 * Errors: NM_ERR_ARG (also: a weight or a scale that is not finite), NM_ERR_SHAPE, NM_ERR_ALLOC, NM_ERR_HIP.
 * Runs after the work already on hip_stream and waits for it; not under stream capture.
 */
int nm_q8_pack(const void* w_dev, nm_dtype_t w_dtype, const float* scales_dev, int channels, int width, int64_t ldw,
               int gated, void* hip_stream, nm_q8_t** out);

int nm_q8_free(nm_q8_t* w);

/* Sizes as given to nm_q8_pack.  Any out pointer may be NULL. */
int nm_q8_dims(const nm_q8_t* w, int* channels, int* width, int* gated);

/* The 8-bit weights [channels][width] and their scales [channels] in caller-allocated host buffers (either may be NULL). */
int nm_q8_export(const nm_q8_t* w, int8_t* w_host, float* scales_host);

/*
 * nm_linear_q8 -- y = product of 8-bit rows with 8-bit weights, a scale for each row and each channel:
 *   a_rc = sum_k q_rk * w_ck                     exact, in 32-bit integers
 *   z_rc = a_rc * (s_r * t_c) + bias_c           fp32
 *   y_rc = z_rc + residual_rc                    plain weights
 *   y_rc = z_rc / (1 + exp(-z_rc)) * z_r,(c+C)   gated weights of 2 C channels (no residual)
 * rounded to nearest even once if y_dtype is NM_BF16.  The result does not depend on the
 * other rows of the call nor on how the sum was divided.
 *   q_dev, ldq      int8 rows of the weights' width at any stride >= 0, any alignment.  Gaps between rows may be read too, and so are
 *                   the aligned 16 bytes that hold the last row's last value; what they hold changes no result.
 *   scales_dev      fp32 [rows]
 *   bias_dev        fp32 [channels] (gated: gates first, as the weights), or NULL
 *   residual_dev    rows of y_dtype at stride ldr, or NULL.  It may be y_dev itself (same stride).
 *   y_dev           rows of y_dtype (NM_F32 or NM_BF16) at stride ldy >= channels (gated: channels / 2)
 *   workspace_dev   at least nm_linear_q8_workspace() bytes, 16-byte aligned; its contents need
 *                   not be kept between calls.  Calls that overlap in time need one each.
 * Errors: NM_ERR_ARG (also: workspace too small), NM_ERR_SHAPE, NM_ERR_UNSUPPORTED (gated with a residual), NM_ERR_HIP.
 */
int nm_linear_q8(const int8_t* q_dev, int64_t rows, int width, int64_t ldq, const float* scales_dev, const nm_q8_t* w,
                 const float* bias_dev, const void* residual_dev, int64_t ldr, void* y_dev, nm_dtype_t y_dtype,
                 int64_t ldy, void* workspace_dev, size_t workspace_bytes, void* hip_stream);

/* Bytes of workspace that nm_linear_q8 needs for these arguments: for rows that do not start at multiples of 16 bytes (address and, with
 * more than one row, stride), and for sums divided over workgroups.  0 for up to NM_Q8_FEW_ROWS rows that do start there. */
enum { NM_Q8_FEW_ROWS = 64 };
int nm_linear_q8_workspace(const int8_t* q_dev, int64_t rows, int64_t ldq, const nm_q8_t* w, size_t* bytes);

/*
 * The calls above with their arguments in one block, for bindings that pay for every argument (as nm_conv2d_args).  dtype is
 * x_dtype or y_dtype.  norm = 0 is nm_quantize_q8, which looks at neither residual, gamma, eps nor residual_out.
 */
typedef struct nm_rows_q8_args {
    const void* x_dev;
    const void* residual_dev;
    const float* gamma_dev;
    void* residual_out_dev;
    int8_t* q_dev;
    float* scales_dev;
    void* hip_stream;
    int64_t dtype, rows, width, ldx, ldr, ldo, ldq, norm;
    double eps;
} nm_rows_q8_args_t;
int nm_rows_q8_args(const nm_rows_q8_args_t* args);

typedef struct nm_dequantize_q8_args {
    const int8_t* q_dev;
    const float* scales_dev;
    void* y_dev;
    void* hip_stream;
    int64_t dtype, rows, width, ldq, ldy;
} nm_dequantize_q8_args_t;
int nm_dequantize_q8_args(const nm_dequantize_q8_args_t* args);

typedef struct nm_linear_q8_args {
    const int8_t* q_dev;
    const float* scales_dev;
    const nm_q8_t* w;
    const float* bias_dev;
    const void* residual_dev;
    void* y_dev;
    void* workspace_dev;
    void* hip_stream;
    int64_t dtype, rows, width, ldq, ldr, ldy, workspace_bytes;
} nm_linear_q8_args_t;
int nm_linear_q8_args(const nm_linear_q8_args_t* args);

#ifdef __cplusplus
}
#endif
#endif /* NM_Q8_H */
