/*
 * nm_mx4.h -- C ABI of libnmconv: feed-forward operators in microscaled 4-bit floating point, with or without experts.
 *
 * A row in MX4 is blocks of 32 adjacent values.  A value is a sign, two bits of exponent and one of mantissa: 0, 0.5, 1,
 * 1.5, 2, 3, 4 or 6 (codes 0 to 7; 8 to 15 the same with the sign), two to a byte, the even one in the low half, 16 bytes a
 * block.  A block has one byte b for the power of two 2^(b - 127) that its values are multiplied with; 255 makes them all NaN.
 * A row of `width` values has B = ceil(width / 32) blocks: 16 B bytes of codes and B bytes of scales.  The codes past the
 * width in the last block are written as zeros and not looked at.
 *
 * Tensors are rows at a stride that the caller gives, in elements (codes and scales: in bytes).  Codes start at multiples
 * of 16 bytes, in address and stride; scales, fp32 and bf16 need the alignment of their element only.  Conventions are
 * otherwise those of nm_q8.h: 0 <= rows <= 2^30 (a call with no rows checks its arguments and enqueues nothing),
 * 1 <= width <= NM_MX4_MAX_WIDTH, strides up to 2^24, an input's rows may overlap or be one and the same (stride 0), an
 * output's must not, and no output may overlap an input but where that is said.  Calls enqueue on `hip_stream` of the
 * current device, allocate nothing and never wait, and may be captured into a graph -- except nm_mx4_pack and the exports,
 * which are synchronous.  Inference only: there are no gradients.
 */
#ifndef NM_MX4_H
#define NM_MX4_H

#include "nm_q8.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element type of rows in MX4, next to NM_F32 and NM_BF16; only the calls of this header know it. */
enum { NM_MX4 = 4 };
enum { NM_MX4_MAX_WIDTH = 65536, NM_MX4_MAX_EXPERTS = 1024 };

/*
 * nm_quantize_mx4 -- every block rounded under its own power of two:
 *   a = max |x_i| of the block,  e = max(floor(log2(a)) - 2, -127)  (a = 0: -127),  scale byte e + 127
 *   code of x_i * 2^-e rounded to the nearest, ties to the even code, at most 6 (exact: no other rounding comes in)
 * A block that holds a NaN or an infinity gets codes of 0 and the scale byte 255.
 *   x_dev      rows of x_dtype (NM_F32 or NM_BF16) at stride ldx, only read
 *   q_dev      codes at stride ldq >= 16 B; scales_dev at stride lds >= B.  Gaps between rows are not touched.
 */
int nm_quantize_mx4(const void* x_dev, nm_dtype_t x_dtype, int64_t rows, int width, int64_t ldx,
                    uint8_t* q_dev, int64_t ldq, uint8_t* scales_dev, int64_t lds, void* hip_stream);

/* nm_dequantize_mx4 -- the values that rows in MX4 stand for (exact in fp32 and in bf16: powers below bf16's range as its subnormals). */
int nm_dequantize_mx4(const uint8_t* q_dev, int64_t ldq, const uint8_t* scales_dev, int64_t lds, int64_t rows, int width,
                      void* y_dev, nm_dtype_t y_dtype, int64_t ldy, void* hip_stream);

/*
 * nm_rmsnorm_mx4 -- residual addition, root-mean-square norm and rounding in one pass:
 *   h = x + residual                             (h = x without one), formed in fp32
 *   n = 1 / sqrt(mean_i(h_i^2) + eps)            the mean and the root in 64 bits, n rounded to fp32
 *   v_i = (h_i * n) * gamma_i                    fp32, two roundings
 *   q, scales = v as by nm_quantize_mx4;  residual_out = h rounded to x_dtype
 * A power of two decides about a whole block, so the sum and n are held in 64 bits until the end: another order of summation then
 * gives another n, and with it perhaps other codes, in some rows of 10^8 (in 32 bits it would in most).  A row for which n is not
 * finite (a zero row with eps = 0) becomes NaN.
 *   gamma_dev         fp32 [width], or NULL for 1;  eps finite, >= 0
 *   residual_out_dev  rows of x_dtype at stride ldo >= width, or NULL.  It may be x_dev or residual_dev itself (same stride).
 */
int nm_rmsnorm_mx4(const void* x_dev, nm_dtype_t x_dtype, int64_t rows, int width, int64_t ldx,
                   const void* residual_dev, int64_t ldr, const float* gamma_dev, double eps,
                   void* residual_out_dev, int64_t ldo, uint8_t* q_dev, int64_t ldq, uint8_t* scales_dev, int64_t lds,
                   void* hip_stream);

/* Weights in MX4 of one product or of several experts' products, laid out for the kernels.  Opaque, owned by the library,
 * immutable after creation, bound to the device that was current in nm_mx4_pack. */
typedef struct nm_mx4 nm_mx4_t;

/*
 * nm_mx4_pack -- lays out w[experts * channels][width] (row stride ldw) for nm_linear_mx4 (1 expert) and nm_experts_mx4.
 *   w_dtype    NM_MX4: codes, with scales_dev at stride lds.
 *              NM_F32 or NM_BF16: each row is rounded as by nm_quantize_mx4; scales_dev must be NULL.
 *   gated      1: of each expert's channels the first half are the gates of the second half (channels must be even)
 *   out        receives the handle; free it with nm_mx4_free
 * Errors: NM_ERR_ARG (also: a weight that is not finite), NM_ERR_SHAPE, NM_ERR_ALLOC, NM_ERR_HIP.
 * Runs after the work already on hip_stream and waits for it; not under stream capture.
 */
int nm_mx4_pack(const void* w_dev, nm_dtype_t w_dtype, const uint8_t* scales_dev, int64_t lds, int experts, int channels,
                int width, int64_t ldw, int gated, void* hip_stream, nm_mx4_t** out);

/* Not before the work that reads it has ended (device memory is freed); other streams may be under capture. */
int nm_mx4_free(nm_mx4_t* w);

/* Sizes as given to nm_mx4_pack.  Any out pointer may be NULL. */
int nm_mx4_dims(const nm_mx4_t* w, int* experts, int* channels, int* width, int* gated);

/* The codes [experts][channels][16 B] and scales [experts][channels][B] in caller-allocated host buffers (either may be NULL). */
int nm_mx4_export(const nm_mx4_t* w, uint8_t* q_host, uint8_t* scales_host);

/*
 * nm_linear_mx4 -- rows in MX4 times weights in MX4:
 *   z_rc = sum_k x_rk * w_ck + bias_c            products exact, sums in fp32
 *   y_rc = z_rc + residual_rc                    plain weights
 *   y_rc = z_rc / (1 + exp(-z_rc)) * z_r,(c+C)   gated weights of 2 C channels (no residual), of the sums z within (2 |z_rc| + 12) 2^-24 of
 *                                                itself (or 2^-148) before it is rounded to y's type; 0 for gates below -174.7
 * rounded once to y_dtype: NM_F32, NM_BF16 (nearest even) or NM_MX4 (as by nm_quantize_mx4 of the fp32 values; no residual).
 * Calls with the same arguments give the same bits.  A row with a NaN gives a row of NaN and touches no other.
 *   q_dev, ldq, scales_dev, lds    rows of the weights' width
 *   bias_dev        fp32 [channels] (gated: gates first, as the weights), or NULL
 *   residual_dev    rows of y_dtype at stride ldr, or NULL.  It may be y_dev itself (same stride).
 *   y_dev           rows of y_dtype at stride ldy (NM_MX4: codes; y_scales_dev at stride ldys, otherwise NULL)
 * Errors: NM_ERR_ARG, NM_ERR_SHAPE, NM_ERR_UNSUPPORTED (a residual with gated weights or with
 * an output in MX4; weights of several experts), NM_ERR_HIP.
 */
int nm_linear_mx4(const uint8_t* q_dev, int64_t ldq, const uint8_t* scales_dev, int64_t lds, int64_t rows, int width,
                  const nm_mx4_t* w, const float* bias_dev, const void* residual_dev, int64_t ldr, void* y_dev,
                  nm_dtype_t y_dtype, int64_t ldy, uint8_t* y_scales_dev, int64_t ldys, void* hip_stream);

/*
 * nm_experts_mx4 -- products grouped by expert: row r of y, for offsets[e] <= r < offsets[e + 1], is the formula of
 * nm_linear_mx4 with expert e's weights and bias, of row r of x, or of row index[r] where an index is given.
 *   offsets_dev     int32 [experts + 1] on the device, not falling, from 0 to at most `entries` (as nm_route writes them).
 *                   Groups may be empty.  Values outside [0, entries] count as the nearer end, a group that ends before
 *                   it begins as empty.  Rows of y in no group are left as they were.  Where offsets fall, groups
 *                   overlap, and what y's rows in any group hold is not defined: parts of one group's answer and of
 *                   another's, or what was there.  Nothing else is written.
 *   index_dev       int32 [entries], or NULL.  An index outside [0, rows) makes its row of y NaN.
 *   entries         rows of y (without an index: also of x, rows = entries)
 *   bias_dev        fp32 [experts][channels], or NULL
 * With an index the rows of x span less than 4 GiB.
 */
int nm_experts_mx4(const uint8_t* q_dev, int64_t ldq, const uint8_t* scales_dev, int64_t lds, int64_t rows, int width,
                   const nm_mx4_t* w, const int32_t* offsets_dev, const int32_t* index_dev, int64_t entries,
                   const float* bias_dev, void* y_dev, nm_dtype_t y_dtype, int64_t ldy, uint8_t* y_scales_dev, int64_t ldys,
                   void* hip_stream);

/*
 * The calls above with their arguments in one block, for bindings that pay for every argument (as nm_conv2d_args).  dtype is
 * x_dtype or y_dtype.  norm = 0 is nm_quantize_mx4, which looks at neither residual, gamma, eps nor residual_out.
 * offsets_dev = NULL is nm_linear_mx4, which looks at neither index_dev nor entries; nm_experts_mx4 looks at no residual.
 */
typedef struct nm_rows_mx4_args {
    const void* x_dev;
    const void* residual_dev;
    const float* gamma_dev;
    void* residual_out_dev;
    uint8_t* q_dev;
    uint8_t* scales_dev;
    void* hip_stream;
    int64_t dtype, rows, width, ldx, ldr, ldo, ldq, lds, norm;
    double eps;
} nm_rows_mx4_args_t;
int nm_rows_mx4_args(const nm_rows_mx4_args_t* args);

typedef struct nm_dequantize_mx4_args {
    const uint8_t* q_dev;
    const uint8_t* scales_dev;
    void* y_dev;
    void* hip_stream;
    int64_t dtype, rows, width, ldq, lds, ldy;
} nm_dequantize_mx4_args_t;
int nm_dequantize_mx4_args(const nm_dequantize_mx4_args_t* args);

typedef struct nm_product_mx4_args {
    const uint8_t* q_dev;
    const uint8_t* scales_dev;
    const nm_mx4_t* w;
    const float* bias_dev;
    const void* residual_dev;
    const int32_t* offsets_dev;
    const int32_t* index_dev;
    void* y_dev;
    uint8_t* y_scales_dev;
    void* hip_stream;
    int64_t dtype, rows, width, ldq, lds, ldr, entries, ldy, ldys;
} nm_product_mx4_args_t;
int nm_product_mx4_args(const nm_product_mx4_args_t* args);

#ifdef __cplusplus
}
#endif
#endif /* NM_MX4_H */
