/*
 * fasgd_client.h -- C ABI of libfasgd.so, the client side: the operators with
 * which a client of the parameter server (fasgd.h) turns a fetched theta into
 * the gradient that it pushes.
 *
 * Conventions are those of fasgd.h: the caller owns all device memory, every
 * call is asynchronous on `stream` and never synchronises the host, all
 * arguments are checked on the host before anything is enqueued, and a
 * rejected call enqueues nothing and leaves its reason in
 * fasgd_last_error().  Beyond them:
 *   - Activations and their gradients are row-major matrices of one
 *     client_dtype whose rows may lie apart: element (r, c) is at
 *     x[r ld + c], ld >= cols.  They need the alignment of their type only.
 *   - Parameters and their gradients are fp32 (slices of a client's copy of
 *     theta and of its flat gradient), 4-byte aligned.
 *   - A size of 0 is valid and enqueues nothing, except that sums over no
 *     rows are written as zeros.  The pointers of an empty array may be NULL.
 */
#ifndef FASGD_CLIENT_H
#define FASGD_CLIENT_H

#include "fasgd.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum client_dtype {
    CLIENT_F32 = 0,
    CLIENT_BF16 = 1,
    CLIENT_F16 = 2
} client_dtype;

/*
 * Dropout from a counter-based generator; the mask is never stored.
 *   y = [residual +] (keep ? x * 65536 / (65536 - thr) : 0),
 *   thr = floor(65536 p + 1/2).
 * Element (r, c) has index J = index_base + r cols + c (its place in the
 * matrix, whatever the row strides are) and is kept iff h >= thr, with h the
 * 16-bit half (J mod 2) of word (J mod 8) / 2 of Philox4x32-10 at counter
 * (J/8 low 32 bits, 0x40000000 | site << 16 | J/8 high 16 bits, T, client)
 * with key (seed low, seed high).  The set bit keeps these draws apart from
 * the server's decisions under the same seed; T is the timestamp of the
 * theta the client works on.  So a dropped element costs nothing but its
 * draw, the probability is p to 1/65536, and the same arguments give the
 * same mask in the backward pass (the same call on the gradient, without
 * residual) and when the gradient is computed again.
 * A dropped element gives 0 (or the residual) whatever x holds there, NaN
 * and infinity too.  The arithmetic is fp32, rounded once.
 *   p           in [0, 1]; 1 drops everything
 *   residual    NULL, or the matrix added
 *   y           may be x or residual (with the same stride)
 *   T           0 <= T < 2^32;  client >= 0;  0 <= site < 16384 (the place
 *               of this dropout in the model)
 *   index_base  index of element (0, 0) in a larger matrix, a multiple of 8;
 *               index_base + rows cols <= 2^51
 */
fasgd_status client_dropout(const void* x, int64_t ldx, const void* residual, int64_t ldr, void* y, int64_t ldy,
                            int64_t rows, int64_t cols, int32_t dtype, double p, uint64_t seed, int64_t T,
                            int32_t client, int32_t site, int64_t index_base, hipStream_t stream);

/*
 * The residual norm: what lies between two blocks of a residual model, in one
 * pass each way.
 *   z = N_post(branch),  u = drop(act(gate) z),
 *   sum = residual_scale residual + u,  normed = N_pre(sum),
 * N(x) = x / sqrt(mean(x^2) + eps) w (rms), or
 * N(x) = (x - mean(x)) / sqrt(mean((x - mean(x))^2) + eps) w [+ b] (layer),
 * over the columns of each row.  N_pre is taken of the sum as it is stored
 * (rounded to dtype), so the backward pass, which reads the stored sum, is
 * the gradient of what the forward pass computed.  All arithmetic is fp32.
 */
typedef enum client_norm_kind {
    CLIENT_NORM_RMS = 0,
    CLIENT_NORM_LAYER = 1
} client_norm_kind;

typedef enum client_gate_form {
    CLIENT_GATE_NONE = 0,
    CLIENT_GATE_CHANNEL = 1,    /* fp32 [cols], a parameter */
    CLIENT_GATE_ROW = 2,        /* fp32 [rows], one per row */
    CLIENT_GATE_FULL = 3        /* a matrix of dtype */
} client_gate_form;

typedef enum client_gate_act {
    CLIENT_GATE_IDENTITY = 0,
    CLIENT_GATE_SIGMOID = 1,
    CLIENT_GATE_TANH = 2
} client_gate_act;

/*
 * What both passes share.  w_post NULL: no norm after the block (z = branch);
 * w_pre NULL: none before the next (no normed output).  A bias needs its
 * norm's weights.  p, seed, T, client, site, index_base as in client_dropout
 * (p = 0: no dropout).  1 <= cols <= 2^30, eps > 0, residual_scale finite.
 */
typedef struct client_residual_norm {
    int64_t rows, cols;
    int32_t dtype;              /* client_dtype of the matrices */
    int32_t kind;               /* client_norm_kind */
    const float* w_post;        /* fp32 [cols], or NULL */
    const float* b_post;
    const float* w_pre;
    const float* b_pre;
    const void* gate;           /* as gate_form says */
    int64_t ld_gate;            /* row stride of a full gate */
    int32_t gate_form;
    int32_t gate_act;
    float residual_scale;
    float eps;
    double p;
    uint64_t seed;
    int64_t T;
    int32_t client;
    int32_t site;
    int64_t index_base;
} client_residual_norm;

/*
 * Forward.  residual may be NULL (sum = u).  stats, fp32 [rows][4], receives
 * the mean and 1/sqrt of each norm (0 and 1 where there is none) for the
 * backward pass.  sum may be residual and normed may be branch (with the
 * same stride), where the caller has no further use for them.
 */
fasgd_status client_residual_norm_forward(const client_residual_norm* op, const void* branch, int64_t ld_branch,
                                          const void* residual, int64_t ld_residual, void* sum, int64_t ld_sum,
                                          void* normed, int64_t ld_normed, float* stats, hipStream_t stream);

/*
 * Backward, from the gradients of sum (dsum, NULL: zero) and of normed
 * (dnormed, required with w_pre, else NULL).  dbranch is written, dresidual
 * (the gradient of residual; NULL: not wanted) may be dsum.  dw_post,
 * db_post, dw_pre, db_pre (fp32 [cols], each NULL: not wanted) and dgate (of
 * the gate's form and type; NULL: not wanted for a channel gate, required
 * for the others) are written, not added to.  The sums over rows are taken
 * in a fixed order, so the result is the same run to run.
 * workspace: client_residual_norm_workspace_bytes(rows, cols) bytes of device
 * scratch, 16-byte aligned, contents irrelevant.
 */
size_t client_residual_norm_workspace_bytes(int64_t rows, int64_t cols);
fasgd_status client_residual_norm_backward(const client_residual_norm* op, const void* branch, int64_t ld_branch,
                                           const void* sum, int64_t ld_sum, const float* stats, const void* dsum,
                                           int64_t ld_dsum, const void* dnormed, int64_t ld_dnormed, void* dbranch,
                                           int64_t ld_dbranch, void* dresidual, int64_t ld_dresidual, float* dw_post,
                                           float* db_post, void* dgate, int64_t ld_dgate, float* dw_pre,
                                           float* db_pre, void* workspace, size_t workspace_bytes,
                                           hipStream_t stream);

/*
 * Matrix products in 8-bit floating point with a scale for each block of 128.
 *
 * An operand is a matrix [rows][k] held for products over k.  Each row's k
 * values lie in blocks of 128, and block kb of row r is held as
 *   value = q 2^(scales[kb lds + r] - 127),
 * q an 8-bit float (OCP e4m3, largest 448; or e5m2, largest 57344) at
 * data[r ld + k].  Scales are powers of two: multiplying by one is exact, so
 * an operand is rounded once, and the matrix instruction applies them.
 * A product needs data to be 16-byte aligned, ld a multiple of 128 and at
 * least k rounded up to one (the values past k must be 0), scales 4-byte
 * aligned and lds a multiple of 4 of at least rows.  k and ld are at most
 * 2^23, rows 2^27.
 */
typedef enum client_fp8_format {
    CLIENT_FP8_E4M3 = 0,
    CLIENT_FP8_E5M2 = 1
} client_fp8_format;

/* added to the output's type: a choice of client_fp8_matmul and client_fp8_linear */
enum { CLIENT_FP8_SHORT_SUMS = 0x100 };

typedef struct client_fp8_operand {
    uint8_t* data;              /* [rows][ld] */
    uint8_t* scales;            /* [ceil(k / 128)][lds], an exponent + 127 each */
    int64_t rows, k, ld, lds;
    int32_t format;             /* client_fp8_format */
} client_fp8_operand;

/*
 * Quantizes x ([rows][cols] of dtype) into by_rows (rows x cols, blocks of
 * 128 along each row of x) and / or by_cols (the transpose, cols x rows,
 * blocks of 128 along each column), from one read of x.  Either may be NULL;
 * both have one format.  block_rows = 1: a scale for each row of an operand
 * and block of 128 (activations and their gradients).  block_rows = 128: one
 * for each 128 x 128 block of x (weights), written for each row all the same,
 * so that both operands hold the same values.
 * The scale of a block with largest finite magnitude amax is 2^e with e the
 * smallest integer that has amax <= 448 2^e (57344 2^e) and e >= -126; e = 0
 * for a block of zeros.  q = x 2^-e rounded to nearest even; what is not
 * finite becomes NaN.  The values past k in an operand's last block are
 * written as zeros.
 */
fasgd_status client_fp8_quantize(const void* x, int64_t ldx, int64_t rows, int64_t cols, int32_t dtype,
                                 int32_t block_rows, const client_fp8_operand* by_rows,
                                 const client_fp8_operand* by_cols, hipStream_t stream);

/*
 * c[m][n] = sum over k of a[m][k] b[n][k] (with accumulate != 0: added to
 * what c holds), [a->rows][b->rows] of c_dtype, for two operands of one k.
 * A linear layer y = x W^T is the product of x and W; its input gradient
 * that of dy and W transposed, its weight gradient that of dy transposed and
 * x transposed.  Sums are fp32 and rounded once (values below 2^-126 are held
 * to 2^-133).
 * c_dtype CLIENT_BF16 or CLIENT_F16 with CLIENT_FP8_SHORT_SUMS added to it
 * takes the matrix instruction of 8-bit values, at twice the rate: each 8
 * consecutive products of a sum, from a multiple of 8 on, are then cut off
 * below 2^-13 of the largest of them before they go into the fp32 sum, an
 * error of up to 7 x 2^-13 of that product for each 8, whatever the sum of
 * them is.
 * Where few outputs leave most of the chip idle, the contraction is split and
 * its parts joined in order through the workspace, so the result is the same
 * run to run.
 * workspace: client_fp8_workspace_bytes(a->rows, b->rows, k) bytes of device
 * scratch, 16-byte aligned, contents irrelevant (the same size serves
 * client_fp8_linear, which also holds its quantized x there).
 */
size_t client_fp8_workspace_bytes(int64_t m, int64_t n, int64_t k);
fasgd_status client_fp8_matmul(const client_fp8_operand* a, const client_fp8_operand* b, void* c, int64_t ldc,
                               int32_t c_dtype, int32_t accumulate, void* workspace, size_t workspace_bytes,
                               hipStream_t stream);

/*
 * y = x W^T for activations x ([m][w->k] of dtype, not quantized before) and
 * weights held as an operand, as serving and evaluation need it: x is
 * quantized in e4m3 as client_fp8_quantize does with block_rows = 1, then
 * multiplied, with the same sums (short ones by the same flag in dtype).  y
 * is [m][w->rows] of dtype, m at most 2^27 as an operand's rows are.
 * workspace: client_fp8_workspace_bytes(m, w->rows, w->k) bytes, as above.
 */
fasgd_status client_fp8_linear(const void* x, int64_t ldx, int64_t m, const client_fp8_operand* w, void* y,
                               int64_t ldy, int32_t dtype, void* workspace, size_t workspace_bytes,
                               hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* FASGD_CLIENT_H */
