/*
 * lora_mx.h -- the multi-LoRA batched linear layer on a backbone held in 4 bits, and the two operators around it: the
 * root-mean-square norm in front of the projections, whose output comes in 8 bits with scales as well, and the conversions
 * in and out of both formats.
 *
 *     Y[t,n] = sum_k Xb[t,k] W[n,k]  +  s_a sum_j (sum_k X[t,k] A_a[j,k]) B_a[n,j] ,   a = adapter of row t's request
 *
 * W is the backbone in 4 bits, Xb the activations: X itself (bf16), or a copy of them in 8 bits.  The adapter term is
 * that of lora_linear(): from X in bf16, on the same plan and the same adapter tables.  Contexts, streams, plans,
 * status codes and the ownership of memory are those of lora_mi355x.h.
 *
 * Operands overlap where they have a byte of their rows in common: rows of one stride may lie side by side in a buffer (packed
 * projections, H and Y as halves, codes with their scales behind them).  Of different strides the extents, first byte to last, decide.
 *
 * Formats (the layout of the OCP microscaling formats): every 32 consecutive values of a row are a block with one scale.
 *     value = element * 2^(scale - 127)          scale: one byte; 255 makes the whole block NaN
 *     LORA_MX_E2M1   elements of 4 bits, two a byte, the even one in the low half: 0 0.5 1 1.5 2 3 4 6 and their negatives
 *     LORA_MX_E4M3   elements of 8 bits: sign, 4 exponent bits (bias 7), 3 mantissa bits; +-448 at most, no infinity, 0x7f NaN
 * Values are meant to be within bf16's normal range: 2^-126 <= |value| < 2^127 where it is not zero.
 */
#ifndef LORA_MX_H
#define LORA_MX_H

#include "lora_mi355x.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum lora_mx_format { LORA_MX_E2M1 = 0, LORA_MX_E4M3 = 1 } lora_mx_format;

#define LORA_MX_BLOCK 32           /* values that share a scale                       */
#define LORA_RMS_NORM_MAX_K 65536  /* longest row of lora_rms_norm()                  */

/* Rows of K values in one of the formats.  Device pointers; codes == NULL: none.  A row of scales takes ld_scales bytes
 * whatever K is (the bytes behind its K / 32 scales may be read and are not used). */
typedef struct lora_mx_rows_t {
    void *codes;        /* [rows, ld_codes] bytes, 16-byte aligned                                          */
    int64_t ld_codes;   /* bytes from row to row: >= K / 2 (E2M1) or K (E4M3), a multiple of 16              */
    void *scales;       /* [rows, ld_scales] bytes, 4-byte aligned                                           */
    int64_t ld_scales;  /* >= K / 32, a multiple of 4                                                       */
    int32_t format;     /* lora_mx_format                                                                   */
    int32_t reserved;   /* must be 0                                                                        */
} lora_mx_rows_t;

/* ---- conversions ----------------------------------------------------------------------------------------- */

typedef struct lora_mx_convert_desc {
    int32_t dtype;      /* lora_dtype of X                                                                  */
    int32_t K;          /* a multiple of 32, > 0                                                            */
    int64_t rows;       /* >= 0                                                                             */
    void *X;            /* device [rows, ldx], 16-byte aligned; lora_mx_quantize() only reads it            */
    int64_t ldx;        /* >= K, a multiple of 8 (bf16) or 4 (fp32)                                         */
    lora_mx_rows_t q;
} lora_mx_convert_desc;

/* q = X: the scale of a block is the smallest power of two (2^-127 to 2^127) with which its largest magnitude is at most
 * 6 (E2M1) or 448 (E4M3), the values divided by it are rounded to nearest, ties to even.  A block of zeros gets the scale
 * 2^-127; one that holds an infinity or a NaN gets 255.  Asynchronous on `stream`; no-op for 0 rows.
 * Errors: INVALID_ARG (null pointers, dtype, format, overlap of X and q), SHAPE, ALIGNMENT; HIP if the launch fails. */
int lora_mx_quantize(lora_ctx *ctx, const lora_mx_convert_desc *desc, lora_stream_t stream);

/* X = q, rounded to nearest where dtype cannot hold a value (it can within the range above).  Errors as above. */
int lora_mx_dequantize(lora_ctx *ctx, const lora_mx_convert_desc *desc, lora_stream_t stream);

/* ---- root-mean-square norm ---------------------------------------------------------------------------------- */

typedef struct lora_rms_norm_desc {
    int32_t dtype;      /* lora_dtype of X, R, H, Y and gamma                                               */
    int32_t K;          /* row length: a multiple of 8 (32 with q), 0 < K <= LORA_RMS_NORM_MAX_K            */
    int64_t rows;       /* >= 0                                                                             */
    float eps;          /* >= 0, finite                                                                     */
    int32_t flags;      /* must be 0                                                                        */
    const void *X;      /* device [rows, ldx]                                                               */
    int64_t ldx;        /* (every ld: >= K, a multiple of 8 (bf16) or 4 (fp32); every pointer 16-byte aligned) */
    const void *R;      /* device [rows, ldr] residual, or NULL                                             */
    int64_t ldr;
    const void *gamma;  /* device [K]                                                                       */
    void *H;            /* device [rows, ldh]: X + R, or NULL.  May be X or R itself (same ld)               */
    int64_t ldh;
    void *Y;            /* device [rows, ldy]: the normed rows, or NULL.  May be X or R itself (same ld)     */
    int64_t ldy;
    lora_mx_rows_t q;   /* the normed rows in E4M3, or codes == NULL                                        */
} lora_rms_norm_desc;

/* h = X + R (X alone without R), in fp32;  y = h / sqrt(mean(h^2) + eps) * gamma, the mean in 64 bits; H and Y are h and y rounded
 * once, q is what lora_mx_quantize() would make of y before any rounding.  At least one of H, Y and q; outputs may not
 * overlap each other, gamma, or -- but for the two cases above -- the inputs.  Rows are independent, and a row's result does not depend on the others.
 * Asynchronous on `stream`; no-op for 0 rows.  Errors: INVALID_ARG, SHAPE, ALIGNMENT; HIP if the launch fails. */
int lora_rms_norm(lora_ctx *ctx, const lora_rms_norm_desc *desc, lora_stream_t stream);

/* ---- the layer ------------------------------------------------------------------------------------------------ */

typedef struct lora_mx_linear_desc {
    int32_t K;          /* d_in:  a multiple of 32, > 0                                                     */
    int32_t N;          /* d_out: > 0                                                                       */
    int32_t flags;      /* must be 0                                                                        */
    int32_t reserved;   /* must be 0                                                                        */
    const void *X;      /* device [T, ldx] bf16.  NULL only with Xq and without adapters (tbl NULL)         */
    int64_t ldx;        /* >= K, a multiple of 8; X smaller than 4 GiB, and above 128 rows without Xq so is 2 T times K
                           rounded up to whole 512                                                          */
    lora_mx_rows_t Xq;  /* [T] rows, E4M3: the base product's activations; codes == NULL: X in bf16. < 4 GiB */
    lora_mx_rows_t W;   /* [N] rows, E2M1; const, externally owned; ld_codes < 16 MiB                       */
    void *Y;            /* device [T, ldy] bf16; must not overlap any input or the workspace                */
    int64_t ldy;        /* >= N, a multiple of 8                                                            */
    const lora_adapter_table_t *tbl; /* host pointer; NULL = backbone product only                        */
    void *workspace;    /* device, 256-byte aligned, lora_mx_linear_workspace_bytes() big                   */
    size_t workspace_bytes;
} lora_mx_linear_desc;

/* A size of desc->workspace in device bytes that serves every lora_mx_linear() of this K and N on up to T rows and ranks up to r_max (with_xq: whether
 * Xq is given; the size without it serves calls with it too).  It holds what lora_linear()'s does (V, the decode path's partial sums of up
 * to 128 rows, the adapter term in fp32); above 128 rows also the activations in two parts of 8 bits (bf16 ones: 2 T bytes for every K, rounded
 * up to whole 512, and 1/32 of that), and partial sums in fp32 where the tiles of T rows alone would leave much of the chip idle.  (A
 * batch that would want more room for those than is left is cut into fewer stretches of K, or none.)  One workspace may serve calls of
 * different shapes as long as it is big enough for each and they do not overlap in time.  0 for invalid arguments. */
size_t lora_mx_linear_workspace_bytes(int64_t T, int32_t K, int32_t N, int32_t r_max, int32_t with_xq);

/* The layer.  Products of the held values are exact and summed in fp32; the adapter term's intermediate is rounded as
 * lora_linear() says; Y is rounded once.  (Activations in bf16 of more than 128 rows are taken apart into two parts of 8 bits:
 * exactly down to 2^-13 of the largest value of their block of 32, off by at most 2^-21 of it below.)  An infinity or a NaN among a
 * row's activations makes that row of Y infinite or NaN, one in a block of W its column, one in an adapter the rows that use it; above 128 rows
 * one in B_a may reach the rows that share a block of 16 with those in the plan's order, and no others.  Returns after enqueueing launches
 * only (it may be captured into a graph as lora_linear() may).  Bitwise reproducible run to run.  Errors, all found before the first launch: INVALID_ARG, PLAN,
 * SHAPE, ALIGNMENT, WORKSPACE_TOO_SMALL; HIP if a launch fails. */
int lora_mx_linear(lora_ctx *ctx, const lora_plan_t *plan, const lora_mx_linear_desc *desc, lora_stream_t stream);

/* Several projections of the same activations in one call (1 <= n <= LORA_MAX_MULTI): descs share X, ldx, Xq and K; each has
 * its own W, N, Y, table and workspace.  Computes what n calls of lora_mx_linear() compute.  Errors as there; INVALID_ARG also
 * for n out of range, descs that differ in the activations or K, or two of which one's Y or workspace overlaps the other's Y,
 * workspace or W. */
int lora_mx_linear_multi(lora_ctx *ctx, const lora_plan_t *plan, const lora_mx_linear_desc *const *descs, int32_t n,
                         lora_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* LORA_MX_H */
