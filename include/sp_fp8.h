/*
 * sp_fp8.h -- linear layers that pruning leaves dense, in 8-bit floating point (libsp, GB300 / sm_103a): the
 * vocabulary's, and those of a small model that drafts tokens.
 *
 * Numbers are e4m3 codes (four bits of exponent, three of mantissa, largest 448) with one fp32 scale for each
 * block of 128: of a weight W [N][K] one per 128 x 128 block, scale[ceil(N/128)][ceil(K/128)]; of a row of
 * activations one per 128 columns.  With a the largest magnitude of a block, in fp32 with each operation rounded on its own:
 *     s = max(a * (1/448), 2^-100)     code = e4m3(x * (1 / s)), to nearest even, limited to +-448
 * A block with a NaN or an infinity has a scale of NaN or infinity, and makes every result that it has a part in NaN.
 *     y[m][n] = bf16( sum over blocks b of sx[m][b] * sw[n/128][b] * sum over k in b of qx[m][k] * qw[n][k] )
 * The inner sums are the tensor cores' (fp32); the outer ones are fp32.
 *
 * The paper (arXiv 2405.03594) quantises to INT8 and leaves the layers that it does not prune alone; it defines none of
 * these operators, so their definitions stand here.  The conventions of sp.h hold: device pointers of the current device,
 * `stream` a cudaStream_t as void*, asynchronous, a status from every call, nothing allocated and no host
 * synchronisation, so every call can be captured in a CUDA graph.
 */
#ifndef SP_FP8_H
#define SP_FP8_H

#include <stddef.h>
#include <stdint.h>

#include "sp.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Quantise activations x (bf16 [m][k], x_stride elements from row to row) by rows:
 *   codes  [m][k] bytes, `stride` from row to row, a multiple of 16 and at least k; bytes behind k are written as 0
 *          as far as the last block of 128 reaches
 *   scale  [ceil(k/128)][scale_stride] fp32: the scale of row r and block b at scale[b * scale_stride + r];
 *          scale_stride a multiple of 4 and at least m
 * codes and scale 16-byte aligned (SP_ERR_ALIGNMENT), k >= 1.  One launch.  m == 0 returns SP_OK. */
sp_status sp_fp8_quantize_rows(const void* x, int64_t x_stride, int64_t m, int64_t k, void* codes, int64_t stride,
                               float* scale, int64_t scale_stride, void* stream);

/* Quantise a weight w (bf16 [n][k], w_stride elements from row to row) by 128 x 128 blocks: codes as above,
 * scale [ceil(n/128)][ceil(k/128)] fp32.  One launch. */
sp_status sp_fp8_quantize_blocks(const void* w, int64_t w_stride, int64_t n, int64_t k, void* codes, int64_t stride,
                                 float* scale, void* stream);

typedef struct sp_fp8_linear_args {
  const void* w;         /* codes [n][k], w_stride bytes from row to row (a multiple of 16)          */
  const float* w_scale;  /* [ceil(n/128)][ceil(k/128)]                                               */
  const void* x;         /* bf16 [m][k], x_stride elements from row to row; NULL: xq holds the rows  */
  const void* xq;        /* codes as sp_fp8_quantize_rows writes them, or NULL where x is given      */
  const float* x_scale;  /* their scales                                                             */
  void* y;               /* bf16 [m][n], y_stride elements from row to row                           */
  int64_t w_stride, x_stride, xq_stride, x_scale_stride, y_stride;
  int64_t m, n, k;
} sp_fp8_linear_args;

/* y = x . W^T.  x is quantised on the way (into the workspace, or on chip where there are few rows).  `workspace` as for
 * sp_linear: sp_fp8_workspace_size bytes, its first SP_WORKSPACE_ZERO_BYTES zero before its first use, calls that share it
 * ordered on one stream; one buffer can serve every call of the library that takes one.  Results are bitwise
 * repeatable for given sizes and device, and the same whether x or xq is given.  y must not overlap x, xq or their scales; what lies
 * beside its rows is left as it is.  SP_ERR_INVALID_ARG for a null pointer, a
 * negative size, n or k of 0, a stride that is too small, both or neither of x and xq; SP_ERR_UNSUPPORTED for sizes above
 * 2^30, strides of codes that are no multiple of 16, or more than 64 rows on a device that holds no pair of CTAs; SP_ERR_ALIGNMENT for codes, x_scale or the workspace off a
 * 16-byte boundary, or bf16 off its own size.  m == 0 returns SP_OK.  One launch, or two.  Of a launch that sp_check reports as
 * SP_ERR_TIMEOUT no result is to be used; the workspace is ready for the next call. */
sp_status sp_fp8_linear(const sp_fp8_linear_args* args, void* workspace_dev, size_t workspace_bytes, void* stream);

/* Failure-path test (nothing calls it in normal use).  sp_fp8_linear, with warp `warp` of CTA `cta` of the product's kernel waiting,
 * before the one that it counts as `block` of its blocks of 128 columns, on a shared-memory barrier that nothing completes, and every
 * wait bounded by wait_ms milliseconds.  The warp gives up and records SP_ERR_TIMEOUT, as any whose wait expires, with the copies
 * and products before that block on their way; y is written within its bounds, with numbers that are worth nothing.
 * The launch ends by itself, and the workspace is ready for the next call.  A cta, warp or block that the kernel does not have
 * gives up nothing.  wait_ms in 1..10000, the others not negative (SP_ERR_INVALID_ARG otherwise); compiled for up to 16 rows, and for
 * more than 64 where a tile has 128 rows of W (SP_ERR_UNSUPPORTED otherwise, with nothing launched), as variants of the kernels of their own. */
sp_status sp_test_expired_fp8(const sp_fp8_linear_args* args, void* workspace_dev, size_t workspace_bytes, int32_t cta,
                              int32_t warp, int32_t block, uint32_t wait_ms, void* stream);

/* Workspace bytes of sp_fp8_linear on the current device for m rows.  Host only. */
sp_status sp_fp8_workspace_size(int64_t m, int64_t n, int64_t k, size_t* bytes);

#ifdef __cplusplus
}
#endif

#endif /* SP_FP8_H */
