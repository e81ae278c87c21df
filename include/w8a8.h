/*
 * libw8a8 -- C ABI of the MI355X (gfx950) W8A8 linear layer: int8 weights with a scale for each output channel, activations
 * quantised to int8 with a scale for each token (paper section 2.2, "W8A8"), for any number of tokens: plain decoding, a draft's
 * verification and whole prompts.  A library of its own beside libw4a16, whose conventions, return codes (include/w4a16.h) and workspaces
 * it shares; it exports w4a16_workspace_init and w4a16_strerror too, so that a program of W8A8 linears needs no other.
 *
 * Layout of codes, weights and activations alike: tiles of 16 rows (channels or tokens) by 64 values of k, 1 KB each, in the order in
 * which the 16x16x64 matrix instruction takes its operands; rows are padded to a multiple of 16, k to a multiple of 128:
 *   code (r, k) at byte ((r / 16) * ceil(K / 128) * 2 + k / 64) * 1024 + (k % 64) / 16 * 256 + (r % 16) * 16 + k % 16
 * Codes of k >= K are zero; what lies in rows beyond the last never reaches a result.
 */
#ifndef W8A8_H
#define W8A8_H

#include "w4a16.h"

#ifdef __cplusplus
extern "C" {
#endif

/* What becomes of the fp16 input before it is quantised. */
#define W8A8_PLAIN 0      /* x [M, K] as it is */
#define W8A8_RMS_NORM 1   /* x [M, K] -> x * gamma / sqrt(mean(x^2) + eps), as rms_norm: fp32, rounded to fp16 */
#define W8A8_SILU_MUL 2   /* x [M, 2 K], gate then up -> silu(gate) * up, silu(t) = t / (1 + exp(-t)): fp32, rounded to fp16 */

/* Bytes of the codes of a [rows, K] matrix in the layout above.  0 if the shape is not supported: K a multiple of 16 up to 65536. */
size_t w8a8_packed_bytes(int rows, int K);

/* int8 [rows, K] row-major -> the layout above, and back.  Exact.  `packed` holds w8a8_packed_bytes(rows, K); padding is zeroed. */
int w8a8_pack(const int8_t *w, void *packed, int rows, int K, void *stream);
int w8a8_unpack(const void *packed, int8_t *w, int rows, int K, void *stream);

/* Codes and scales of M tokens, each on its own: with x' what `pre` makes of the fp16 input,
 *   scale[m] = max_k |x'[m, k]| / 127 (fp32),   code = x' / scale rounded to the nearest whole number, ties to even
 * A row of zeros gets scale 0 and codes 0, a row with an infinity or a NaN in x' scale NaN and codes 0 (its outputs are NaN).
 * codes: w8a8_packed_bytes(M, K) bytes in the layout above (rows >= M are not written); scale fp32 [M].  gamma fp16 [K], given with
 * W8A8_RMS_NORM and with nothing else; eps >= 0. */
int w8a8_quantize(const void *x, int pre, const void *gamma, float eps, void *codes, float *scale, int M, int K, void *stream);

/* Scratch of w8a8_gemm and w8a8_linear for these sizes; the size for the largest M serves every smaller one. */
size_t w8a8_workspace_bytes(int M, int N, int K);

/* y[m, n] = (sum_k codes[m, k] * w[n, k]) * scale[m] * w_scale[n] (+ residual[m, n]): the sum in 32-bit integers, exact; the rest in fp32,
 * rounded to fp16 once.  codes, scale: w8a8_quantize's; packed: w8a8_pack's of the weight [N, K]; w_scale fp32 [N]; residual fp16 [M, N]
 * or NULL, y fp16 [M, N]; residual may be y.  N a multiple of 8, K of 16, K <= 65536, M <= 2^20.  `workspace` holds
 * w8a8_workspace_bytes(M, N, K) and has been initialised with w4a16_workspace_init. */
int w8a8_gemm(const void *codes, const float *scale, const void *packed, const float *w_scale, const void *residual, void *y, int M, int N, int K,
              void *workspace, size_t workspace_bytes, void *stream);

/* w8a8_quantize into the workspace, then w8a8_gemm: the same results bit for bit.  x, too, may be y. */
int w8a8_linear(const void *x, int pre, const void *gamma, float eps, const void *packed, const float *w_scale, const void *residual, void *y, int M,
                int N, int K, void *workspace, size_t workspace_bytes, void *stream);

/* How w8a8_gemm, and w8a8_linear behind its quantisation, would run a product, so that a test can show which kernels it has compared with the
 * oracle.  out receives 4 ints: [0] 0 = weights streamed for few tokens, 1 = tiles, [1] tokens and [2] channels of a workgroup's tile, [3] workgroups
 * that share a tile's walk along k.  (w8a8_linear has a kernel of its own for one token of K up to 4096.)  Host only: touches no GPU.  Errors as
 * w8a8_gemm's size checks. */
int w8a8_gemm_plan_describe(int M, int N, int K, int *out);

#ifdef __cplusplus
}
#endif
#endif /* W8A8_H */
