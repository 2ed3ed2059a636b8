/*
 * rotq - online Hadamard rotate-and-quantize for MI355X (gfx950).
 *
 * C ABI of the inference-time hot path of rotation-based W/A/KV quantization
 * (arXiv 2504.13989): every token row is multiplied by a normalised Hadamard
 * matrix (section 2.3.2 Eq. 1 for orders 2^k; section 2.3.3 / Appendix B
 * Algorithm 2 for Paley orders; zero-padding of section 4.2 Eq. 2 when the row is
 * narrower than the order) and then quantized per token with the symmetric uniform
 * quantizer of section 2.1 under a clip ratio (section 3.1).
 *
 * Conventions
 *   - Order n = p * 2^k, where 2^k is the largest power of two for which p is 1 or a
 *     Paley order <= 256: p = q+1 with q prime, q = 3 (mod 4) (Algorithm 2), or
 *     p = 2(q+1) with q prime, q = 1 (mod 4) (Paley II; not in the paper, standard
 *     construction H = C (x) [[1,1],[1,-1]] + I (x) [[1,-1],[-1,-1]]).  Where both
 *     exist for one p the first is used.  n must be a multiple of 8 and at least 32 (packed rows are
 *     whole bytes); where no block of at most 256 exists a Paley block of up to 4096 is taken.  The
 *     fast kernels serve 16-bit rows of the orders rq_next_order returns (2^k >= 32, block <= 256);
 *     fp32 rows to be quantized per token on orders with 2^k <= 512 (Sylvester: up to 2^14) have an fp64
 *     kernel of their own; every other case (other calls on fp32 rows, unaligned rows, other orders) runs
 *     on a general kernel that keeps the row in the 160 KB of LDS, which bounds n: 2^15 for Sylvester
 *     orders and 20448 for block orders; fp32 rows are quantized from an fp64 copy of the row and stop at
 *     n = 2^14 (Sylvester) and 9728 (block orders).  A row call on an order beyond what its kernels can
 *     hold returns RQ_ERR_NO_ORDER.
 *   - H_n = H_p (x) H_{2^k}: flat index j = a * 2^k + c (a < p, c < 2^k),
 *     H_n[i, j] = H_p[i / 2^k, j / 2^k] * (-1)^popcount((i % 2^k) & (j % 2^k)).
 *   - Rotated row: y = H_n pad(x) / sqrt(n), pad() appends n - d zeros.
 *   - Quantizer: amax = max_j |y_j|; Delta = clip * amax / (2^b - 1);
 *     code_j = clamp(round_half_even(y_j / Delta), -2^(b-1), 2^(b-1) - 1);
 *     amax == 0 gives Delta = 0 and all-zero codes.  Arithmetic is fp32.
 *   - Packed codes: row r starts at byte r * n * b / 8; element j of the rotated row is
 *     the b-bit field at bits [j*b, (j+1)*b) of the row's little-endian bit stream (stream
 *     bit i = bit i % 8 of byte i / 8), holding the code's low b bits (two's complement).
 *   - scales[r] = Delta of row r, so that y^_j = code_j * scales[r].
 *
 * All functions return RQ_OK (0) or a negative error code; none throws or aborts.
 * Argument errors are detected on the host before any HIP call.  Data values are not
 * validated (NaN / Inf propagate: such a row has no useful codes and a scale that is
 * infinite, NaN or 0; other rows are not affected).  The hot-path calls enqueue work on the
 * caller's stream and return without synchronising and without allocating.
 *
 * The kernel is chosen by order, type and number of rows, and different kernels add in
 * different orders.  The same row can therefore have other last bits in a call with another
 * number of rows: scales a few parts in 10^7 apart, and another code where a value lies that
 * close to a rounding boundary (about one code byte in 10^7).  In rq_rotate_quantize this
 * concerns 16-bit rows of the powers of two from 2048 to 8192, and of orders 128 pb with
 * 97 <= pb <= 256 whose block is made of pairs of rows (14336, 18944 and 28672 among them): there the
 * border is at two rows for each compute unit, from pb = 161 on at one.  Calls with
 * the same number of rows give the same bits.
 */
#ifndef ROTQ_H
#define ROTQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define RQ_OK             0
#define RQ_ERR_ARG       -1   /* bad pointer, size, stride, bit-width, clip, alignment, workspace */
#define RQ_ERR_NO_ORDER  -2   /* n has no supported factorisation p * 2^k, n % 8 != 0, or no kernel can hold a row of n */
#define RQ_ERR_HIP       -3   /* HIP allocation / launch failure, or the handle has no device table */
#define RQ_ERR_NOMEM     -4   /* host allocation failure */
#define RQ_ERR_TOO_LARGE -5   /* rq_quant_error_noalloc: rows * n_clips exceeds the static scratch buffer */

#define RQ_BF16 0             /* X elements are bfloat16 (2 bytes) */
#define RQ_F32  1             /* X elements are float (4 bytes) */
#define RQ_F16  2             /* IEEE half precision (2 bytes): rows of X, and results of rq_rotate / rq_dequantize_rotate */

#define RQ_KIND_SYLVESTER 0
#define RQ_KIND_PALEY1    1
#define RQ_KIND_PALEY2    2

#define RQ_MAX_CLIPS 64
#define RQ_GROUP 128

/* Opaque.  The factorisation and the device tables do not change after rq_hadamard_build, and the
 * row calls take the handle as const: one handle may serve any number of host threads and streams at
 * once.  Two fields are written later, both atomically: the kernel selector of
 * rq_hadamard_set_variant (a test hook; calls already running keep the kernel they chose) and the
 * diagnostic name read by rq_hadamard_last_kernel (the most recent call on any thread). */
typedef struct rq_hadamard rq_hadamard_t;

/*
 * Build the rotation of order n (sections 2.3.2, 2.3.3, Appendix B Algorithm 2): factor
 * n = p * 2^k, build the +-1 block H_p from Legendre symbols in integer arithmetic on the
 * host, and, when a GPU is present, upload the block tables to the current device.
 * Without a GPU the handle is host-only: the info/dense calls work, the hot-path calls
 * return RQ_ERR_HIP.
 * The largest 2^k is taken for which p is 1 or a Paley order of at most 256; where there is none, a
 * large Paley block of at most 4096 is used, up to the whole dimension (section 5.2.2:
 * 1544 = 1543 + 1).
 *   n    [in]  rotation order, multiple of 8 (packed rows are whole bytes)
 *   out  [out] host pointer receiving the handle; owned by the caller, released with
 *              rq_hadamard_free.  Untouched on error.
 * Errors: RQ_ERR_ARG (out NULL, n < 32), RQ_ERR_NO_ORDER (n not a multiple of 8, or no
 * factorisation), RQ_ERR_NOMEM, RQ_ERR_HIP.
 */
int rq_hadamard_build(int n, rq_hadamard_t** out);

/* Release a handle and its device tables (NULL is a no-op).  Work already enqueued that
 * uses the handle must have completed. */
void rq_hadamard_free(rq_hadamard_t* h);

/*
 * Factorisation held by a handle.  Any output pointer may be NULL.
 *   n      order;  p  block order (1 = pure Sylvester);  kind  RQ_KIND_*;
 *   q      the prime of the Paley construction (0 for Sylvester);  log2m  k.
 * Errors: RQ_ERR_ARG (h NULL).
 */
int rq_hadamard_info(const rq_hadamard_t* h, int* n, int* p, int* kind, int* q, int* log2m);

/*
 * Test hook: the dense un-normalised matrix H_n, n*n entries of +-1, row-major, written
 * to HOST memory host_out (caller-owned, n*n bytes).  Refused for n > 8192.
 * Errors: RQ_ERR_ARG.
 */
int rq_hadamard_dense(const rq_hadamard_t* h, int8_t* host_out);

/*
 * Dimension expansion helper (section 4.2): the smallest order n >= d that
 * rq_hadamard_build accepts with 2^k >= 32 and a block of at most 256 (the orders the fast
 * kernels serve).  n_out is a host pointer.
 * Errors: RQ_ERR_ARG (d < 1, n_out NULL), RQ_ERR_NO_ORDER (none below 2^30).
 */
int rq_next_order(int d, int* n_out);

/*
 * Rotate and quantize `rows` token rows (sections 2.1, 2.3, 3.1, 4.2; see Conventions).
 *   h       [in]  handle of order n >= d, with device tables on the current device
 *   X       [in]  DEVICE pointer, rows x d elements of `dtype`, row-major with leading
 *                 dimension ld >= d (in elements); aligned to the element size.  A row of
 *                 width d < n is treated as zero-padded to n.  Not modified.
 *   bits    [in]  3 or 4
 *   clip    [in]  clip ratio in (0, 1]
 *   codes   [out] DEVICE pointer, rows * n * bits / 8 bytes, 4-byte aligned, caller-owned
 *   scales  [out] DEVICE pointer, rows floats, caller-owned
 *   stream  [in]  hipStream_t (NULL = the null stream)
 * rows == 0 is a successful no-op (X, codes and scales may then be NULL).
 * Errors: RQ_ERR_ARG (NULL pointer, rows < 0, d < 1, d > n, ld < d, bits not 3/4, clip not in
 * (0,1] or NaN, misaligned pointer, unknown dtype), RQ_ERR_NO_ORDER (no kernel can hold a row of
 * this order and type, see Conventions), RQ_ERR_HIP.
 */
int rq_rotate_quantize(const rq_hadamard_t* h,
                       const void* X, int dtype, int64_t rows, int d, int64_t ld,
                       int bits, float clip,
                       void* codes, float* scales, void* stream);

/*
 * Rotate, then quantize asymmetrically in groups of RQ_GROUP consecutive rotated values (the
 * KV-cache setting of section 5.1: 3-bit asymmetric quantization with a group size of 128;
 * rotation as in sections 2.3, 4.2).  The paper names the scheme without a formula; per group g
 * of the rotated row y:
 *   lo = clip * min(y_g), hi = clip * max(y_g), Delta = (hi - lo) / (2^b - 1),
 *   code_j = clamp(round_half_even((y_j - lo) / Delta), 0, 2^b - 1),  y^_j = code_j * Delta + lo.
 * A constant group has Delta = 0 and all-zero codes.
 *   h       [in]  handle whose order n is a multiple of RQ_GROUP
 *   codes   [out] DEVICE, rows * n * bits / 8 bytes: unsigned b-bit fields, bitstream layout as
 *                 in rq_rotate_quantize
 *   scales  [out] DEVICE, rows * (n / RQ_GROUP) floats: Delta, row-major [row][group]
 *   mins    [out] DEVICE, rows * (n / RQ_GROUP) floats: lo
 * Other arguments, ownership and the rows == 0 rule as in rq_rotate_quantize.
 * Errors: RQ_ERR_ARG (as rq_rotate_quantize, or n not a multiple of RQ_GROUP), RQ_ERR_NO_ORDER
 * (no kernel can hold a row of this order), RQ_ERR_HIP.
 */
int rq_rotate_quantize_asym(const rq_hadamard_t* h,
                            const void* X, int dtype, int64_t rows, int d, int64_t ld,
                            int bits, float clip,
                            void* codes, float* scales, float* mins, void* stream);

/*
 * Measurement aid (no operation of the paper): a kernel with the memory traffic of
 * rq_rotate_quantize on 16-bit rows of width n and no arithmetic - it reads every row with the same
 * loads and writes n * bits / 8 bytes of codes and one float per row (an xor fold of the input, not
 * a quantization).  Its duration is the practical floor for a rotate_quantize launch of that shape
 * on this chip; bench.py reports it next to the real kernel.
 *   X       [in]  DEVICE, rows x n 16-bit elements, leading dimension ld >= n (a multiple of 8),
 *                 16-byte aligned
 *   n       [in]  a multiple of 512, at most 8192
 *   codes   [out] DEVICE, rows * n * bits / 8 bytes, 4-byte aligned;  scales [out] DEVICE, rows floats
 * Errors: RQ_ERR_ARG, RQ_ERR_HIP.
 */
int rq_stream_reference(const void* X, int64_t rows, int n, int64_t ld, int bits, void* codes,
                        float* scales, void* stream);

/*
 * The per-token symmetric quantizer of section 2.1 (with the clip ratio of section 3.1) on the
 * rows as they are, without a rotation: for activations whose rotation has been fused into the
 * neighbouring weights offline (section 2.2), so that only the quantizer remains online.
 *   X       [in]  DEVICE, rows x d elements of `dtype`, leading dimension ld >= d
 *   d       [in]  row width, a multiple of 32
 *   codes   [out] DEVICE, rows * d * bits / 8 bytes, 4-byte aligned (signed fields, same layout)
 *   scales  [out] DEVICE, rows floats: Delta = clip * max|x| / (2^b - 1)
 * Runs on the current device.  rows == 0 is a successful no-op.
 * Errors: RQ_ERR_ARG, RQ_ERR_HIP.
 */
int rq_quantize(const void* X, int dtype, int64_t rows, int d, int64_t ld,
                int bits, float clip, void* codes, float* scales, void* stream);

/*
 * The asymmetric group quantizer of rq_rotate_quantize_asym on the rows as they are, without a
 * rotation (section 5.1 for a tensor whose rotation is fused into the producing weights, e.g. the
 * value cache): per group of RQ_GROUP consecutive values lo = clip * min, hi = clip * max,
 * Delta = (hi - lo) / (2^b - 1), code = clamp(round((x - lo) / Delta), 0, 2^b - 1).
 *   X       [in]  DEVICE, rows x d elements of `dtype`, leading dimension ld >= d
 *   d       [in]  row width, a multiple of RQ_GROUP
 *   codes   [out] DEVICE, rows * d * bits / 8 bytes, 4-byte aligned (unsigned fields, same bit stream)
 *   scales  [out] DEVICE, rows * d / RQ_GROUP floats: Delta of each group
 *   mins    [out] DEVICE, rows * d / RQ_GROUP floats: lo of each group
 * Runs on the current device.  rows == 0 is a successful no-op.
 * Errors: RQ_ERR_ARG, RQ_ERR_HIP.
 */
int rq_quantize_asym(const void* X, int dtype, int64_t rows, int d, int64_t ld,
                     int bits, float clip, void* codes, float* scales, float* mins, void* stream);

/*
 * Rotation alone with a floating-point result: Y = (H_n pad(x) / sqrt(n))[:d_out] for every row,
 * or with H_n^T when transpose = 1.  Three uses:
 *   - the online rotation of a tensor that is not quantized afterwards (section 2.2: the part of
 *     the rotations that "needs to be done at inference"), e.g. the query heads, which must carry
 *     the same per-head rotation as the keys that go into the quantized cache;
 *   - offline weight fusion (section 4.2, Eq. 2): W' = H_n pad(W) / sqrt(n) is this call on the
 *     rows of W^T (input side) or of W (output side), so that rotate(x) W' = x W;
 *   - the inverse rotation x = H_n^T y / sqrt(n) (H_n^T H_n = n I, section 2.3) with
 *     transpose = 1 and d_out = the un-padded width.
 *   X        [in]  DEVICE, rows x d, leading dimension ld, `dtype` (as rq_rotate_quantize)
 *   Y        [out] DEVICE, rows x d_out elements of out_dtype (RQ_F32, or RQ_BF16 / RQ_F16 rounded
 *                  to nearest even), leading dimension ld_out >= d_out; 1 <= d_out <= n
 * rows == 0 is a successful no-op.
 * Errors: RQ_ERR_ARG, RQ_ERR_NO_ORDER (the row does not fit the kernel's LDS), RQ_ERR_HIP.
 */
int rq_rotate(const rq_hadamard_t* h, const void* X, int dtype, int64_t rows, int d, int64_t ld,
              int transpose, void* Y, int out_dtype, int d_out, int64_t ld_out, void* stream);

/*
 * Dequantize packed codes and rotate back (the inverse of rq_rotate_quantize up to the
 * quantization error): y^ = code * Delta (mins == NULL, signed codes) or code * Delta_g + lo_g
 * (mins != NULL, unsigned codes in groups of RQ_GROUP as written by rq_rotate_quantize_asym),
 * then Y = (H_n^T y^ / sqrt(n))[:d_out] with transpose = 1 (transpose = 0 applies H_n).
 *   codes, scales, mins [in] DEVICE, layouts as the quantizing calls write them
 *   Y                   [out] as in rq_rotate
 * Errors: RQ_ERR_ARG, RQ_ERR_NO_ORDER, RQ_ERR_HIP.
 */
int rq_dequantize_rotate(const rq_hadamard_t* h, const void* codes, const float* scales,
                         const float* mins, int64_t rows, int bits, int transpose,
                         void* Y, int out_dtype, int d_out, int64_t ld_out, void* stream);

/*
 * Dequantize in the rotated, normalised domain (section 2.1: X^ = round(X / Delta) * Delta), no
 * rotation: Y[r, j] = code_j * scales[r] for the signed codes rq_rotate_quantize / rq_quantize write.
 *   h       [in]  handle of the order n the codes were written with (n codes per row)
 *   codes   [in]  DEVICE, rows * n * bits / 8 bytes, 4-byte aligned
 *   scales  [in]  DEVICE, rows floats
 *   Y       [out] DEVICE, rows x n floats, row-major, leading dimension n, 4-byte aligned, caller-owned
 * The product is a single fp32 multiplication.  rows == 0 is a successful no-op.
 * Errors: RQ_ERR_ARG (NULL or misaligned pointer, rows < 0, bits not 3/4), RQ_ERR_HIP.
 */
int rq_dequantize(const rq_hadamard_t* h, const void* codes, const float* scales, int64_t rows, int bits,
                  float* Y, void* stream);

/*
 * The same for the unsigned group codes of rq_rotate_quantize_asym / rq_quantize_asym (section 5.1):
 * Y[r, j] = code_j * scales[r, g] + mins[r, g], g = j / RQ_GROUP, one fused multiply-add.
 *   scales, mins [in] DEVICE, rows * (n / RQ_GROUP) floats each
 * Errors: RQ_ERR_ARG (as rq_dequantize, or n not a multiple of RQ_GROUP), RQ_ERR_HIP.
 */
int rq_dequantize_asym(const rq_hadamard_t* h, const void* codes, const float* scales, const float* mins,
                       int64_t rows, int bits, float* Y, void* stream);

/*
 * Lemma "Expanding limit" (section 4.2): the largest number of added dimensions d for which a
 * product over n + d dimensions at bits_reduced bits costs no more bit operations than the
 * product over n dimensions at `bits` bits: (n + d) * bits_reduced <= n * bits, i.e.
 * floor(n (bits - bits_reduced) / bits_reduced).  Host-only; d_max is a HOST pointer.
 * Errors: RQ_ERR_ARG (n < 1, bits_reduced < 1, bits_reduced > bits, bits > 64, NULL).
 */
int rq_expand_limit(int n, int bits, int bits_reduced, int64_t* d_max);

/* Bytes of device workspace rq_quant_error needs for (rows, n_clips); 0 on bad arguments. */
size_t rq_quant_error_workspace(int64_t rows, int n_clips);

/*
 * Quantization error of the rotated rows for several clip ratios in one pass (the
 * objective a clip-ratio search evaluates repeatedly; sections 3.1, 4.1):
 *   mse[k] = (1 / (rows * n)) * sum over rows, j of (code_j * Delta_k - y_j)^2,
 * with y, Delta_k = clips[k] * amax / (2^b - 1) and code_j as in rq_rotate_quantize.
 *   clips     [in]  HOST pointer, n_clips floats in (0, 1]; read before the call returns
 *   n_clips   [in]  1 .. RQ_MAX_CLIPS
 *   mse       [out] DEVICE pointer, n_clips floats, caller-owned
 *   workspace [in]  DEVICE pointer, at least rq_quant_error_workspace(rows, n_clips) bytes,
 *                   8-byte aligned, caller-owned; contents are scratch
 * Other arguments as in rq_rotate_quantize.  rows == 0 writes zeros to mse (X may then be NULL).
 * The result is deterministic (fixed reduction order).
 * Errors: RQ_ERR_ARG (as above, n_clips out of range, a clip not in (0,1], workspace too small
 * or misaligned), RQ_ERR_NO_ORDER (as rq_rotate_quantize), RQ_ERR_HIP.
 */
int rq_quant_error(const rq_hadamard_t* h,
                   const void* X, int dtype, int64_t rows, int d, int64_t ld, int bits,
                   const float* clips, int n_clips,
                   float* mse, void* workspace, size_t workspace_bytes, void* stream);

/*
 * rq_quant_error with the asymmetric group quantizer of rq_rotate_quantize_asym (sections 4.1, 5.1:
 * the objective of a clip search on the KV cache): mse[k] = (1 / (rows * n)) * sum of
 * (code * Delta_g + lo_g - y)^2 at clip ratio clips[k].  The order n must be a multiple of RQ_GROUP.
 * Arguments, workspace size (rq_quant_error_workspace) and errors as rq_quant_error.
 */
int rq_quant_error_asym(const rq_hadamard_t* h,
                        const void* X, int dtype, int64_t rows, int d, int64_t ld, int bits,
                        const float* clips, int n_clips,
                        float* mse, void* workspace, size_t workspace_bytes, void* stream);

/*
 * For callers that cannot allocate device memory - code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc: rq_quant_error without a workspace argument.  The per-row
 * partial sums go to a static device array of RQ_NOALLOC_SCRATCH_BYTES that every GPU the library runs
 * on holds until the process ends (its address on the handle's device is taken when the handle is
 * built).  The call allocates nothing and frees nothing; same kernels and same results as
 * rq_quant_error.
 *   limit: rq_quant_error_workspace(rows, n_clips) <= RQ_NOALLOC_SCRATCH_BYTES, i.e.
 *          rows * n_clips <= 524288 (e.g. 8192 rows x 64 clip ratios); beyond it RQ_ERR_TOO_LARGE.
 * All calls on one GPU share the array: calls that may overlap in time on that GPU (different
 * streams, or different host threads) race on it and must be ordered by the caller.  The handle's
 * device must be the current device.
 * Other arguments and errors as rq_quant_error.
 */
#define RQ_NOALLOC_SCRATCH_BYTES (4u << 20)
int rq_quant_error_noalloc(const rq_hadamard_t* h,
                           const void* X, int dtype, int64_t rows, int d, int64_t ld, int bits,
                           const float* clips, int n_clips, float* mse, void* stream);

/* Bytes of device workspace rq_gbs_search needs for `rows` rows; 0 on bad arguments. */
size_t rq_gbs_workspace(int64_t rows);

/*
 * Clip-ratio search for one projection: the inner loop of the Gradual Binary Search
 * (section 4.1, Algorithm 1) with f(clip) = rq_quant_error of X at that single clip ratio as
 * the objective (the paper's objective, perplexity of a model, is not available here).
 * a = 0, b = 1, m = 1/2; iterations alternate the probes (a + m)/2 and (b + m)/2; a probe with
 * f(x) < f(m) becomes the new middle and the far bracket end moves to the old middle, otherwise
 * the bracket end on the probe's side moves to the probe; stops when b - a <= eps or after
 * max_evals evaluations of f.  The probes and their values are those of that loop taken one at a
 * time; they are evaluated ahead, and the comparisons are taken on the device.  For eps >= 1 / 256 every
 * probe there can be is a multiple of 1 / 512: bf16 and fp16 rows of the wave and workgroup kernels (16-byte
 * aligned, ld and d multiples of 8) are passed over once with all of these evaluated at once, where the search may take
 * enough steps to be worth it ("grid_search").  Otherwise, rows the chip can hold in registers are rotated once and
 * searched in one launch ("gbs_resident", or, to the same values bit for bit, with a launch for every three steps where
 * other work keeps that one from running, "gbs_stepped"); other tensors take a few launches of rq_quant_error's kernels
 * enqueued together, each of which evaluates every probe the next few steps can ask for.  f is summed in an order
 * of the search's own: it agrees with rq_quant_error to 2e-6 (relative), not to the last bit (nor do searches that
 * take different forms).  The same call gives the same result.
 * The call waits for the result: a calibration call, not a hot-path call (not for a stream under
 * capture).  Besides the workspace a search uses static device memory (as rq_quant_error_noalloc does: 16.9 MB, 1 MB
 * for each of 16 searches at once, part of the library on every device it is loaded on) and 256 KB of
 * device and 33 KB of pinned host memory that the first search on a device allocates and that stay until the process
 * ends; where the pinned memory cannot be had the results are copied back on `stream` instead, and more than 16 searches
 * at once on a device allocate 1 MB for the call.  Searches may run on any number of threads and streams; one at a
 * time per device takes the "gbs_resident" form, where others take its steps one launch at a time.
 *   eps          [in]  bracket width to stop at, > 0
 *   max_evals    [in]  1 .. 256
 *   workspace    [in]  DEVICE, >= rq_gbs_workspace(rows) bytes, 8-byte aligned, scratch
 *   clip_out     [out] HOST, the final middle m
 *   mse_out      [out] HOST, f(m)
 *   trace_clips  [out] HOST, max_evals floats or NULL: the probes in evaluation order
 *   trace_mse    [out] HOST, max_evals floats or NULL: f at those probes
 *   n_evals      [out] HOST or NULL: number of evaluations made
 * X, dtype, rows (>= 1), d, ld, bits as in rq_rotate_quantize.
 * Errors: RQ_ERR_ARG, RQ_ERR_NO_ORDER, RQ_ERR_HIP.
 */
int rq_gbs_search(const rq_hadamard_t* h, const void* X, int dtype, int64_t rows, int d, int64_t ld,
                  int bits, float eps, int max_evals, void* workspace, size_t workspace_bytes,
                  void* stream, float* clip_out, float* mse_out, float* trace_clips,
                  float* trace_mse, int* n_evals);

/* rq_gbs_search with rq_quant_error_asym as the objective (n a multiple of RQ_GROUP). */
int rq_gbs_search_asym(const rq_hadamard_t* h, const void* X, int dtype, int64_t rows, int d, int64_t ld,
                       int bits, float eps, int max_evals, void* workspace, size_t workspace_bytes,
                       void* stream, float* clip_out, float* mse_out, float* trace_clips,
                       float* trace_mse, int* n_evals);

/*
 * The 4-bit paged key / value cache: where the keys and values of a served model go once they are rotated and quantized
 * (section 5.1: asymmetric, a group a head row), and attention that reads them.
 *
 * A cache is `pages` pages of page_size tokens in one piece of device memory, page after page.  A token is named by its slot,
 * page * page_size + place in the page.  For each kv head a page has one block of page_size * (head_dim + 8) bytes:
 *     key codes         page_size rows of head_dim / 2 bytes; element j is the nibble at bits [4 j, 4 j + 4) of the row's
 *                       little-endian bit stream
 *     value codes       [page_size / 4][16][head_dim / 64][4] halfwords: halfword [t / 4][r][f][t % 4] holds elements
 *                       r * head_dim / 16 + 4 f + 0 .. 3 of token t, the first in its low bits
 *     key parameters    page_size dwords: step in the low half, centre in the high half, both bfloat16
 *     value parameters  likewise
 * and an element is (code - 7.5) * step + centre.  Quantizer, per head row y (fp32, every operation rounded to nearest even):
 *     lo = clip * min(y), hi = clip * max(y), step = bf16((hi - lo) / 15), centre = bf16((hi + lo) / 2),
 *     code = clamp(rne((y - centre) * (1 / step) + 7.5), 0, 15);
 * a step below 2^-100 is stored as 0.  A row with infinities or NaN has a step that is NaN; other rows are not affected.
 * Keys are rotated by the handle's H_n / sqrt(n), n = head_dim (a Sylvester order: 64, 128); h NULL: not at all.  Queries
 * then carry the same rotation, which rq_kv4_attention applies to them.  Values are stored as they come: their rotation is folded into
 * the neighbouring weights (section 2.2).
 * The calls take the current device, enqueue on `stream` and neither wait nor allocate; all of them can be captured in a graph.
 */
#define RQ_KV4_MAX_HEADS 1024

typedef struct rq_kv4 {
    void* data;        /* DEVICE, pages * rq_kv4_page_bytes(...) bytes, 16-byte aligned; caller-owned */
    int64_t pages;     /* at most 2^31 - 1 */
    int kv_heads;      /* 1 .. RQ_KV4_MAX_HEADS */
    int head_dim;      /* 64 or 128 */
    int page_size;     /* tokens of a page: 16, 32, 64, 128 or 256 */
} rq_kv4_t;

/* Bytes of a page: kv_heads * page_size * (head_dim + 8); 0 on bad arguments. */
size_t rq_kv4_page_bytes(int kv_heads, int head_dim, int page_size);

/*
 * Rotate (keys), quantize and write the rows of `tokens` tokens to their slots.
 *   K, V      [in]  DEVICE, element [token][head][i] at token * *_token_stride + head * *_head_stride + i (strides in elements, >= 0)
 *   dtype     [in]  RQ_BF16, RQ_F16 or RQ_F32
 *   slots     [in]  DEVICE, tokens int64; a token whose slot is negative or not in the cache is left out.  Two tokens of a
 *                   call must not have the same slot.
 *   clip      [in]  clip ratio in (0, 1]
 * Errors: RQ_ERR_ARG (bad cache, order of h not head_dim, dtype, clip, negative stride, NULL or misaligned pointer), RQ_ERR_HIP.
 */
int rq_kv4_append(const rq_hadamard_t* h, const rq_kv4_t* cache, const void* K, const void* V, int dtype, int64_t tokens,
                  int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride, int64_t v_head_stride,
                  const int64_t* slots, float clip, void* stream);

/*
 * The rows of `rows` slots as numbers: K and V [rows][kv_heads][head_dim] of out_dtype, rounded to nearest even.  With h the keys
 * are rotated back to the original basis, with NULL they are the values that are stored.  A slot that is negative or not in
 * the cache gives zeros.
 *   K, V      [out] DEVICE, 16-byte aligned
 * Errors: RQ_ERR_ARG, RQ_ERR_HIP.
 */
int rq_kv4_read(const rq_hadamard_t* h, const rq_kv4_t* cache, const int64_t* slots, int64_t rows, void* K, void* V, int out_dtype,
                void* stream);

/*
 * Copy whole pages, page src[i] to page dst[i] in each of `layers` caches that lie layer_stride bytes apart: forked sequences whose
 * last page becomes their own, and compaction.  No page may be named twice in dst, nor be both in src and in dst (but for
 * src[i] == dst[i], which does nothing); a pair with a page that is not in the cache is left out.
 *   src, dst      [in]  DEVICE, `pairs` int32 each
 *   layer_stride  [in]  at least pages * page bytes, a multiple of 16; not looked at with one layer
 * Errors: RQ_ERR_ARG, RQ_ERR_HIP.
 */
int rq_kv4_copy_pages(const rq_kv4_t* cache, int layers, int64_t layer_stride, const int32_t* src, const int32_t* dst, int64_t pairs,
                      void* stream);

/*
 * Bytes of device workspace rq_kv4_attention needs for such a call on the current device; 0 where it needs none and on bad
 * arguments.  decode: q_start will be NULL.
 */
size_t rq_kv4_attention_workspace(const rq_kv4_t* cache, int64_t tokens, int heads, int batch, int decode, int window, int64_t max_len);

/*
 * Attention of a batch of sequences over their cached keys and values:
 *     o = sum_j softmax_j(scale * q . k_j) v_j   over the positions j that the query sees.
 * Sequence b has kv_lens[b] positions, position j in slot table[b][j / page_size] * page_size + j % page_size.  Its queries are tokens
 * q_start[b] .. q_start[b + 1] - 1 and stand at its last positions: query i of n at kv_lens[b] - n + i.  A causal query sees
 * positions up to its own, others all of the sequence; with a window w > 0 only those later than its own minus w.  A query that sees
 * nothing gets zeros (and -infinity in lse).
 * Query head x reads kv head x / (heads / kv_heads).
 *
 * What is rounded: queries are rotated as the keys were (h), multiplied by scale * log2(e) and by a power of two of the row's, in fp32,
 * and rounded to fp16 (for fp16 results: to two fp16 numbers); probabilities times the steps of the values are rounded to fp16; all else
 * is fp32.  bf16 results of the kernel for many queries (rq_kv4_attention_plan: many) come from keys, values and
 * probabilities rounded to fp16 each, weights below 2^-32 of a row's largest count as 0 there.
 * Steps (there: elements) carry a power of two on their way into fp16, which follows the largest among the keys that a row tile has come
 * to, whether all of its rows see that key or not.  Beside a value whose step is the largest, values lose digits whose steps are
 * less than 2^-20 of it, and are lost below 2^-31; there: elements of keys and of values below 2^-28 of the largest, and below 2^-40.
 * A key or value that is not finite makes the results of rows that see it NaN, and of no others.  (So may a finite key whose product
 * with a query row, scaled to at most 1, leaves fp32: elements of 2^120 and more.)
 *   Q            [in]  DEVICE, element [token][head][i] at token * q_token_stride + head * q_head_stride + i
 *   dtype        [in]  RQ_BF16 or RQ_F16, of Q and O
 *   tokens       [in]  0 .. 2^24
 *   heads        [in]  a multiple of kv_heads, at most 256 times it
 *   table        [in]  DEVICE, batch x width int32 page numbers; what stands behind a sequence's last page does not matter, and a
 *                      number that is not in the cache stands for page 0
 *   kv_lens      [in]  DEVICE, batch int32; values are taken to be in 0 .. max_len
 *   q_start      [in]  DEVICE, batch + 1 int32, ascending from 0 to tokens; NULL: one token a sequence (tokens == batch)
 *   scale        [in]  of the scores, finite, > 0
 *   causal       [in]  0 or 1;  window [in]  0: none
 *   max_len      [in]  no sequence is longer; at most width * page_size and 2^30.  It bounds the work that is laid out.
 *   O            [out] as Q with its own strides, which are head_dim at least where there are two tokens, two heads; rows must not overlap
 *                      each other nor Q
 *   lse          [out] DEVICE, tokens x heads floats, log of the sum of exp(scale * q . k_j), or NULL
 *   workspace    [in]  DEVICE, >= rq_kv4_attention_workspace(...) bytes, 16-byte aligned, scratch; NULL where that is 0
 * Long sequences are split over workgroups and joined in a fixed order: the same call gives the same bits.
 * Errors: RQ_ERR_ARG, RQ_ERR_HIP.
 */
int rq_kv4_attention(const rq_hadamard_t* h, const rq_kv4_t* cache, const void* Q, int dtype, int64_t tokens, int heads,
                     int64_t q_token_stride, int64_t q_head_stride, const int32_t* table, int batch, int width, const int32_t* kv_lens,
                     const int32_t* q_start, float scale, int causal, int window, int64_t max_len, void* O, int64_t o_token_stride,
                     int64_t o_head_stride, float* lse, void* workspace, size_t workspace_bytes, void* stream);

/*
 * How rq_kv4_attention lays out such a call (testing / measurement): by these numbers alone, on a device of `compute_units`; 0: the
 * current device's.  tokens and batch at least 1.
 */
typedef struct rq_kv4_plan {
    int many;          /* 0: the kernel for few queries a sequence, 1: the one for many */
    int rows;          /* queries x heads of a row tile, all of one sequence and kv head */
    int waves;         /* of a workgroup; many: of a group of them */
    int groups;        /* many: groups of a workgroup, which share its keys out */
    int tiles;         /* row tiles of a kv head at most */
    int workers;       /* few: workgroups of a kv head that share all keys out; 0: a workgroup a row tile */
    int chunk, chunks; /* many: a row tile's keys, from the first that one of its rows sees (rounded down to 64), are `chunks` times
                          `chunk` at most, a workgroup each */
} rq_kv4_plan_t;

int rq_kv4_attention_plan(const rq_kv4_t* cache, int dtype, int64_t tokens, int heads, int batch, int decode, int causal, int window,
                          int64_t max_len, int compute_units, rq_kv4_plan_t* plan);

/*
 * Bytes of device workspace rq_kv4_prefix_attention needs for such a call on the current device; 0 where it needs none and on bad
 * arguments.  At most 2^30 (but for a query whose heads alone take more): partial results are fp32 and two of each result at least, and calls
 * with more of them take their queries in turns, the same kernels one after the other.  decode: q_start will be NULL.
 */
size_t rq_kv4_prefix_attention_workspace(const rq_kv4_t* cache, int64_t tokens, int heads, int groups, int batch, int decode, int window,
                                         int64_t max_prefix, int64_t max_len);

/*
 * rq_kv4_attention for sequences that begin alike (branches of a prompt, requests behind a system prompt): the pages that a group of them
 * shares are read for all of its queries together.  Sequences group_start[g] .. group_start[g + 1] - 1 have the first prefix_lens[g]
 * positions in common, position j in slot prefix_table[g][j / page_size] * page_size + j % page_size; position prefix_lens[g] + j of
 * sequence b is in slot table[b][j / page_size] * page_size + j % page_size, and there are kv_lens[b] of these.  The queries of a sequence
 * stand at the last of all its positions, and see what rq_kv4_attention's do.  Any group may have one sequence or none, any prefix and any
 * sequence no positions; a prefix need not end with its page.
 *   prefix_table [in]  DEVICE, groups x prefix_width int32 page numbers;  prefix_lens: DEVICE, groups int32, taken to be in 0 .. max_prefix
 *   group_start  [in]  DEVICE, groups + 1 int32, ascending from 0 to batch
 *   table, kv_lens, max_len   of what is behind the prefixes; max_prefix: no prefix is longer, at most prefix_width * page_size;
 *                max_prefix + max_len at most 2^30
 * Other arguments and errors as rq_kv4_attention; the same call gives the same bits.
 * What is rounded: as in rq_kv4_attention, for prefixes and what is behind them by the kernel that takes either.  Which one does goes by the
 * rows of a whole group, not of a sequence: bf16 results of single queries, too, come from keys, values and probabilities of the prefix
 * rounded to fp16 each where many of them share a long one (rq_kv4_prefix_attention_plan: many; own_many: what is behind).
 * Where it is of no use: with a window that hides positions, or with max_prefix below 64, each sequence takes its prefix and its own
 * positions by itself, on one workgroup for each 16 of its queries x heads or fewer, however long (plan: separate).  There, and for sequences that
 * share little of what they see, rq_kv4_attention on whole tables is as fast or faster: 16 x 32 heads behind 4096 positions, window 1024,
 * 10.8 and 11.0 us; two sequences of 8 heads behind 65536, window 60000, 23 and 195; one of 131072 positions behind 32, 28 and 489.
 */
int rq_kv4_prefix_attention(const rq_hadamard_t* h, const rq_kv4_t* cache, const void* Q, int dtype, int64_t tokens, int heads,
                            int64_t q_token_stride, int64_t q_head_stride, const int32_t* prefix_table, int groups, int prefix_width,
                            const int32_t* prefix_lens, const int32_t* group_start, const int32_t* table, int batch, int width, const int32_t* kv_lens,
                            const int32_t* q_start, float scale, int causal, int window, int64_t max_prefix, int64_t max_len, void* O,
                            int64_t o_token_stride, int64_t o_head_stride, float* lse, void* workspace, size_t workspace_bytes, void* stream);

/*
 * How rq_kv4_prefix_attention lays out such a call (testing / measurement), as rq_kv4_attention_plan does.
 */
typedef struct rq_kv4_prefix_plan {
    int separate;      /* 1: each sequence takes its prefix and its own positions in one launch (then only own_rows, waves count) */
    int waves;         /* of a workgroup: separate; else 4 for few rows, 4 times the groups of waves for many */
    int many, own_many;                /* kernel for many rows: for the prefixes, for what is behind them */
    int shared_rows, own_rows;         /* queries x heads of a row tile */
    int shared_chunk, shared_chunks;   /* a row tile's keys of the prefix: shared_chunks times shared_chunk at most */
    int own_chunk, own_chunks;         /* behind it */
} rq_kv4_prefix_plan_t;

int rq_kv4_prefix_attention_plan(const rq_kv4_t* cache, int dtype, int64_t tokens, int heads, int groups, int batch, int decode, int window,
                                 int64_t max_prefix, int64_t max_len, int compute_units, rq_kv4_prefix_plan_t* plan);

/*
 * How much attention the positions of cached sequences receive, for deciding which of them to keep:
 *     weights[b][y][j] <- decay * weights[b][y][j] + sum over the queries of sequence b and the heads x of kv head y of
 *                         exp(scale * q . k_j - lse)
 * for the positions j < kv_lens[b]; a query adds to positions that it sees only, and weights behind a sequence's last position stay what
 * they are.  With decay 0 the old weights are not read.
 * Arguments and what a query sees are rq_kv4_attention's; its lse is the one wanted here (that of bf16 results is off by the rounding of
 * their queries, about 2^-12 of a score: so are the weights).  Here queries are rounded to 22 bits, all else is fp32.  Not finite: a key makes its
 * own weights NaN, a query those of all positions that it sees.
 *   lse          [in]  DEVICE, tokens x heads floats
 *   tokens       [in]  0 .. 2^24 (none: the weights decay)
 *   decay        [in]  0 .. 1
 *   weights      [inout] DEVICE, element [b][y][j] at b * w_seq_stride + y * w_head_stride + j; rows of max_len must not overlap
 *   max_len      [in]  times batch, at most 2^37
 *   workspace    [in]  DEVICE, >= rq_kv4_attention_weights_workspace(...) bytes, 16-byte aligned, scratch; NULL where that is 0 (none for single
 *                      queries of 16 heads a kv head at most; else 4 head_dim + 16 bytes for each query and head, and 4 for each position and kv
 *                      head in each share of the queries)
 * The same call gives the same bits.  Errors: RQ_ERR_ARG, RQ_ERR_HIP.
 */
size_t rq_kv4_attention_weights_workspace(const rq_kv4_t* cache, int64_t tokens, int heads, int batch, int decode, int window, int64_t max_len);
int rq_kv4_attention_weights(const rq_hadamard_t* h, const rq_kv4_t* cache, const void* Q, int dtype, int64_t tokens, int heads,
                             int64_t q_token_stride, int64_t q_head_stride, const float* lse, const int32_t* table, int batch, int width,
                             const int32_t* kv_lens, const int32_t* q_start, float scale, int causal, int window, int64_t max_len, float decay,
                             float* weights, int64_t w_seq_stride, int64_t w_head_stride, void* workspace, size_t workspace_bytes, void* stream);

/*
 * The positions of each layer, sequence and kv head that are worth keeping: the first `sinks`, the last `recent`, and of those between the
 * ones with the largest weights, `keep` in all (ties: the lower positions; NaN is less than any number).
 *   weights      [in]  DEVICE, element [layer][b][y][j] at layer * w_layer_stride + b * w_seq_stride + y * w_head_stride + j
 *   n            [in]  positions of a row of weights, at most 2^30; kv_lens are taken to be in 0 .. n
 *   kv_lens      [in]  DEVICE, batch int32
 *   keep         [in]  at least sinks + recent
 *   index        [out] DEVICE, layers x batch x kv_heads x keep int32, each row ascending; a sequence of no more than `keep` positions keeps
 *                      all of them, and -1 stands in the places behind
 * Errors: RQ_ERR_ARG, RQ_ERR_HIP.
 */
int rq_kv4_select(const float* weights, int layers, int batch, int kv_heads, int64_t n, int64_t w_layer_stride, int64_t w_seq_stride,
                  int64_t w_head_stride, const int32_t* kv_lens, int64_t keep, int64_t sinks, int64_t recent, int32_t* index, void* stream);

/*
 * The kept rows moved together: position i of a kv head becomes what its position index[layer][b][y][i] was, as it is stored.  A row
 * with a negative index or one that the table has no page for is not written.
 * In place (new_table NULL): index has to ascend, from at least i at place i on, as rq_kv4_select's does; a page must not be another
 * sequence's too.  Else the pages of new_table are written, none of which may be read by the call, nor be named twice.
 *   layers, layer_stride   as in rq_kv4_copy_pages; the tables hold for all layers
 *   index        [in]  DEVICE, layers x batch x kv_heads x keep int32
 *   table        [in]  DEVICE, batch x width int32;  new_table: batch x new_width.  Places of `keep` positions at least where they are written
 *   weights      [inout] DEVICE, as in rq_kv4_select, or NULL: moved along in place (index ascending here too); 0 from there to the end of
 *                      a row, for tokens to come.  n at least keep; rows must not overlap
 * Errors: RQ_ERR_ARG, RQ_ERR_HIP.
 */
int rq_kv4_evict(const rq_kv4_t* cache, int layers, int64_t layer_stride, const int32_t* index, int64_t keep, const int32_t* table, int batch, int width,
                 const int32_t* new_table, int new_width, float* weights, int64_t n, int64_t w_layer_stride, int64_t w_seq_stride,
                 int64_t w_head_stride, void* stream);

/*
 * Select the kernel family for subsequent hot-path calls on this handle (testing /
 * measurement): 0 = automatic (fastest available), 1 = the general LDS kernel; for long
 * power-of-two rows 2 = one wave per row at any row count, 3 / 4 = a row split over 2 / 4 waves
 * at any row count (automatic picks by the number of rows); 5 .. 7 are automatic but for
 * the searches: for tensors that fit the chip's registers 5 = a launch for every three steps ("gbs_stepped"),
 * 6 = one launch ("gbs_resident") whose workgroups do not wait for each other, so that it gives up and the
 * former takes over; 7 = no pinned memory (for every tensor the results copied back; the former form again where
 * automatic takes the latter).
 * Errors: RQ_ERR_ARG.
 */
int rq_hadamard_set_variant(rq_hadamard_t* h, int variant);

/* Name of the kernel family the last hot-path call on this handle used ("" if none). */
const char* rq_hadamard_last_kernel(const rq_hadamard_t* h);

/* Static description of an error code. */
const char* rq_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* ROTQ_H */
