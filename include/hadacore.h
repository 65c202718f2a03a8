/*
 * hadacore.h -- C ABI of libhadacore: batched, normalized Walsh-Hadamard
 * transform of fp16/bf16 rows on AMD Instinct MI355X (gfx950).
 *
 * Operation (HadaCore, arXiv 2412.08832, Sec. 2.1-2.2 and Sec. 2.4):
 * for every row i < m of an m x n matrix x of 16-bit floats,
 *
 *     out[i][j] = scale * sum_{k<n} (-1)^popcount(j & k) * in[i][k],  j < n,
 *
 * i.e. each row is multiplied on the right by the Sylvester-ordered
 * Walsh-Hadamard matrix H_n (natural order, +-1 entries), and by `scale`.
 * The normalized transform of the paper is scale = 1/sqrt(n); H_n is never
 * stored.  n is a power of two from 1 to 2^16: the paper's sizes are 2^7 to
 * 2^15 (Sec. 2.3-2.4 and Sec. 3.2 bound them at 2^15); the smaller ones and
 * 2^16 are supported as well (n = 1 is the identity times `scale`), and
 * hadamard_transform_ws goes on to 2^20.  In-place operation
 * (Appendix B) is supported.
 *
 * Numerics: inputs are scaled before any addition -- by `scale`, or by its
 * power-of-two part with the remaining factor (in [1, 2)) applied at the end --
 * so that large bf16 rows cannot overflow fp32 partial sums; all intermediates
 * are fp32 and the result is rounded once to the output dtype with
 * round-to-nearest-even.  Subnormals are preserved.
 * NaN/Inf propagate as IEEE arithmetic dictates.  Results are deterministic:
 * repeated calls, and in-place vs out-of-place calls, give identical bits.
 *
 * Memory: all pointers are DEVICE pointers owned by the caller; the library
 * never allocates, frees or retains them.  Rows are contiguous (element
 * stride 1) and start every `row_stride` elements; elements between n and the
 * row stride are neither read nor written.  Row strides are at most 2^26
 * elements (bytes for quantized codes), which keeps every offset inside a
 * group of rows handled by one wave below 2^32 bytes, and multiples of
 * min(n, 8) elements (codes: min(n, 16) bytes), so that every row starts on a
 * boundary of its access width.
 *
 * Streams: work is enqueued asynchronously on `stream` (a hipStream_t; NULL
 * means the default stream), which must belong to the current device (the
 * architecture check and launch shape use it), and the call returns without
 * synchronizing.
 * Buffers must stay alive until that work completes.  Faults in the enqueued
 * kernel surface at the caller's next synchronization, not here.  A call
 * enqueues kernel launches only (no allocation, memset or synchronization),
 * so it can be captured into a HIP graph once the first call on a device has
 * run outside capture (that call caches the device check); calls on
 * different streams may run concurrently.
 *
 * Kernels: per transform size the library picks one of two front ends for the
 * first stages, both giving results within fp32 rounding of each other: fp32
 * VALU butterflies, or one radix-32 step on the matrix cores (MFMA) applied
 * directly to the 16-bit inputs (n >= 128 only).  The environment variable
 * HADACORE_VARIANT set to "valu" or "mfma" forces one of them for n >= 128
 * (testing and tuning; read on every call); unset keeps the measured per-size
 * choice.  For 2^16 < n < 2^20 "passes" and "parts" force one of the two ways of
 * hadamard_transform_ws, and "parts-defer" also sets the waits of an in-place
 * call to zero, so that its parts go through the workspace; "parts-wait-N" to at
 * most N polls.  "tiles-64", "tiles-64x128", "tiles-128" and "tiles-256" force the
 * tile of the FP8 products (the last not for 32-bit outputs).
 *
 * Launches: a call is one kernel launch, or up to two for n > 2^16; m so
 * large that a launch would exceed 2^31 work-items (2^33 elements) is split
 * into several launches of consecutive rows on the same stream, with the
 * same result.
 *
 * Output alignment (performance only): an output (or code array) that starts
 * on a 128-byte boundary, with contiguous rows or a row pitch and row size
 * that are multiples of 128 bytes, takes a store path that is 1-3% faster at
 * most sizes.  Any other valid layout gives the same bytes.
 *
 * Errors: arguments are validated synchronously before anything is enqueued;
 * on error nothing is enqueued and a nonzero status is returned.  No call
 * aborts or throws.  The library keeps no state beyond a per-device cache of
 * the architecture check, the compute-unit count and the address of the
 * scratch array of hadamard_transform_ws_noalloc, and is safe to call from
 * several host threads.
 */
#ifndef HADACORE_H
#define HADACORE_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define HADACORE_VERSION 10400 /* 1.4.0: routing, the exchange by expert, low-rank adapters */

typedef int32_t hadacore_dtype;
#define HADACORE_FP16 0 /* IEEE binary16 */
#define HADACORE_BF16 1 /* bfloat16 */
#define HADACORE_FP32 2 /* IEEE binary32: outputs of the FP8 products; logits, exchange, adapters */

typedef int32_t hadacore_status;
#define HADACORE_SUCCESS 0
#define HADACORE_ERROR_INVALID_VALUE 1      /* m < 0, null pointer with m > 0, non-finite scale */
#define HADACORE_ERROR_INVALID_SIZE 2       /* n not a power of two in [1, 65536] (2^20 for _ws) */
#define HADACORE_ERROR_INVALID_DTYPE 3      /* dtype not HADACORE_FP16 / HADACORE_BF16 */
#define HADACORE_ERROR_INVALID_STRIDE 4     /* row stride < n, > 2^26, or not a multiple of min(n, 8) */
#define HADACORE_ERROR_MISALIGNED 5         /* in or out not 16-byte aligned */
#define HADACORE_ERROR_OVERLAP 6            /* in/out overlap without being the same layout */
#define HADACORE_ERROR_LAUNCH 7             /* the HIP runtime rejected the kernel launch */
#define HADACORE_ERROR_UNSUPPORTED_DEVICE 8 /* current device is not gfx950 */
#define HADACORE_ERROR_TOO_LARGE 9          /* m >= 2^31, or m * row stride > 2^40 */
#define HADACORE_ERROR_WORKSPACE 10         /* workspace NULL or below the required size */
#define HADACORE_ERROR_SCRATCH 11           /* hadamard_transform_ws_noalloc: needs more than
                                               HADACORE_NOALLOC_SCRATCH_BYTES of workspace */

/*
 * hadamard_transform -- out = scale * in * H_n for m dense rows of n elements.
 *   in     device pointer to m*n 16-bit values, 16-byte aligned (read only
 *          unless in == out)
 *   out    device pointer to m*n 16-bit values, 16-byte aligned; out == in
 *          selects in-place operation, any other overlap is rejected
 *   m      number of rows, >= 0; m == 0 returns HADACORE_SUCCESS and enqueues
 *          nothing (pointers may then be NULL)
 *   n      transform length, a power of two in [1, 65536]
 *   dtype  HADACORE_FP16 or HADACORE_BF16 (input and output share it)
 *   scale  finite fp32 multiplier; 1/sqrt(n) gives the orthonormal transform
 *   stream hipStream_t to enqueue on (NULL = default stream)
 * Same as hadamard_transform_strided with both row strides equal to n.
 */
hadacore_status hadamard_transform(const void *in, void *out, int64_t m, int64_t n,
                                   hadacore_dtype dtype, float scale, void *stream);

/*
 * hadamard_transform_strided -- as hadamard_transform, with row i of the input
 * at in + i*in_row_stride and row i of the output at out + i*out_row_stride
 * (strides in elements, each >= n, <= 2^26 and a multiple of min(n, 8)).  In-place operation
 * requires in == out and in_row_stride == out_row_stride.
 */
hadacore_status hadamard_transform_strided(const void *in, int64_t in_row_stride, void *out,
                                           int64_t out_row_stride, int64_t m, int64_t n,
                                           hadacore_dtype dtype, float scale, void *stream);

/*
 * hadamard_transform_workspace_size -- bytes of device workspace that
 * hadamard_transform_ws needs for m rows of n elements: 4*m*n (one fp32 value
 * per element) for 2^16 < n <= 2^20, 0 for n <= 2^16.  Returns 0 as well for
 * arguments hadamard_transform_ws rejects; the call reports why.
 */
int64_t hadamard_transform_workspace_size(int64_t m, int64_t n);

/*
 * hadamard_transform_ws -- as hadamard_transform_strided, for n up to 2^20.
 * Sizes above 2^16 (the paper's range ends at 2^15, Sec. 3.2) do not fit one
 * workgroup's registers in fp32.  They run in one of two ways with the same
 * results, chosen by measured speed from n, m and the mode.
 *  - In one pass (most of 2^17 and 2^18, some of 2^19): several workgroups share
 *    a row, each reading all of it and computing a part of the outputs.  In
 *    place they wait for each other's reads through words in the workspace, with
 *    a wait that is bounded for the whole launch: a part that cannot be stored in
 *    time goes through the workspace.
 *  - In two passes (2^20, and the rest): pass 1 applies `scale` and the stages on
 *    index bits 15..log2(n)-1 (between the 2^15-element blocks of a row) into
 *    fp32 values in the workspace, pass 2 the stages on bits 0..14 within each
 *    block, and rounds once, with 12 bytes of HBM traffic per element.
 * Every intermediate stays fp32, so the numerics are those of the one-pass
 * sizes.  For n <= 2^16 the call is hadamard_transform_strided and the workspace
 * is not touched.
 *   workspace        device pointer, 16-byte aligned, at least
 *                    hadamard_transform_workspace_size(m, n) bytes, not
 *                    overlapping in or out (NULL allowed for n <= 2^16)
 *   workspace_bytes  its size in bytes
 * The workspace is scratch: its contents on return are unspecified, and two
 * calls in flight at once need two workspaces.  Other arguments, strides,
 * streams and errors as for hadamard_transform_strided, plus
 * HADACORE_ERROR_WORKSPACE.  The quantizing entry points stop at n = 2^16.
 */
hadacore_status hadamard_transform_ws(const void *in, int64_t in_row_stride, void *out,
                                      int64_t out_row_stride, int64_t m, int64_t n,
                                      hadacore_dtype dtype, float scale, void *workspace,
                                      int64_t workspace_bytes, void *stream);

/*
 * hadamard_transform_ws_noalloc -- hadamard_transform_ws for callers that
 * cannot allocate device memory (code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc): the same kernels and results, with
 * the workspace taken from a fixed array inside the library instead of
 * an argument.  The call itself allocates nothing (no hipMalloc, hipFree or
 * allocating library routine).
 *   The array is HADACORE_NOALLOC_SCRATCH_BYTES (32 MiB) of device memory per
 *   GPU, held from the library's first use on that GPU until the process
 *   ends; for n > 2^16 the call needs hadamard_transform_workspace_size(m, n)
 *   <= HADACORE_NOALLOC_SCRATCH_BYTES (m * n <= 2^23 elements: e.g. 64 rows of
 *   2^17, 8 rows of 2^20) and returns HADACORE_ERROR_SCRATCH beyond that,
 *   enqueuing nothing.  For n <= 2^16 it is hadamard_transform_strided.
 *   Every call on one GPU uses that GPU's one array: calls that can overlap
 *   in time on the same GPU (different streams, host threads) race and give
 *   undefined results; calls in one stream's order are safe.  Nothing in the
 *   array needs to start at zero (every call writes what it reads).  The first
 *   call on a device looks up that device's address of the array
 *   (HADACORE_ERROR_LAUNCH if the runtime cannot give it); run that call outside
 *   graph capture.
 * Other arguments, strides, streams and errors as for hadamard_transform_ws.
 */
#define HADACORE_NOALLOC_SCRATCH_BYTES (32LL << 20)
hadacore_status hadamard_transform_ws_noalloc(const void *in, int64_t in_row_stride, void *out,
                                              int64_t out_row_stride, int64_t m, int64_t n,
                                              hadacore_dtype dtype, float scale, void *stream);

/*
 * hadamard_transform_fp8 -- the transform fused with per-row quantization to
 * OCP FP8 e4m3 (the fused Hadamard transform + quantization that the paper
 * names as future work, Sec. 5; rotations precede FP8 attention, Sec. 4.2).
 * For every row i, with y = scale * in[i] * H_n computed as above:
 *     amax_i          = max_j |y_j|   (NaN ignored unless the row is all NaN)
 *     out_scales[i]   = amax_i / 448  (fp32, correctly rounded)
 *     out_codes[i][j] = e4m3 round-to-nearest-even of y_j * (448 / amax_i)
 *                       (448/amax_i taken as 0 where it is not finite: a zero
 *                       or NaN row, or amax_i < 448 * 2^-128, whose codes are
 *                       then +-0)
 * so that y_j ~ decode_e4m3(out_codes[i][j]) * out_scales[i].  e4m3: 1 sign,
 * 4 exponent (bias 7) and 3 fraction bits, largest finite 448, 0x7f NaN.
 *   in              device pointer, m rows of n 16-bit values at in_row_stride
 *                   elements (>= n, <= 2^26, multiple of min(n, 8)), 16-byte
 *                   aligned
 *   out_codes       device pointer, m rows of n bytes at out_row_stride bytes
 *                   (>= n, <= 2^26, multiple of min(n, 16)), 16-byte aligned
 *   out_scales      device pointer to m floats, 4-byte aligned
 * The three ranges must not overlap (OVERLAP otherwise).  Other arguments,
 * streams, ownership and errors as for hadamard_transform.
 */
hadacore_status hadamard_transform_fp8(const void *in, int64_t in_row_stride, void *out_codes,
                                       int64_t out_row_stride, float *out_scales, int64_t m,
                                       int64_t n, hadacore_dtype dtype, float scale, void *stream);

/*
 * hadamard_transform_int8 -- the transform fused with symmetric per-row INT8
 * quantization, the integer counterpart of hadamard_transform_fp8 (rotations
 * spread outliers so that one scale per row loses less, Sec. 1).  For every
 * row i, with y = scale * in[i] * H_n computed as above and amax_i as for FP8:
 *     out_scales[i]   = amax_i / 127  (fp32, correctly rounded)
 *     out_codes[i][j] = round-half-to-even of y_j * (127 / amax_i), an int8 in
 *                       [-127, 127] (the product rounded to fp32 first)
 * so that y_j ~ out_codes[i][j] * out_scales[i].  A row whose amax is 0, Inf or
 * NaN, or so small that 127 / amax_i overflows fp32 (amax_i < 127 * 2^-128),
 * gets all-zero codes; its scale is still amax_i / 127.  Arguments, layout,
 * alignment, overlap rules, streams and errors as for hadamard_transform_fp8.
 */
hadacore_status hadamard_transform_int8(const void *in, int64_t in_row_stride, void *out_codes,
                                        int64_t out_row_stride, float *out_scales, int64_t m,
                                        int64_t n, hadacore_dtype dtype, float scale, void *stream);

/*
 * FP8 codes with a scale for each block of 128, and their products.
 *
 * A block of 128 values y is stored as e4m3 codes and one fp32 scale, as a row is by
 * hadamard_transform_fp8:
 *     amax = max |y| (NaN ignored unless the block is all NaN),
 *     scale = amax / 448, code = e4m3 of y * (448 / amax), 448 / amax taken as 0 where
 *     it is not finite.
 * A block lies along a row (activations), down a column (the operands of a weight
 * gradient, transposed), or is a tile of 128 x 128 (weights).  The last block of a row, column
 * or tile may be shorter.  The products take the codes as they are: a NaN code, or an Inf
 * or NaN scale, reaches the outputs of its own row and column as IEEE arithmetic dictates.
 *
 * Rows of codes start every `row_stride` bytes, a multiple of 16 and at most 2^22 for
 * the products (2^26 for hadamard_transform_fp8_blocks), from a 16-byte aligned
 * address.  The products read codes in 16-byte pieces: every row of codes must be
 * readable up to the next multiple of 16 bytes; what lies there is ignored.  Rows of
 * scales start every `scales_row_stride` floats.
 *
 * Groups: `ends` is a device array of `groups` int32, the end of each group of rows (or
 * tokens), in order: group g is [ends[g - 1], ends[g]), the first starts at 0, and a
 * group may be empty.  Values outside [0, rows] are taken as the nearest inside; ends that
 * go down give unspecified outputs, but no access out of bounds.  The host does not read
 * them: no call waits for the GPU.
 *
 * Streams, ownership, errors and graph capture are as for the transforms.
 *
 * HADACORE_ERROR_TOO_LARGE: sizes, batches and groups of 2^30 and more (rows of
 * hadamard_transform_fp8_blocks: 2^31); rows times their stride, or matrices times theirs,
 * past 2^42 (2^40 there); for hadacore_quantize_fp8_tiles more than 65535 matrices, or more than
 * 65535 * 128 rows; for the products tiles that take 2^32 work-items or more (at most 512 for
 * each 16 x 16 outputs).
 */

/*
 * hadamard_transform_fp8_blocks -- each row of k values rotated in blocks of n, and
 * quantized with a scale for each 128 of the row.  With y = scale * H_n applied to
 * each n consecutive values (n = 1: the values times `scale`), code row i holds the codes
 * of y[i], and out_scales[i * scales_row_stride + b] the scale of columns 128 b .. 128 b + 127.
 *   in              m rows of k 16-bit values, in_row_stride elements apart (>= k, <= 2^26).
 *                   n >= 128: 16-byte aligned and the stride a multiple of 8; n <= 64: any
 *                   stride, 2-byte aligned
 *   out_codes       m rows of k bytes, out_row_stride (>= k, multiple of 16, <= 2^26) apart
 *   out_scales      m rows of ceil(k / 128) floats
 *   k               a multiple of n, >= 0
 *   n               a power of two in [1, 32768]
 * Rows without gaps take one launch; others one for each n columns if n >= 128.  The
 * three ranges must not overlap.
 */
hadacore_status hadamard_transform_fp8_blocks(const void *in, int64_t in_row_stride,
                                              void *out_codes, int64_t out_row_stride,
                                              float *out_scales, int64_t scales_row_stride,
                                              int64_t m, int64_t k, int64_t n,
                                              hadacore_dtype dtype, float scale, void *stream);

/*
 * hadacore_padded_tokens -- the places that `tokens` tokens in `groups` groups may
 * take when each group is padded to a multiple of 128, whatever the groups:
 * floor((tokens + 127 min(groups, tokens)) / 128) * 128.  0 for negative arguments; the largest
 * multiple of 128 where the places pass int64.
 */
int64_t hadacore_padded_tokens(int64_t tokens, int64_t groups);

/*
 * hadacore_quantize_fp8_columns -- codes of a tall matrix, transposed, with a scale for
 * each 128 rows of a column: the operands of a weight gradient, which sums over rows
 * (tokens).  Each group of rows is padded with zeros to a multiple of 128, and the groups
 * follow each other; out_codes[c][p] is the code of column c at padded place p, and
 * out_scales[c][p / 128] its scale.  Places after the last group, up to
 * hadacore_padded_tokens(m, groups), get zero codes and scales.  Rows after the last end
 * are left out.
 *   in          m rows of k 16-bit values, any stride >= k (<= 2^26), 2-byte aligned
 *   ends        the groups' ends; NULL with groups = 1: one group of all rows; not read
 *               with groups = 0
 *   out_codes   k rows of hadacore_padded_tokens(m, groups) bytes
 *   out_scales  k rows of a 128th of that
 * Ranges must not overlap.  m is at most 2^22 by the stride of the codes.
 */
hadacore_status hadacore_quantize_fp8_columns(const void *in, int64_t in_row_stride,
                                              const int32_t *ends, int64_t groups,
                                              void *out_codes, int64_t out_row_stride,
                                              float *out_scales, int64_t scales_row_stride,
                                              int64_t m, int64_t k, hadacore_dtype dtype,
                                              void *stream);

/*
 * hadacore_quantize_fp8_tiles -- codes of `batch` m x k matrices with a scale for each
 * tile of 128 x 128: weights.  out_codes_t, unless NULL, gets the codes transposed (k
 * rows of m bytes), for the product with the transposed weights; their scales are
 * out_scales transposed.
 *   in                   m rows of k 16-bit values, any stride >= k (<= 2^26), 2-byte aligned
 *   out_scales           ceil(m / 128) rows of ceil(k / 128) floats
 *   *_batch_stride       elements (bytes, floats) from one matrix to the next; not used for
 *                        batch <= 1.  Output matrices must not interleave.
 * Ranges must not overlap.
 */
hadacore_status hadacore_quantize_fp8_tiles(const void *in, int64_t in_row_stride,
                                            int64_t in_batch_stride, void *out_codes,
                                            int64_t out_row_stride, int64_t out_batch_stride,
                                            void *out_codes_t, int64_t out_t_row_stride,
                                            int64_t out_t_batch_stride, float *out_scales,
                                            int64_t scales_row_stride,
                                            int64_t scales_batch_stride, int64_t batch,
                                            int64_t m, int64_t k, hadacore_dtype dtype,
                                            void *stream);

/*
 * hadacore_matmul_fp8 -- out = A B^T for codes A (m x k) and B (n x k):
 *     out[i][j] = sum_b a_scales[i][b] * b_scales[j'][b] * sum_{c in block b} A[i][c] B[j][c],
 * j' = j for b_scale_rows = 1 and j / 128 for b_scale_rows = 128 (weights in tiles).  The two
 * scales are multiplied first, in fp32: their product has to be in its range (one that passes it
 * gives NaN even with zero codes, one below it 0).
 * The products of codes are exact, the blocks are joined in fp32, and the result is
 * rounded once, to nearest even.  The 128 products inside a block
 *   - are added in fp32 for outputs of HADACORE_FP32;
 *   - are added by the FP8 matrix cores for outputs of 16 bits, which keep about 17 bits
 *     below the block's largest product |A[i][c] B[j][c]|: their sum is within 2^-9 of that
 *     product (1.3e-5 of the result, as measured, for N(0, 1) values; more where large
 *     products cancel).
 *   a, b            codes; a_scales m rows of ceil(k / 128) floats, b_scales n (or
 *                   ceil(n / 128)) rows
 *   out             m rows of n values of out_dtype (HADACORE_FP16, _BF16 or _FP32),
 *                   out_row_stride elements apart (>= n, <= 2^26), aligned to its values
 *   k               >= 0; k = 0 gives zeros
 * The output must not overlap the inputs.
 */
hadacore_status hadacore_matmul_fp8(const void *a, int64_t a_row_stride, const float *a_scales,
                                    int64_t a_scales_row_stride, const void *b,
                                    int64_t b_row_stride, const float *b_scales,
                                    int64_t b_scales_row_stride, int32_t b_scale_rows, void *out,
                                    int64_t out_row_stride, hadacore_dtype out_dtype, int64_t m,
                                    int64_t n, int64_t k, void *stream);

/*
 * hadacore_matmul_fp8_grouped -- hadacore_matmul_fp8 with rows of A sorted by group (expert)
 * and a B of its own for each group: out[i] = A[i] B[g]^T for the rows i of group g.  B
 * is `groups` matrices of n x k codes with a scale per tile of 128 x 128,
 * b_batch_stride bytes (a multiple of 16) and b_scales_batch_stride floats apart.  Rows
 * after the last end get zeros.  Sums are hadacore_matmul_fp8's.
 */
hadacore_status hadacore_matmul_fp8_grouped(const void *a, int64_t a_row_stride,
                                            const float *a_scales, int64_t a_scales_row_stride,
                                            const void *b, int64_t b_row_stride,
                                            int64_t b_batch_stride, const float *b_scales,
                                            int64_t b_scales_row_stride,
                                            int64_t b_scales_batch_stride, const int32_t *ends,
                                            int64_t groups, void *out, int64_t out_row_stride,
                                            hadacore_dtype out_dtype, int64_t m, int64_t n,
                                            int64_t k, void *stream);

/*
 * hadacore_weight_gradient_fp8_grouped -- the weight gradients of such a product: for each
 * group g, out[g] (n x k) = sum over the group's tokens t of A[:, t] B[:, t]^T, where A
 * (n rows: output gradients) and B (k rows: inputs) are what
 * hadacore_quantize_fp8_columns gives for the same tokens and `ends`: rows of `places` =
 * hadacore_padded_tokens(tokens, groups) codes, a multiple of 128 (INVALID_SIZE).  A group
 * without tokens gets zeros.  ends = NULL with groups = 1: one group of all tokens.  The
 * outputs are out_batch_stride elements apart.  Sums are hadacore_matmul_fp8's.
 */
hadacore_status hadacore_weight_gradient_fp8_grouped(
    const void *a, int64_t a_row_stride, const float *a_scales, int64_t a_scales_row_stride,
    const void *b, int64_t b_row_stride, const float *b_scales, int64_t b_scales_row_stride,
    const int32_t *ends, int64_t groups, void *out, int64_t out_row_stride,
    int64_t out_batch_stride, hadacore_dtype out_dtype, int64_t places, int64_t n, int64_t k,
    void *stream);

/*
 * Tokens and weights of their own: routing, the exchange by expert, low-rank adapters.
 *
 * A router gives each of m tokens k of its experts.  A slot is a (token, choice) pair, t * k + j.
 * hadacore_group_tokens sorts slots by group (expert, adapter): `ends` as above, `rows` the place of
 * each slot and `slots` the slot of each place.  hadacore_dispatch_rows copies the tokens' rows to
 * their places, where the products by expert take them, and hadacore_combine_rows joins the
 * products' rows by weight.  The adapters take tokens in place, by `ends` and `slots` (k = 1).
 *
 * Values are fp16, bf16 or fp32 (HADACORE_FP32) where a dtype is named; rows start at any
 * value's address, `*_row_stride` elements apart (at least their width, at most 2^26).  Arrays of
 * int32 and fp32 are dense.  All sums are fp32 or wider, joined in an order that the sizes fix, and
 * rounded once: results repeat to the bit.  Wrong ends, rows and slots give unspecified
 * results, but no access out of bounds.  Outputs must not overlap each other or an input unless
 * stated.  Workspaces are scratch: two calls in flight at once need two (a captured graph keeps its
 * own as long as it may run).  Streams, ownership, errors and graph capture are as for the
 * transforms.
 *
 * HADACORE_ERROR_TOO_LARGE: 2^30 slots and more; rows times their stride past 2^42; for the
 * exchange 2^32 work-items (256 for each token of a gradient, and for each 16 KiB copied or 2048
 * values, 1024 of fp32, joined); for the adapters 2^27 tokens, rows of more than 2^22 values, more
 * than HADACORE_MAX_GROUPS adapters, or 2^32 work-items (256 for each 16 to 128 tokens of an adapter
 * by 512 outputs, or 256 from rank 129).
 */
#define HADACORE_MAX_EXPERTS 1024
#define HADACORE_MAX_CHOICES 32
#define HADACORE_MAX_GROUPS 4095
#define HADACORE_MAX_RANK 256

/* Bytes of workspace of hadacore_route (0 for few tokens, and for arguments that it rejects). */
int64_t hadacore_route_workspace_size(int64_t m, int64_t experts);

/*
 * hadacore_route -- the k largest logits of each token, their softmax weights, how many
 * tokens each expert got, and the balance loss.  With p_t the softmax of token t's logits,
 * c_e how often expert e was chosen, and T the tokens that have an expert:
 *     loss = experts * sum_e (c_e / sum c) * (sum_t p_te / T),
 *     out_slopes[e] = d loss / d p_te = experts * c_e / (sum c * T)   (c has no gradient).
 * Equal logits: the lower index first (-0 is 0; NaN is above all).  An expert whose logit is -Inf is
 * never chosen, and a token without enough of others gets -1 and weight 0 there; so does a token
 * whose `valid` is 0, which counts nowhere.  A NaN or +Inf logit makes its token's p NaN.
 * Weights are p of the chosen, divided by their sum if `renormalize`.  Without any
 * choice (m = 0 included) counts, slopes and loss are 0.
 *   logits      m rows of `experts` (1 to HADACORE_MAX_EXPERTS) values
 *   valid       m bytes, or NULL: all are valid
 *   k           1 to HADACORE_MAX_CHOICES and at most `experts` (INVALID_SIZE otherwise)
 *   out_experts, out_weights  m * k values, in falling order of the logits
 *   workspace   hadacore_route_workspace_size(m, experts) bytes, 16-byte aligned
 */
hadacore_status hadacore_route(const void *logits, int64_t logits_row_stride, hadacore_dtype dtype,
                               const uint8_t *valid, int64_t m, int64_t experts, int64_t k,
                               int32_t renormalize, int32_t *out_experts, float *out_weights,
                               int32_t *out_counts, float *out_loss, float *out_slopes,
                               void *workspace, int64_t workspace_bytes, void *stream);

/*
 * hadacore_route_gradient -- the gradient of the logits for those of the weights (m * k, or NULL)
 * and of the loss (one value on the device, or NULL), from what hadacore_route took and gave.
 * Rows of tokens without an expert get zeros.
 */
hadacore_status hadacore_route_gradient(const void *logits, int64_t logits_row_stride,
                                        hadacore_dtype dtype, const int32_t *chosen,
                                        const float *weights, const float *slopes,
                                        const float *dweights, const float *dloss, int64_t m,
                                        int64_t experts, int64_t k, int32_t renormalize, void *out,
                                        int64_t out_row_stride, void *stream);

/* Bytes of workspace of hadacore_group_tokens (0 for few slots, and for arguments it rejects). */
int64_t hadacore_group_workspace_size(int64_t slots, int64_t groups);

/*
 * hadacore_group_tokens -- slots sorted by group, in their own order inside a group.
 *   ids        `slots` int32; one outside [0, groups) is of no group
 *   out_ends   `groups` (at most HADACORE_MAX_GROUPS) values: the end of each group's places
 *   out_rows   `slots` values: the place of each slot, -1 for a slot of no group
 *   out_slots  `slots` values: the slot of each place; behind the last end the slots of no group
 */
hadacore_status hadacore_group_tokens(const int32_t *ids, int64_t slots, int64_t groups,
                                      int32_t *out_ends, int32_t *out_rows, int32_t *out_slots,
                                      void *workspace, int64_t workspace_bytes, void *stream);

/*
 * hadacore_dispatch_rows -- row t of `in` (m rows of `width` values of 1, 2 or 4 bytes, codes and
 * their scales as well) copied to the places rows[t * k + j] of `out` (m * k rows).  Places behind the
 * last end get zeros.  Its gradient is hadacore_combine_rows without weights.  Each place is to be
 * the row of one slot at most (as hadacore_group_tokens gives them).
 */
hadacore_status hadacore_dispatch_rows(const void *in, int64_t in_row_stride, int32_t value_bytes,
                                       const int32_t *rows, const int32_t *ends, int64_t groups,
                                       void *out, int64_t out_row_stride, int64_t m, int64_t k,
                                       int64_t width, void *stream);

/*
 * hadacore_combine_rows -- out[t] = sum_j weights[t * k + j] * in[rows[t * k + j]], `in` of `places`
 * rows.  weights = NULL: the sum.  A row outside [0, places) adds nothing, whatever its weight.
 */
hadacore_status hadacore_combine_rows(const void *in, int64_t in_row_stride, int64_t places,
                                      hadacore_dtype dtype, const int32_t *rows,
                                      const float *weights, void *out, int64_t out_row_stride,
                                      int64_t m, int64_t k, int64_t width, void *stream);

/*
 * hadacore_combine_gradient -- the gradients of such a join of m * k rows y:
 *     dy[rows[t * k + j]] = weights[t * k + j] * dout[t]   (zeros behind the last end),
 *     dweights[t * k + j] = <dout[t], y[rows[t * k + j]]>  (0 for a slot of no group).
 * dy or dweights may be NULL; y is read for dweights only.
 */
hadacore_status hadacore_combine_gradient(const void *dout, int64_t dout_row_stride, const void *y,
                                          int64_t y_row_stride, hadacore_dtype dtype,
                                          const int32_t *rows, const int32_t *ends, int64_t groups,
                                          const float *weights, void *dy, int64_t dy_row_stride,
                                          float *dweights, int64_t m, int64_t k, int64_t width,
                                          void *stream);

/* Bytes of workspace of hadacore_adapters (0 for few tokens, and for arguments that it rejects). */
int64_t hadacore_adapters_workspace_size(int64_t m, int64_t k, int64_t n, int64_t rank,
                                         int64_t groups);

/*
 * hadacore_adapters -- out[t] = y[t] + scales[g] * up[g]^T (down[g] x[t]) for the tokens t of each
 * group g; tokens of no group (behind the last end) get y[t].
 *   x           m rows of k values of `dtype` (HADACORE_FP16 or _BF16)
 *   down, up    `groups` matrices of `rank` (1 to HADACORE_MAX_RANK) rows of k, of n values of
 *               `dtype`: both rank-major; batch strides in elements, not used for one group.
 *               Adapters of different ranks: zero rows behind the smaller one's
 *   scales      one fp32 for each group, or NULL: 1
 *   ends        the groups' ends among the places; NULL with groups = 1: all rows, with 0: none
 *   slots       the token of each place (hadacore_group_tokens with k = 1), each token once; NULL:
 *               the tokens themselves are sorted
 *   y, out      m rows of n values of out_dtype (`dtype` or HADACORE_FP32); y may be out (in place),
 *               or NULL: zeros
 *   hidden      NULL, or m rows of fp32 (16-byte aligned, a stride of a multiple of 4 and at least
 *               rank rounded up to 16): down[g] x[t] by place, zeros up to that width; places behind
 *               the last end are left as they were.  The gradient of the weights takes it
 * The gradients of x are the same call on dout with `down` and `up` exchanged and y = NULL; dout, as x, is
 * of `dtype`, also where the output was of 32 bits.
 * Between the products h is fp32, and the second takes all of its 24 bits (for fp16 above 2^-35 of
 * the row's largest).  Inf may give NaN.
 */
hadacore_status hadacore_adapters(const void *x, int64_t x_row_stride, const void *down,
                                  int64_t down_row_stride, int64_t down_batch_stride,
                                  const void *up, int64_t up_row_stride, int64_t up_batch_stride,
                                  const float *scales, const int32_t *ends, const int32_t *slots,
                                  int64_t groups, const void *y, int64_t y_row_stride, void *out,
                                  int64_t out_row_stride, hadacore_dtype dtype,
                                  hadacore_dtype out_dtype, float *hidden,
                                  int64_t hidden_row_stride, int64_t m, int64_t k, int64_t n,
                                  int64_t rank, void *workspace, int64_t workspace_bytes,
                                  void *stream);

/* Bytes of workspace of hadacore_adapter_gradient (0 where it needs none, or rejects). */
int64_t hadacore_adapter_gradient_workspace_size(int64_t m, int64_t width, int64_t rank,
                                                 int64_t groups);

/*
 * hadacore_adapter_gradient -- out[g] (rank x width) = scales[g] * sum over the places p of g of
 * hidden[p] x[token of p]^T: the gradient of `up` from hidden and dout, and that of `down` from the
 * hidden of the gradient's call (dout, roles exchanged) and x.  A group without tokens gets
 * zeros.  All 24 bits of hidden are taken (for fp16 above 2^-35 of the rank's largest value in the
 * group), and a rank's values show in its own row only, Inf and NaN too.  out_dtype is `dtype` or
 * HADACORE_FP32; other arguments as for hadacore_adapters.
 */
hadacore_status hadacore_adapter_gradient(const float *hidden, int64_t hidden_row_stride,
                                          const void *x, int64_t x_row_stride,
                                          hadacore_dtype dtype, const float *scales,
                                          const int32_t *ends, const int32_t *slots,
                                          int64_t groups, void *out, int64_t out_row_stride,
                                          int64_t out_batch_stride, hadacore_dtype out_dtype,
                                          int64_t m, int64_t width, int64_t rank,
                                          void *workspace, int64_t workspace_bytes, void *stream);

/*
 * hadacore_stream_copy -- copies `bytes` bytes from device pointer `src` to
 * device pointer `dst` with 16-byte vector loads and stores on `stream`.  Both
 * pointers 16-byte aligned, bytes a multiple of 16, ranges disjoint.  It moves
 * the same HBM bytes per element as the transform and serves as its measured
 * bandwidth ceiling (the paper's Appendix B compares against a device copy).
 */
hadacore_status hadacore_stream_copy(const void *src, void *dst, int64_t bytes, void *stream);

/* Static, human-readable name of a status code (never NULL). */
const char *hadacore_status_string(hadacore_status status);

/* HADACORE_VERSION of the loaded library. */
int32_t hadacore_version(void);

#ifdef __cplusplus
}
#endif

#endif /* HADACORE_H */
