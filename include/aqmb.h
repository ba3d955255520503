/*
 * aqmb - multi-bitwidth additive-codebook linear layers on AMD Instinct MI355X (gfx950).
 *
 * A quantized linear layer stores a weight matrix W (d_out rows, d_in columns) as
 *   - M code planes: plane m holds, for every output row i and input group j
 *     (g consecutive weights of row i), the index b_{ijm} of a codeword of codebook m;
 *   - M codebooks C_0..C_{M-1}, each 2^B codewords of g fp16 values;
 *   - one fp16 scale s_i per output row.
 * At precision level k (1 <= k <= M) the layer uses only the first k codebooks:
 *   W_k[i, j*g + t] = s_i * sum_{m<k} C_m[b_{ijm}][t]
 * (Drop-by-Drop, section 5: partial reconstruction from the first k codebooks;
 * section 3.2: groups are consecutive along d_in and concatenated; the per-row
 * scale is the "Scales: d_out*16" term of the size estimate in appendix C).
 * One stored set of codes serves every k; planes m >= k are never read.
 *
 * Conventions for every entry point:
 *   - Data pointers passed to aqmb_create/gemv/gemm/dequant are DEVICE pointers on
 *     the current HIP device. Row-major, densely packed, 16-byte aligned
 *     (x, y, X, Y, W, codes, codebooks and scales).
 *   - `stream` is a hipStream_t (0 = the null stream). gemv/gemm/dequant only
 *     enqueue work on it and return; results are valid once the stream is synced.
 *   - Arguments are validated on the host before anything is enqueued. On any
 *     error nothing is launched and no output byte is written; the status says
 *     why and aqmb_last_error() gives a message for the calling thread.
 *   - No exception or abort crosses this interface.
 *   - A layer is read-only after creation (it is the stored format (C, b, s) that
 *     Alg. 1 returns): every compute call reads the layer and writes only the
 *     caller's outputs, so calls on one layer may run concurrently on different
 *     streams. Only aqmb_load_planes, aqmb_drop_planes and aqmb_destroy change a
 *     layer, and they must not overlap other calls on it.
 *   - Device scratch memory that a kernel needs for partial results (the lookup-
 *     table GEMV, the prefix distortion) is taken per call from the device's
 *     stream-ordered pool (hipMallocAsync / hipFreeAsync on `stream`), so two
 *     calls never share it. Every other call needs no scratch. Kernel choice does
 *     not depend on environment variables: aqmb_gemv_select and aqmb_gemm_select
 *     choose a kernel explicitly.
 */
#ifndef AQMB_H
#define AQMB_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct aqmb_layer_s* aqmb_layer_t;
typedef void* aqmb_stream_t; /* a hipStream_t */

typedef enum {
  AQMB_OK = 0,
  AQMB_EINVAL = 1,        /* bad argument: null pointer, k outside [1, M], sizes that do not fit */
  AQMB_EUNSUPPORTED = 2,  /* valid in the method but not implemented: g != 8, B not 8 or 16, batch > 16, dtype */
  AQMB_ENOMEM = 3,        /* device allocation failed */
  AQMB_EHIP = 4           /* a HIP runtime call or kernel launch failed; see aqmb_last_error() */
} aqmb_status;

/* AQMB_F8: OCP e4m3 (largest value 448, no infinities); AQMB_I8: signed 8-bit integers. Both are taken
 * only by the operators between the layers (aqmb_rms_norm and below), always with scales. */
typedef enum { AQMB_F16 = 0, AQMB_BF16 = 1, AQMB_F32 = 2, AQMB_F8 = 3, AQMB_I8 = 4 } aqmb_dtype;

typedef struct {
  int32_t d_out;          /* output rows of W, >= 1 */
  int32_t d_in;           /* input columns of W, >= g, a multiple of g */
  int32_t group_size;     /* g: weights per group; 8 is supported */
  int32_t num_codebooks;  /* M: 1..8 */
  int32_t code_bits;      /* B: 4 (16 codewords), 8 (uint8 codes, 256 codewords) or 16 (uint16 codes, 65536 codewords) */
} aqmb_desc;

/* Largest batch accepted by aqmb_gemv. */
#define AQMB_MAX_BATCH 16

/*
 * Create a layer from device buffers (Alg. 1 stores a layer as AQLMFormat(C, b, s)).
 *   codes     [M][d_out][d_in/g] uint8 (B = 8), uint16 (B = 16), or uint8 holding values 0..15
 *             (B = 4; stored two per byte): plane-major.
 *   codebooks [M][2^B][g] fp16 bit patterns; codeword c of codebook m is g contiguous values.
 *   scales    [d_out] fp16 bit patterns.
 * The library copies everything into device memory it owns, re-tiling the codes
 * inside each plane for coalesced reads while keeping planes outermost, so that
 * level k reads only the first k planes. Synchronous: returns after the copy on
 * `stream` has finished; the caller may free its buffers afterwards.
 * Code values >= 2^B cannot occur for B = 8 or 16 (they fill their type); for B = 4 they are
 * refused (EINVAL).
 * Errors: EINVAL (null pointer, bad sizes, 4-bit codes above 15), EUNSUPPORTED (g, B or M not supported),
 * ENOMEM, EHIP. On error *out is set to NULL.
 */
aqmb_status aqmb_create(aqmb_layer_t* out, const aqmb_desc* desc, const void* codes,
                        const uint16_t* codebooks, const uint16_t* scales, aqmb_stream_t stream);

/*
 * Run-time loading of code planes (the dynamic loading the paper's discussion of future work
 * names as an application of droppable codebooks: a device keeps only the planes its precision
 * level needs). Planes are stored outermost, so level k needs exactly planes 0..k-1.
 *   aqmb_create_prefix  like aqmb_create with only the first `resident` planes in device memory
 *                       (1 <= resident <= M); codes is [resident][d_out][d_in/g], codebooks and
 *                       scales are complete ([M][2^B][g], [d_out]).
 *   aqmb_load_planes    append the next n_planes planes (codes [n_planes][d_out][d_in/g], plane
 *                       `resident` first); the layer's code memory is reallocated.
 *   aqmb_drop_planes    keep planes 0..keep-1 (1 <= keep <= resident) and free the others.
 *   aqmb_resident_planes  the number of resident planes.
 * Every compute call with k above the resident count returns EINVAL; aqmb_prefix_distortion
 * covers the resident levels. load and drop are synchronous, wait for the device before the old
 * code memory is freed, and must not run concurrently with other calls on the same layer.
 * Errors: EINVAL (bad handle, null pointer, plane counts out of range, 4-bit codes above 15),
 * ENOMEM, EHIP. On error the layer is unchanged.
 */
aqmb_status aqmb_create_prefix(aqmb_layer_t* out, const aqmb_desc* desc, int resident, const void* codes,
                               const uint16_t* codebooks, const uint16_t* scales, aqmb_stream_t stream);
aqmb_status aqmb_load_planes(aqmb_layer_t layer, int n_planes, const void* codes, aqmb_stream_t stream);
aqmb_status aqmb_drop_planes(aqmb_layer_t layer, int keep);
aqmb_status aqmb_resident_planes(aqmb_layer_t layer, int* resident);

/* Free a layer and its device memory (waits for the device first). NULL is a no-op.
 * (The counterpart of aqmb_create: the stored format (C, b, s) of Alg. 1 is released.)
 * EINVAL for a handle that is not a live layer. */
aqmb_status aqmb_destroy(aqmb_layer_t layer);

/* Copy the layer's descriptor into *out. EINVAL for a bad handle or a null out. */
aqmb_status aqmb_get_desc(aqmb_layer_t layer, aqmb_desc* out);

/*
 * Decode GEMV: y[b][i] = sum_t x[b][t] * W_k[i][t] for b < batch (section 5 reconstruction,
 * applied as a product without forming W_k).
 *   x  [batch][d_in],  dtype x_dtype in {F16, BF16}
 *   y  [batch][d_out], dtype y_dtype in {F16, BF16, F32}
 * Products and sums are carried in fp32; the result is rounded once to y_dtype
 * (round to nearest even). 1 <= batch <= AQMB_MAX_BATCH.
 * Errors: EINVAL (bad handle, null pointer, k outside [1, M], batch < 1),
 * EUNSUPPORTED (batch > AQMB_MAX_BATCH, dtype), EHIP.
 */
aqmb_status aqmb_gemv(aqmb_layer_t layer, int k, const void* x, aqmb_dtype x_dtype, int batch,
                      void* y, aqmb_dtype y_dtype, aqmb_stream_t stream);

/*
 * The GEMV kernels. Each computes the quantity aqmb_gemv defines, to the same contract (fp32
 * products and sums, one rounding to y_dtype); they differ in speed only.
 *   AQMB_GEMV_AUTO    the library's choice for the layer, k, batch and x dtype (what aqmb_gemv runs)
 *   AQMB_GEMV_DIRECT  the direct-gather kernel of the layer's code width: codewords gathered per
 *                     code and dotted with x on the vector ALUs, 16 rows per workgroup. 8-bit
 *                     codes: k <= 4 and rows of at most 2048 groups (16384 inputs); 4- and 16-bit
 *                     codes: every k and row
 *   AQMB_GEMV_MMA     the matrix-core kernel (8- and 4-bit codes; every k, batch and row length)
 *   AQMB_GEMV_LUT     per-group lookup tables LUT_m[j][c] = <x_j, C_m[c]> in LDS, one read per
 *                     code (8-bit codes); its split-K partial sums take per-call scratch from the
 *                     stream-ordered pool (ENOMEM if that fails)
 * DIRECT with 8-bit codes also refuses when its codebook replicas and x tile do not fit in LDS
 * for the row length and batch (batch above 2 on rows of several thousand inputs).
 */
typedef enum {
  AQMB_GEMV_AUTO = 0,
  AQMB_GEMV_DIRECT = 1,
  AQMB_GEMV_MMA = 2,
  AQMB_GEMV_LUT = 3
} aqmb_gemv_kernel;

/*
 * aqmb_gemv with the kernel named by `kernel` (section 5 reconstruction, as aqmb_gemv). For
 * tests and tuning: every kernel can be checked against the same reference whatever the default
 * choice is. Arguments as aqmb_gemv.
 * Errors: those of aqmb_gemv; EUNSUPPORTED when the kernel cannot serve this layer, k, batch
 * or row length (see aqmb_gemv_kernel); EINVAL for an unknown kernel; ENOMEM (LUT scratch).
 */
aqmb_status aqmb_gemv_select(aqmb_layer_t layer, int k, const void* x, aqmb_dtype x_dtype, int batch,
                             void* y, aqmb_dtype y_dtype, aqmb_gemv_kernel kernel, aqmb_stream_t stream);

/* Most layers accepted by one aqmb_gemv_multi call. */
#define AQMB_MAX_MULTI 16

/*
 * Decode GEMV of several layers that read the same input (fused projections such as q/k/v or
 * gate/up): for each l < n_layers, ys[l][b][i] = sum_t x[b][t] * W_k^(l)[i][t], exactly what
 * aqmb_gemv(layers[l], k, x, x_dtype, batch, ys[l], y_dtype, stream) computes (same arithmetic,
 * same rounding), in one launch when either
 *   - every layer has 8-bit codes, k <= 4, aqmb_gemv would use the direct-gather kernel (batch 1;
 *     on rows of more than 512 groups only bf16 x at k < 3) and, for rows of more than 512
 *     groups, k = 1, or
 *   - n_layers >= 2, every layer would take the matrix-core kernel (batch >= 2, and batch 1 on
 *     rows of more than 512 groups: see aqmb_gemv's kernel choice in the library source) and all
 *     have the same code width (layers on both sides of the device's compute-unit count, in 16-row
 *     blocks, only where aqmb_gemv treats bf16 x alike in both);
 * otherwise the layers are launched one after another. In one launch the row blocks of all layers
 * are shared out evenly over the compute units.
 *   layers  n_layers live handles, all with the same d_in and on the same device
 *   x       [batch][d_in], dtype x_dtype in {F16, BF16}
 *   ys      n_layers device pointers, ys[l] is [batch][d_out of layer l], dtype y_dtype
 * 1 <= n_layers <= AQMB_MAX_MULTI; k must be valid for every layer. Nothing is launched when
 * validation fails.
 * Errors: EINVAL (null pointer, bad handle, n_layers < 1, d_in or device differ, k outside
 * [1, M] of some layer, batch < 1), EUNSUPPORTED (n_layers > AQMB_MAX_MULTI, batch >
 * AQMB_MAX_BATCH, dtype), EHIP.
 */
aqmb_status aqmb_gemv_multi(const aqmb_layer_t* layers, int n_layers, int k, const void* x, aqmb_dtype x_dtype,
                            int batch, void* const* ys, aqmb_dtype y_dtype, aqmb_stream_t stream);

/*
 * Prefill GEMM (the section 5 partial reconstruction applied to n_tokens inputs at once, the
 * product Y = W X of section 2.2 in row-major form): Y[n][i] = s_i * sum_t X[n][t] * Wb_k[i][t]
 * for n < n_tokens, where Wb_k is the
 * unscaled reconstruction sum_{m<k} C_m[b_{ijm}] formed as a binary32 left fold over m and
 * rounded to nearest-even bf16 (the operand fed to bf16 matrix cores); accumulation is fp32.
 *   X  [n_tokens][d_in]  bf16 (no other activation dtype: convert before the call)
 *   Y  [n_tokens][d_out] dtype y_dtype in {BF16, F32}
 * Requires B = 8 or B = 4. Errors: EINVAL (bad handle, null pointer, k outside [1, M],
 * n_tokens < 1), EUNSUPPORTED (B = 16, dtype), EHIP.
 */
aqmb_status aqmb_gemm(aqmb_layer_t layer, int k, const void* X, int n_tokens, void* Y,
                      aqmb_dtype y_dtype, aqmb_stream_t stream);

/*
 * The prefill GEMM's tilings (the same arithmetic and rounding; they differ in speed only).
 *   AQMB_GEMM_AUTO     the library's choice (what aqmb_gemm runs): from 17 tokens and up to k = 4 a
 *                      kernel that splits the inputs over a workgroup's waves, where it is estimated
 *                      faster; else 16-row tiles up to 144 tokens, else the large tile that needs
 *                      the fewest rounds of workgroups
 *   AQMB_GEMM_ROWS16   16 weight rows per workgroup, all tokens in tiles of 16 (made for few tokens)
 *   AQMB_GEMM_256x128, AQMB_GEMM_128x128, AQMB_GEMM_128x64
 *                      tokens x weight rows per workgroup of the large-tile kernel
 */
typedef enum {
  AQMB_GEMM_AUTO = 0,
  AQMB_GEMM_ROWS16 = 1,
  AQMB_GEMM_256x128 = 2,
  AQMB_GEMM_128x128 = 3,
  AQMB_GEMM_128x64 = 4
} aqmb_gemm_tiling;

/* aqmb_gemm with the tiling named by `tiling` (tests and tuning). Errors: those of aqmb_gemm;
 * EINVAL for an unknown tiling. */
aqmb_status aqmb_gemm_select(aqmb_layer_t layer, int k, const void* X, int n_tokens, void* Y,
                             aqmb_dtype y_dtype, aqmb_gemm_tiling tiling, aqmb_stream_t stream);

/*
 * The prefill GEMM of aqmb_gemm (section 5 partial reconstruction, same definition, arguments and
 * errors) with a caller-owned device workspace. Where aqmb_gemm_workspace_bytes reports a
 * non-zero size and `workspace_bytes` is at least that size, the call runs in two passes: the
 * unscaled bf16 weights Wb_k (the same binary32 fold and rounding) are written once into the
 * workspace, tiled in matrix-core operand order, and a dense kernel multiplies X by them. The
 * output is bit-identical to aqmb_gemm's for the same arguments. Otherwise (workspace null or too
 * small, or the size is 0) the call is exactly aqmb_gemm.
 *   workspace        device memory, 256-byte aligned, owned by the caller; the call writes it
 *                    (stream-ordered on `stream`), so calls that share a workspace must be ordered
 *   workspace_bytes  its size in bytes
 * Errors: those of aqmb_gemm; EINVAL for a workspace that is not 256-byte aligned.
 */
aqmb_status aqmb_gemm_ws(aqmb_layer_t layer, int k, const void* X, int n_tokens, void* Y,
                         aqmb_dtype y_dtype, void* workspace, size_t workspace_bytes,
                         aqmb_stream_t stream);

/*
 * *bytes = the workspace aqmb_gemm_ws needs to run the two-pass GEMM for (k, n_tokens) on this
 * layer (2 bytes per weight, rows rounded up to 32 and d_in to 64), or 0 where that path does not
 * apply: it is taken with 4- or 8-bit codes when the one-pass choice is the 256 x 128 tiling and
 * that tiling fills every compute unit, at k >= 3 always and at k <= 2 for problems of several rounds
 * of 256 x 256 tiles. Errors: EINVAL (bad handle, null bytes, k outside [1, M], n_tokens < 1).
 */
aqmb_status aqmb_gemm_workspace_bytes(aqmb_layer_t layer, int k, int n_tokens, size_t* bytes);

/*
 * Dequantize (the section 5 partial reconstruction W_k written out as a dense matrix):
 * W[i][t] = W_k[i][t] in w_dtype in {F16, BF16, F32}, bit-exact to this evaluation
 * order: each fp16 codebook entry is taken exactly to binary32; the entries of planes
 * 0..k-1 are summed as a binary32 left fold (C_0 + C_1, then + C_2, ...), each sum rounded
 * to nearest even; the fold is multiplied by s_i in binary32 (one rounding, no fused
 * multiply-add); the product is rounded to nearest even into w_dtype. Subnormals are kept.
 *   W  [d_out][d_in]
 * Errors: EINVAL (bad handle, null pointer, k outside [1, M]), EUNSUPPORTED (dtype), EHIP.
 */
aqmb_status aqmb_dequant(aqmb_layer_t layer, int k, void* W, aqmb_dtype w_dtype, aqmb_stream_t stream);

/*
 * Distortion of every precision level in one pass (section 5: the error of each partial
 * reconstruction, which the training loop of Alg. 1 drives down level by level; the weighted
 * MSE of section 2.2, Eq. wmse-task): for k = 1..M,
 *   D[k-1] = ||(W - W_k) X||_F^2 / (d_out * n)
 * with the calibration inputs given as the rows of Xt = X^T.
 *   W   [d_out][d_in] fp16: the weights being quantized (w_dtype must be F16)
 *   Xt  [n][d_in]     fp16: one calibration input per row (x_dtype must be F16)
 *   D   one double per resident level (M unless planes were dropped or never loaded), device memory
 * The products W X and C_m[b_m] X run on fp16 matrix cores (each product of two fp16 values
 * exact, sums in fp32), the per-output differences W X - s_i sum_{m<k} (C_m[b_m] X) in fp32, the
 * sums of their squares in fp64, added in a fixed order: the result is reproducible.
 * The Hessian form of the same quantity, tr[(W - W_k) H (W - W_k)^T] / d_out with H = X X^T / n,
 * is obtained by passing any factor F with F F^T = H (e.g. a Cholesky factor) as Xt = F^T,
 * n = d_in, and multiplying D by d_in.
 * Requires B = 8 or B = 4. The per-workgroup sums (at most 256 x 8 doubles) take per-call scratch
 * from the stream-ordered pool, freed on `stream` after the final sum.
 * Errors: EINVAL (bad handle, null pointer, n < 1, misaligned pointer), EUNSUPPORTED (B = 16,
 * dtype other than F16, n > 2^30), ENOMEM (scratch), EHIP.
 */
aqmb_status aqmb_prefix_distortion(aqmb_layer_t layer, const void* W, aqmb_dtype w_dtype, const void* Xt,
                                   aqmb_dtype x_dtype, int n, double* D, aqmb_stream_t stream);

/*
 * aqmb_prefix_distortion without any device allocation, for callers that cannot allocate (code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc). Same arguments,
 * kernels, arithmetic and result as aqmb_prefix_distortion. Its per-workgroup sums live in a
 * fixed array of the library, 16 KiB per device (256 workgroups x 8 levels of doubles; the need is
 * the same for every layer and n), held until the process ends; the call allocates and frees
 * nothing. Every call on one device shares that device's array, so calls that overlap on one
 * device (different streams, or other threads) race and give wrong results: order them.
 * Errors: those of aqmb_prefix_distortion except ENOMEM; EUNSUPPORTED if the kernels ever need
 * more scratch than the array holds.
 */
aqmb_status aqmb_prefix_distortion_noalloc(aqmb_layer_t layer, const void* W, aqmb_dtype w_dtype, const void* Xt,
                                           aqmb_dtype x_dtype, int n, double* D, aqmb_stream_t stream);

/* Widest beam accepted by aqmb_beam_search. */
#define AQMB_MAX_BEAM 16

/*
 * Code search (Appendix C, code optimisation: a beam search over combinations of codewords that
 * minimise the quantization error; Algorithm 1 updates the assignments b this way): for every
 * group (row i, group j) of a dense weight matrix, beam search over codebooks 0..k-1 for the
 * codes c_0..c_{k-1} that minimise the group's squared error ||w_ij - s_i sum_m C_m[c_m]||^2.
 * Stage m extends each kept partial tuple by every codeword of codebook m and keeps the `beam`
 * best; the last stage keeps the best one (beam 1 is greedy residual coding). Groups are
 * independent (the plain squared error of the weights, X = I in the weighted MSE of §2.2).
 * Every comparison is decided in binary32 in this order: S_m[c][t] = s_i * C_m[c][t] (exact for
 * fp16 operands); the residual of a kept tuple is w - S_0[c_0] - ... with each subtraction
 * rounded; a candidate's d_t = fl(r_t - S_m[c][t]) and e = d_0 d_0 + d_1 d_1 + ... + d_7 d_7
 * with every product and every sum rounded, left to right, no fused multiply-add; candidates are
 * ordered by e, equal e by the code tuple (lexicographically).
 *   desc       the layer shape: d_out, d_in, g = 8, M codebooks, B = 8 or 4
 *   W          [d_out][d_in] fp16 (device, 16-byte aligned): the weights to encode
 *   codebooks  [M][2^B][8] fp16 (device, 16-byte aligned); codebooks 0..k-1 are used
 *   scales     [d_out] fp16 (device)
 *   codes      [k][d_out][d_in/8] uint8 (device, output; values < 2^B): plane-major, the layout
 *              aqmb_create takes
 *   errors     [d_out][d_in/8] float (device, output; may be NULL): e of the chosen tuple
 * 1 <= k <= M, 1 <= beam <= AQMB_MAX_BEAM. Work: 2^B (1 + (k - 1) beam) candidates per group.
 * Errors: EINVAL (null pointer, misaligned W or codebooks, k outside [1, M], beam < 1),
 * EUNSUPPORTED (B = 16, beam > AQMB_MAX_BEAM), EHIP.
 */
aqmb_status aqmb_beam_search(const aqmb_desc* desc, int k, int beam, const void* W, const uint16_t* codebooks,
                             const uint16_t* scales, uint8_t* codes, float* errors, aqmb_stream_t stream);

/*
 * The same code search with the data-aware objective of §2.2 (Eq. wmse-task: the weighted MSE
 * (1/n) ||(W - W_hat) X||_F^2 over calibration inputs X, which App. C's code optimisation
 * minimises): the error of group (i, j) is d^T H_j d with d = w_ij - s_i sum_m C_m[c_m] and H_j
 * the 8 x 8 diagonal block of H = X X^T / n for inputs 8 j .. 8 j + 7 (terms coupling different
 * groups are left out, so groups stay independent; with every H_j = I this is aqmb_beam_search's
 * objective). Every comparison is decided in binary32 in this order, with r the kept tuple's
 * residual (as in aqmb_beam_search) and C the unscaled candidate codeword:
 *   b_t = sum_u H_tu r_u and A = sum_t r_t b_t per kept tuple; Q = sum_t C_t (sum_u H_tu C_u) per
 *   codeword; T = sum_t C_t b_t and e = (A - (2 s_i) T) + (s_i s_i) Q per candidate,
 * every product and sum rounded, sums left to right over t, u = 0..7, no fused multiply-add;
 * candidates ordered by e, equal e by the code tuple.
 *   H       [d_in/8][8][8] fp32 (device, 4-byte aligned): the symmetric blocks H_j, row-major
 *   others  as for aqmb_beam_search; errors receive e of the chosen tuple
 * Work: 2^B (1 + (k - 1) beam) candidates per group, one workgroup per group j and 256 rows.
 * Errors: those of aqmb_beam_search; EINVAL also for a NULL or misaligned H.
 */
aqmb_status aqmb_beam_search_weighted(const aqmb_desc* desc, int k, int beam, const void* W,
                                      const uint16_t* codebooks, const uint16_t* scales, const float* H,
                                      uint8_t* codes, float* errors, aqmb_stream_t stream);

/*
 * Average storage bits per weight at level k (appendix C, Eq. avg_bits): codebooks
 * 16*g*k*2^B bits, codes d_out*(d_in/g)*B bits per used plane, scales 16*d_out bits,
 * over d_out*d_in weights. The printed codes term lacks the per-plane factor; the
 * worked example there (about 2.002 bits for d_in=8192, d_out=28672, g=8, M=2, B=8)
 * needs it. Returns a negative value for a null or invalid descriptor or k outside [1, M].
 */
double aqmb_bits_per_weight(const aqmb_desc* desc, int k);

/*
 * ---------------------------------------------------------------------------------------------
 * The operators between the layers of a decode step: the norm that feeds a projection, the product
 * with plain 4-bit weights (for the layers of a model that are not additively coded), attention of
 * one new token over a paged key-value cache, the cache's upkeep, and what requests bring and get
 * back (rotary positions, low-rank adapters, log probabilities). The conventions above hold,
 * except that data pointers need only the alignment of their elements and rows may be strided
 * (strides in elements, the last dimension dense). Sums, softmax statistics and scales are held in
 * binary32. Nothing here allocates device memory except aqmb_w4_create.
 */

/*
 * Root-mean-square norm of each row with the residual's addition:
 *   h = x + residual (binary32; h = x without a residual), residual_out = h rounded to `dtype`,
 *   v_t = h_t * (1 / sqrt(mean(h^2) + eps)) * (weight_t + weight_offset)
 * and y = v rounded once (nearest even) for y_dtype F16, BF16 or F32; or, for y_dtype F8 or I8, per
 * group of `scale_group` columns (0: the whole row; the last group of a row may be shorter):
 *   a = max(max |v|, 2^-100), y = round(v * (L / a)) to nearest even, scale = a / L,
 *   L = 448 for F8, 127 for I8, both quotients rounded to binary32
 * so that y * scale stands for v. A group that holds a value that is not finite gets the scale NaN
 * and y = 0. h is not rounded before it is squared or scaled; a row whose squares overflow binary32
 * gives zeros, as the formula does.
 *   x        [rows][cols], `dtype` in {F16, BF16}, row stride x_stride
 *   residual, residual_out  [rows][cols] `dtype`, row stride residual_stride: both or neither given
 *   weight   [cols] `dtype`
 *   y        [rows][cols] y_dtype, row stride y_stride
 *   scales   [rows][ceil(cols / scale_group)] fp32, dense; NULL unless y_dtype is F8 or I8
 * y may be x and residual_out may be residual or x (same strides); no other overlap.
 * 1 <= cols <= AQMB_MAX_NORM_COLS; scale_group 0, 32, 64 or 128.
 * Errors: EINVAL (null or misaligned pointer, rows or cols < 1, a stride below cols, one residual
 * pointer without the other, scales missing or not wanted, negative or NaN eps), EUNSUPPORTED
 * (dtype, cols above the limit, scale_group, rows * max(8, ceil(cols / 8)) of 2^31 or more, with rows rounded up to
 * a multiple of 16 where cols <= 64), EHIP.
 */
#define AQMB_MAX_NORM_COLS 32768
aqmb_status aqmb_rms_norm(const void* x, aqmb_dtype dtype, int64_t x_stride, const void* residual,
                          void* residual_out, int64_t residual_stride, const void* weight, float weight_offset,
                          float eps, int rows, int cols, void* y, aqmb_dtype y_dtype, int64_t y_stride,
                          float* scales, int scale_group, aqmb_stream_t stream);

/*
 * Layers of 4-bit integers with a scale (and, optionally, a zero point) for every group of
 * group_size consecutive weights of a row:
 *   W[i][t] = scales[i][t / group_size] * (q[i][t] - zeros[i][t / group_size])
 *   weights  [d_out][ceil(d_in / 2)] uint8: q[i][t] is the low nibble of byte t / 2 for even t, the
 *            high nibble for odd t (an odd row's last high nibble is ignored)
 *   scales   [d_out][ceil(d_in / group_size)] fp16 bit patterns
 *   zeros    the same shape, uint8; NULL: 8 everywhere (symmetric quantization)
 * d_in need not be a multiple of the group size. The library copies everything into device memory
 * it owns, re-tiled for the matrix cores; aqmb_w4_create is synchronous (the caller may free its
 * buffers afterwards). A layer is read-only after creation.
 * Errors: EINVAL (null pointer, sizes < 1 or > 2^30, d_out * d_in >= 2^32, 2^24 tiles of 16 x 128 weights or
 * more, the last ones counted whole), EUNSUPPORTED (group_size other than 32, 64, 128), ENOMEM, EHIP; on error
 * *out is NULL. aqmb_w4_destroy waits for the device; NULL is a no-op, EINVAL for a handle that is not a live layer.
 */
typedef struct aqmb_w4_s* aqmb_w4_t;
typedef struct {
  int32_t d_out;
  int32_t d_in;
  int32_t group_size;     /* 32, 64 or 128 */
} aqmb_w4_desc;
aqmb_status aqmb_w4_create(aqmb_w4_t* out, const aqmb_w4_desc* desc, const uint8_t* weights,
                           const uint16_t* scales, const uint8_t* zeros, aqmb_stream_t stream);
aqmb_status aqmb_w4_destroy(aqmb_w4_t layer);
aqmb_status aqmb_w4_get_desc(aqmb_w4_t layer, aqmb_w4_desc* out);

/*
 * Decode product with such a layer, y[b][i] = sum_t X[b][t] W[i][t] for b < batch, where
 * X = x for x_dtype F16 or BF16, and X[b][t] = x[b][t] * x_scales[b][t / x_scale_group] for F8 and
 * I8 (what aqmb_rms_norm writes; x_scale_group 0: one scale for each row). Within a group the
 * products q * x and the sum of x (for the zero point) are formed on the matrix cores: exact
 * products, sums in binary32 (I8: exact in int32); the groups are scaled and added in binary32, in
 * a fixed order; one rounding to y_dtype in {F16, BF16, F32}. The weights enter as 16 + q (I8: as q); the 16 and the
 * zero point come off a group's sums before its scale. These sums cannot overflow while every |X| <= 2^112; above
 * (BF16 x, or 8-bit x with such scales) outputs may be NaN where the formula is finite. An X that is not finite
 * makes all of its row's outputs not finite.
 *   x  [batch][d_in], row stride x_stride; y [batch][d_out], row stride y_stride
 * 1 <= batch <= AQMB_MAX_BATCH.
 * Errors: EINVAL (bad handle, null or misaligned pointer, batch < 1, a stride below the row,
 * x_scales missing or not wanted, layer on another device), EUNSUPPORTED (batch > AQMB_MAX_BATCH,
 * dtype, x_scale_group other than 0 and the layer's group size), EHIP.
 */
aqmb_status aqmb_w4_gemv(aqmb_w4_t layer, const void* x, aqmb_dtype x_dtype, int64_t x_stride,
                         const float* x_scales, int x_scale_group, int batch, void* y, aqmb_dtype y_dtype,
                         int64_t y_stride, aqmb_stream_t stream);

/*
 * A paged key-value cache of one attention layer: n_pages pages of page_size token slots. The
 * caller owns the memory; this struct only describes it.
 *   k, v     page p starts at element p * page_stride; inside a page, dense,
 *            AQMB_KV_HEAD_MAJOR [n_kv_heads][page_size][head_dim] or
 *            AQMB_KV_SLOT_MAJOR [page_size][n_kv_heads][head_dim]
 *   dtype    F16, BF16, or F8 with one scale for every token and head:
 *   k_scale, v_scale  fp32, dense, [n_pages][n_kv_heads][page_size] or
 *            [n_pages][page_size][n_kv_heads] as the layout; NULL unless dtype is F8
 * head_dim: a multiple of 8 up to 256; page_size 1..32768; page_stride >= n_kv_heads * page_size *
 * head_dim and a multiple of 8; k and v 16-byte aligned (8-byte for F8).
 */
typedef enum { AQMB_KV_HEAD_MAJOR = 0, AQMB_KV_SLOT_MAJOR = 1 } aqmb_kv_layout;
typedef struct {
  void* k;
  void* v;
  float* k_scale;
  float* v_scale;
  int64_t page_stride;
  int32_t dtype;          /* aqmb_dtype */
  int32_t layout;         /* aqmb_kv_layout */
  int32_t n_pages;
  int32_t page_size;
  int32_t n_kv_heads;
  int32_t head_dim;
} aqmb_kv_cache;

/*
 * Attention of one new token per sequence over the cache: for every sequence s and head h,
 *   score_t = scale * <q[s][h], K_t>, out[s][h] = sum_t softmax(score)_t V_t, over the positions
 *   t < lengths[s], and t >= lengths[s] - window where window > 0
 * with K_t, V_t of head h / (n_heads / n_kv_heads) in slot t % page_size of page
 * page_table[s][t / page_size]. A sequence with no position gives out = 0 and lse = -infinity.
 * lse (may be NULL): the logarithm of the softmax's denominator, log sum_t exp(score_t), fp32
 * [n_seqs][n_heads], with which results over disjoint parts of a context can be joined. A score that is NaN
 * or +infinity makes out and lse of its head NaN; one of -infinity weighs nothing (a head that has no other is as
 * one without a position).
 *   q, out      [n_seqs][n_heads][head_dim] F16 or BF16 (`dtype`; the cache's own type, or any of
 *               the two with an F8 cache), stride between sequences q_stride / out_stride, each a
 *               multiple of 8; 16-byte aligned
 *   page_table  int32, row s at s * table_stride, of ceil(max_length / page_size) entries; those that
 *               no position < lengths[s] needs may hold anything. A page outside [0, n_pages) is
 *               skipped: its positions do not exist.
 *   lengths     int32 [n_seqs], device memory; values outside [0, max_length] are clamped
 *   max_length  an upper bound of the lengths, <= table_stride * page_size and <= 2^27: fixes, with window, n_seqs
 *               and the cache's shape, how a sequence's work is split and in which order it is summed. A
 *               sequence's result does not depend, to the bit, on the lengths and contents of the others; under
 *               another bound or beside another number of sequences its last digits may differ
 * Slots that hold no token may hold anything (NaN included). Scores and softmax are binary32; the
 * probabilities enter the matrix cores as two 16-bit parts (22 bits with an F16 cache, 16 with a BF16 or F8 one).
 * One rounding to `dtype`.
 * workspace: aqmb_paged_attention_workspace_bytes bytes of device memory, 16-byte aligned, written
 * by the call (calls that share one must be ordered); 0 bytes: NULL is fine.
 * Errors: EINVAL (null or misaligned pointer, sizes < 1, n_heads not a multiple of n_kv_heads,
 * max_length < 0 or above the table, negative window, workspace too small, scales missing or not
 * wanted), EUNSUPPORTED (dtype, head_dim, page_size), EHIP.
 */
aqmb_status aqmb_paged_attention(const aqmb_kv_cache* cache, const void* q, aqmb_dtype dtype, int64_t q_stride,
                                 int n_heads, const int32_t* page_table, int64_t table_stride,
                                 const int32_t* lengths, int n_seqs, int max_length, float scale, int window,
                                 void* out, int64_t out_stride, float* lse, void* workspace,
                                 size_t workspace_bytes, aqmb_stream_t stream);
aqmb_status aqmb_paged_attention_workspace_bytes(const aqmb_kv_cache* cache, int n_heads, int n_seqs,
                                                 int max_length, int window, size_t* bytes);

/*
 * Write new tokens into the cache: token i's keys and values go to slot slots[i] % page_size of page
 * slots[i] / page_size. A slot outside [0, n_pages * page_size) (such as -1 for padding) is skipped;
 * slots of one call must differ. For an F8 cache each token and head is scaled as aqmb_rms_norm
 * scales a group (L = 448, its a the largest magnitude of the head's values).
 *   k, v   [n_tokens][n_kv_heads][head_dim] F16 or BF16 (`dtype`; the cache's own type, or any of
 *          the two for an F8 cache), stride between tokens k_stride / v_stride
 *   slots  int64 [n_tokens], device memory
 * Errors: EINVAL (null or misaligned pointer, n_tokens < 1, stride below a token), EUNSUPPORTED (dtype,
 * n_tokens * n_kv_heads above 2^26 - 4), EHIP.
 */
aqmb_status aqmb_kv_append(const aqmb_kv_cache* cache, const void* k, int64_t k_stride, const void* v,
                           int64_t v_stride, aqmb_dtype dtype, const int64_t* slots, int n_tokens,
                           aqmb_stream_t stream);

/*
 * Copy page src[i] to page dst[i], keys, values and scales, in every cache of `caches` (the layers of
 * a model; all of the same shape and type), in one launch. A pair with a page outside [0, n_pages) is
 * skipped. No page may be a dst twice, nor a dst of one pair and the src of another.
 *   src, dst  int32 [n_pairs], device memory
 * 1 <= n_caches <= AQMB_MAX_CACHES.
 * Errors: EINVAL (null pointer, n_caches or n_pairs < 1, caches that differ), EUNSUPPORTED
 * (n_caches above the limit), EHIP.
 */
#define AQMB_MAX_CACHES 64
aqmb_status aqmb_kv_copy_pages(const aqmb_kv_cache* caches, int n_caches, const int32_t* src, const int32_t* dst,
                               int n_pairs, aqmb_stream_t stream);

/*
 * Bookkeeping of the pages on the host: which pages each sequence holds, with reference counts.
 * No call touches the GPU; calls on one pool must not overlap. Sequences are small integers
 * 0..max_seqs-1, given out lowest first.
 *   aqmb_pages_add      a new, empty sequence. ENOMEM when max_seqs are live.
 *   aqmb_pages_fork     a new sequence that shares all pages of `seq`, the last, partly filled one
 *                       included. ENOMEM as above. The tokens of `seq` have to be written (or their writing
 *                       enqueued) before: what the new one copies on its first write is the page as it is then.
 *   aqmb_pages_extend   n_tokens more tokens: slots[n_tokens] receives their cache slots (the
 *                       argument of aqmb_kv_append). Where the first of them falls into a page that
 *                       another sequence shares, the sequence gets a page of its own and
 *                       (*copy_src, *copy_dst) say which page to copy before writing, else both
 *                       are -1. ENOMEM, with nothing changed, when too few pages are free.
 *                       The copy has to be enqueued before the next fork, free or compact on this pool (after
 *                       an ENOMEM too: the pairs that came before it stand), since a freed page is given out
 *                       again at once. The pairs of extends with nothing of the kind between them never
 *                       conflict: one call may copy them all.
 *   aqmb_pages_free     ends a sequence; pages that no other one shares become free.
 *   aqmb_pages_compact  moves used pages from the end of the pool into free ones at its start, so
 *                       that the used pages are 0..used-1: the *n_pairs copies to make are written
 *                       to src / dst (room for n_pages / 2 each), and every sequence's table is
 *                       changed already. The copies do not overlap (the argument of
 *                       aqmb_kv_copy_pages); make them before the next append.
 *   aqmb_pages_table    the sequence's length and pages: *n_used = ceil(length / page_size) entries
 *                       go to table (room for `capacity` >= that many; EINVAL otherwise, with *length and
 *                       *n_used set). table may be NULL with capacity 0 to ask for the sizes only.
 *   aqmb_pages_counts   pages free, and sequences live. Either pointer may be NULL.
 * Free pages are given out lowest first. Errors otherwise: EINVAL (bad handle, null pointer, a
 * sequence that is not live, n_tokens < 0, sizes < 1), ENOMEM (host memory).
 */
typedef struct aqmb_pages_s* aqmb_pages_t;
aqmb_status aqmb_pages_create(aqmb_pages_t* out, int n_pages, int page_size, int max_seqs);
aqmb_status aqmb_pages_destroy(aqmb_pages_t pool);
aqmb_status aqmb_pages_add(aqmb_pages_t pool, int* seq);
aqmb_status aqmb_pages_fork(aqmb_pages_t pool, int seq, int* child);
aqmb_status aqmb_pages_extend(aqmb_pages_t pool, int seq, int n_tokens, int64_t* slots, int32_t* copy_src,
                              int32_t* copy_dst);
aqmb_status aqmb_pages_free(aqmb_pages_t pool, int seq);
aqmb_status aqmb_pages_compact(aqmb_pages_t pool, int32_t* src, int32_t* dst, int* n_pairs);
aqmb_status aqmb_pages_table(aqmb_pages_t pool, int seq, int32_t* table, int capacity, int* n_used, int* length);
aqmb_status aqmb_pages_counts(aqmb_pages_t pool, int* n_free, int* n_live);

/*
 * Rotary positions. Of every head the first rotary_dim values form rotary_dim / 2 pairs (a, b), turned by the
 * angle position * frequencies[i] of pair i:
 *   a' = amplitude * (a cos - b sin), b' = amplitude * (b cos + a sin), inverse: by the angle's negative (what the
 *   gradient of the turned values is turned by)
 *   AQMB_ROTARY_HALF         pair i is values i and i + rotary_dim / 2
 *   AQMB_ROTARY_INTERLEAVED  pair i is values 2 i and 2 i + 1
 * The other values of a head stay as they are.
 *   frequencies  fp64 [rotary_dim / 2], radians per position, device memory, 8-byte aligned
 *                (aqmb_rotary_frequencies gives the usual ones)
 *   rotary_dim   even, 2..head_dim
 */
typedef enum { AQMB_ROTARY_HALF = 0, AQMB_ROTARY_INTERLEAVED = 1 } aqmb_rotary_layout;
typedef struct {
  const double* frequencies;
  int32_t rotary_dim;
  int32_t layout;         /* aqmb_rotary_layout */
  float amplitude;
  int32_t inverse;        /* 0 or 1 */
} aqmb_rotary_desc;

/*
 * Frequencies f_i = base^(-2 i / rotary_dim), i < rotary_dim / 2, in HOST memory, and the amplitude that goes with
 * them, scaled for a context `factor` times the original one:
 *   AQMB_ROTARY_PLAIN    as they are (scaling NULL is the same); amplitude 1
 *   AQMB_ROTARY_LINEAR   f_i / factor; amplitude 1
 *   AQMB_ROTARY_BASE     of the base base * factor^(rotary_dim / (rotary_dim - 2)): the first stays, the last is
 *                        divided by factor (rotary_dim 2: as plain); amplitude 1
 *   AQMB_ROTARY_RAMP     between f_i / factor and f_i by the pair's index: with d(n) = rotary_dim / 2 *
 *                        log(original_length / (2 pi n)) / log(base) the index that turns n times over the original
 *                        length, lo = max(floor(d(high)), 0), hi = min(ceil(d(low)), rotary_dim - 1), t = clamp((i - lo) /
 *                        max(hi - lo, 0.001), 0, 1), the frequency is f_i (1 - t) + f_i / factor t; amplitude
 *                        0.1 log(factor) + 1
 *   AQMB_ROTARY_TURNS    between them by the turns n_i = original_length f_i / (2 pi) themselves: t = clamp((n_i -
 *                        low) / (high - low), 0, 1), the frequency is f_i / factor (1 - t) + f_i t; amplitude 1
 * All in binary64. Either output may be NULL.
 * Errors: EINVAL (rotary_dim odd or < 2, base not finite or <= 1, factor not finite or < 1, original_length < 1, low
 * or high not finite, low <= 0 or high <= low where they are used), EUNSUPPORTED (unknown kind).
 */
typedef enum { AQMB_ROTARY_PLAIN = 0, AQMB_ROTARY_LINEAR = 1, AQMB_ROTARY_BASE = 2, AQMB_ROTARY_RAMP = 3,
               AQMB_ROTARY_TURNS = 4 } aqmb_rotary_kind;
typedef struct {
  int32_t kind;           /* aqmb_rotary_kind */
  int32_t original_length;/* RAMP and TURNS only, as the next two */
  double factor;
  double low, high;       /* turns over the original length (RAMP: 1 and 32 are usual; TURNS: 1 and 4) */
} aqmb_rotary_scaling;
aqmb_status aqmb_rotary_frequencies(int rotary_dim, double base, const aqmb_rotary_scaling* scaling,
                                    double* frequencies, float* amplitude);

/*
 * Turns the queries and keys of n_tokens tokens. An angle is the binary64 product of the position (as a binary64
 * number) and the frequency, reduced by whole turns before it is rounded further: sine and cosine are within 2^-22 of that
 * angle's, up to 2^75 radians. They and the turn are binary32, with one rounding to `dtype`.
 *   q, q_out   [n_tokens][n_heads][head_dim] F16 or BF16 (`dtype`), stride between tokens q_stride / q_out_stride
 *   k, k_out   the same with n_kv_heads; both NULL (n_kv_heads 0): no keys
 *   positions  int64 [n_tokens], device memory, of any size and sign
 * q_out may be q and k_out may be k (same stride); no other overlap. head_dim: a multiple of 8 up to 256.
 * Errors: EINVAL (null or misaligned pointer, sizes < 1, a stride below a token, rotary_dim odd or outside
 * [2, head_dim], amplitude not finite, unknown layout or inverse), EUNSUPPORTED (dtype, head_dim, n_heads or n_kv_heads above
 * 65535, n_tokens * (n_heads + n_kv_heads rounded up to a multiple of 8) of 2^27 or more), EHIP.
 */
aqmb_status aqmb_rotary(const aqmb_rotary_desc* rotary, const void* q, int64_t q_stride, void* q_out,
                        int64_t q_out_stride, int n_heads, const void* k, int64_t k_stride, void* k_out,
                        int64_t k_out_stride, int n_kv_heads, aqmb_dtype dtype, int head_dim, const int64_t* positions,
                        int n_tokens, aqmb_stream_t stream);

/*
 * The same with the keys written into a cache at once, and the values beside them: q_out = q turned, and what
 * aqmb_kv_append does with the turned keys and v, in one launch. With a 16-bit cache the results are those of the two
 * calls to the bit; with an F8 cache the keys are scaled from their binary32 values, with one rounding less.
 *   k, v   [n_tokens][cache's n_kv_heads][cache's head_dim] `dtype` as aqmb_kv_append, strides k_stride, v_stride
 *   slots  int64 [n_tokens] as aqmb_kv_append; q_out is written for every token, also where the slot is skipped
 * Errors: those of aqmb_rotary and aqmb_kv_append, with n_heads + 2 n_kv_heads in the limit of the former.
 */
aqmb_status aqmb_rotary_append(const aqmb_kv_cache* cache, const aqmb_rotary_desc* rotary, const void* q,
                               int64_t q_stride, void* q_out, int64_t q_out_stride, int n_heads, const void* k,
                               int64_t k_stride, const void* v, int64_t v_stride, aqmb_dtype dtype,
                               const int64_t* positions, const int64_t* slots, int n_tokens, aqmb_stream_t stream);

/*
 * Low-rank adapters of many requests beside one projection: the caller's stacks of n_adapters pairs of matrices.
 *   a       [n_adapters][rank][d_in] F16 or BF16 (`dtype`), dense
 *   b       [n_adapters][d_out][rank] `dtype`, dense
 *   scales  fp32 [n_adapters]; NULL: 1 everywhere
 *   ranks   int32 [n_adapters]: how many rows of an adapter's a and columns of its b are its own (clamped to
 *           [0, rank]); what lies behind them is not used and may hold anything. NULL: rank everywhere
 * All in device memory, read when a call runs: an adapter may be exchanged between calls.
 * 1 <= rank <= AQMB_MAX_RANK, 1 <= n_adapters <= AQMB_MAX_ADAPTERS; d_in and d_out of any size up to 2^23.
 */
#define AQMB_MAX_RANK 256
#define AQMB_MAX_ADAPTERS 8192
typedef struct {
  const void* a;
  const void* b;
  const float* scales;
  const int32_t* ranks;
  int32_t dtype;          /* aqmb_dtype */
  int32_t n_adapters;
  int32_t rank;
  int32_t d_in;
  int32_t d_out;
} aqmb_adapters;

/*
 * out[i] = base[i] + scales[n] * B_n (A_n x[i]) with n = index[i]; out[i] = base[i] where index[i] is outside
 * [0, n_adapters) (-1: a request without an adapter). Products are exact and summed in binary32 on the matrix cores;
 * A_n x times the scale enters the second product as two (F16, 22 bits of the row's largest) or three (BF16, 24 bits)
 * 16-bit parts; one rounding to y_dtype. A row whose A_n x holds a value that is not finite, or
 * with BF16 one that times the scale is above 3.38e38, where 16 bits end, gives values that are not finite.
 *   x      [n_rows][d_in] of the adapters' dtype, row stride x_stride
 *   index  int32 [n_rows], device memory, in any order
 *   base   [n_rows][d_out] y_dtype in {F16, BF16, F32}, row stride base_stride; what aqmb_gemv or aqmb_w4_gemv gave
 *   out    the same type, row stride out_stride
 * Where x or a starts at an odd element, the two bytes before it, in the same aligned four, are read too (and not used).
 * out may be base (same stride; then rows without an adapter are not touched); no other overlap. A row's sums do not depend on the
 * other rows' contents, only on their number.
 * workspace: aqmb_adapters_workspace_bytes bytes of device memory, 16-byte aligned, written by the call (calls that
 * share one must be ordered); 0 bytes: NULL is fine.
 * Errors: EINVAL (null or misaligned pointer, sizes < 1, a stride below a row, out in place with another stride,
 * workspace too small), EUNSUPPORTED (dtype, rank, n_adapters, d_in, d_out, n_rows above 2^22 - 64,
 * (min(n_rows, n_adapters + 1) + n_rows / 64) * ceil(d_out / 256) of 2^24 or more), EHIP.
 */
aqmb_status aqmb_adapters_add(const aqmb_adapters* adapters, const void* x, int64_t x_stride, const int32_t* index,
                              int n_rows, const void* base, int64_t base_stride, void* out, int64_t out_stride,
                              aqmb_dtype y_dtype, void* workspace, size_t workspace_bytes, aqmb_stream_t stream);
aqmb_status aqmb_adapters_workspace_bytes(const aqmb_adapters* adapters, int n_rows, size_t* bytes);

/*
 * Of every row of logits, with z = scale * logits: the log probabilities z_t - log sum exp z of given tokens, the
 * logarithm of the sum, the entropy - sum p log p, and the largest values with their log probabilities, in
 * descending order (equal ones: the lower token first; -0 equals 0).
 *   logits        [rows][vocab] F16, BF16 or F32 (`dtype`), row stride `stride`
 *   targets       int64 [rows][n_targets], dense; a negative one (padding) gets 0, one >= vocab NaN
 *   logprobs      fp32 [rows][n_targets]; targets and logprobs both NULL with n_targets 0
 *   lse, entropy  fp32 [rows], or NULL
 *   top_ids, top_logprobs  int64 and fp32 [rows][n_top]; n_top 0: both NULL, else either may be NULL
 * A value of -infinity has probability 0 (log probability -infinity) and may be among the top ones where fewer others
 * are there; n_top <= vocab. A row of nothing but -infinity: lse and log probabilities -infinity, entropy 0. A row with a NaN
 * or +infinity: everything NaN, top_ids -1. Sums are binary32, relative to the largest value. A row's results do not depend on the others' contents.
 * workspace: aqmb_log_probs_workspace_bytes bytes of device memory, 16-byte aligned, written by the call (calls that
 * share one must be ordered); 0 bytes: NULL is fine.
 * Errors: EINVAL (null or misaligned pointer, sizes < 1, n_targets < 0, n_top < 0 or > vocab, stride below vocab, scale NaN, below
 * 2^-120 or above 2.35e38 (the largest binary32 number times log 2), outputs without inputs, no output at all, workspace too small), EUNSUPPORTED (dtype, n_top > AQMB_MAX_TOP, rows above 2^22), EHIP.
 */
#define AQMB_MAX_TOP 64
aqmb_status aqmb_log_probs(const void* logits, aqmb_dtype dtype, int64_t stride, int rows, int vocab, float scale,
                           const int64_t* targets, int n_targets, float* logprobs, float* lse, float* entropy,
                           int64_t* top_ids, float* top_logprobs, int n_top, void* workspace, size_t workspace_bytes,
                           aqmb_stream_t stream);
aqmb_status aqmb_log_probs_workspace_bytes(aqmb_dtype dtype, int rows, int vocab, int n_top, size_t* bytes);

/* Static description of a status code. Never NULL. */
const char* aqmb_strerror(aqmb_status status);

/* Message describing the last error on the calling thread ("" if none). Never NULL. */
const char* aqmb_last_error(void);

/* Validate arguments exactly as the entry points do, without touching the GPU.
 * op: 0 = gemv, 1 = gemm, 2 = dequant, 3 = prefix distortion, 4 = beam search. For gemv `n` is
 * the batch, for gemm the token count, for the distortion the number of inputs, for the beam
 * search the beam width (in = W, out = codes, dtypes ignored), ignored for dequant;
 * `in_dtype` is x's dtype (gemv) or Xt's (distortion), `out_dtype` the output dtype or, for
 * the distortion, W's dtype; `in`/`out` are x/y, X/Y, -/W, or Xt/D. `k` is not checked for
 * the distortion. Returns the status the entry point would return before launching anything
 * (the distortion's W pointer is checked by the entry point itself). */
aqmb_status aqmb_validate(const aqmb_desc* desc, int op, int k, int n, aqmb_dtype in_dtype,
                          aqmb_dtype out_dtype, const void* in, const void* out);

#ifdef __cplusplus
}
#endif

#endif /* AQMB_H */
