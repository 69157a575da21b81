/*
 * slim.h - C ABI of libslim: the SLiM compressed linear layer on AMD Instinct MI355X (gfx950).
 *
 * The layer (thesis "Compression Trinity", SLiM chapter, section "Quantized sparse plus
 * low-rank approximation of LLMs"; SLoPe chapter, eq. sparse_plus_low_rank) is
 *
 *     Y = X * Wc^T + (X * L) * R,      Wc = dequant(Q(M (.) W))
 *
 * where M keeps two of every four consecutive weights along the reduction dimension K,
 * Q is symmetric AbsMax 4-bit quantisation per group of 128 weights of a row, and L*R is
 * a rank-r adapter kept as a parallel dense path. SLoPe's double-pruned input gradient
 * (SLoPe chapter, "Double-pruned Backward Pass", eq. sparse_backward_input) is
 *
 *     dX = dY * W^{R,C} + (dY * R^T) * L^T,
 *
 * where W^{R,C} is Wc pruned 2:4 a second time along N, so that the backward contraction is
 * sparse along its own reduction dimension too.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * Shapes: W is [N x K] (N output features, K input features), X is [M x K], Y is [M x N],
 * L is [K x r], R is [r x N], dY is [M x N], dX is [M x K]. Activations, outputs and the
 * adapter factors as given are dense row-major with no padding between rows; the packed
 * weights and the forward's adapter factors use the layouts below.
 *
 * Pointers: every array argument is a DEVICE pointer unless the comment says "host". The
 * caller allocates and owns every buffer, including workspace. The library never frees
 * anything and never keeps a pointer after a call returns.
 *
 * Alignment: device arrays must be 16-byte aligned.
 *
 * Streams: `stream` is a hipStream_t cast to void* (NULL = the null stream). Work is
 * enqueued on it; slim_linear and slim_linear_bwd_dx return without synchronising, and a
 * kernel fault shows up at the caller's next synchronisation of that stream.
 *
 * Errors: every entry point returns an slim_status. Argument checks run on the host before
 * anything is enqueued; when a check fails nothing is launched and the outputs are not
 * touched. No C++ exception crosses the ABI.
 *
 * Packed format (all multi-byte words little-endian)
 * --------------------------------------------------
 * Words. Per row and 16 consecutive reduction positions (four aligned 2:4 groups, g = 0..3):
 *   one code word (uint32): nibble g = u of group g's lower kept position, nibble g + 4 = u of
 *     its higher kept position, where u = q + 8 and q in [-7, 7] is the signed code;
 *   one index half-word (uint16): nibble g = i0 | i1 << 2, the kept offsets i0 < i1 (0..3).
 * Per row and 128 consecutive reduction positions (one quantisation group): one fp16 scale
 *   s16 = fp16_RNE(fp32(max |w| of the group) / 7).
 * The value of kept weight (n, k) is (u - 8) * s16[n, k / 128]; every other weight is zero.
 *
 * Layout. Rows are kept in blocks of 16 and the reduction in chunks of 128 (nch = reduction
 * length / 128). Row n, chunk c owns slot ((n / 16) * nch + c) * 16 + n % 16, which holds its 8
 * code words at bytes 32 slot .. 32 slot + 31 of `codes`, its 8 index half-words at bytes
 * 16 slot .. 16 slot + 15 of `meta` and its scale at element `slot` of `scales`:
 *   codes  uint8 [rows/16][nch][16][32], meta uint8 [rows/16][nch][16][16], scales fp16 [rows/16][nch][16].
 * One chunk of a 16-row block is thus contiguous (512 B of codes, 256 B of index words, 32 B of
 * scales). The forward pack has rows n and reduction k; the backward pack (codesT, metaT) has
 * rows k and reduction n, and its scales are scalesT fp16 [K/128][N] = s16[n, k/128].
 * 3.125 bits per dense weight (0.390625 bytes).
 *
 * Precision
 * ---------
 * Products accumulate in fp32 and Y / dX are fp32. Operands reach the matrix cores in fp16:
 *   - dequantised forward weights (u - 8) * s16, rounded to fp16 once;
 *   - activations (X, dY): each row of activations is multiplied by a power of two 2^e chosen
 *     so that its largest magnitude lies in [16, 32), rounded to fp16, and the fp32 results are
 *     multiplied by 2^-e (both exact), so bf16 inputs of any magnitude keep fp16's relative
 *     precision. At M <= 32 the exponent is chosen per slice of the reduction that one block
 *     or wave stages (at most 1024 positions); at M > 32 per whole row;
 *   - backward: the scale s16[n, k/128] multiplies the (row-scaled) gradient, and the product is
 *     rounded to fp16 once; the codes enter as exact small integers;
 *   - adapter: the first product (X L, or dY R^T) accumulates in fp32. At M <= 32 it stays fp32
 *     and is row-scaled into fp16 for the second product per pass of at most 512 ranks; at
 *     M > 32 it is formed from the row-scaled activations and stored in fp16, so its entries
 *     must stay below 65504 after that scaling: |T[m, j]| < 2^11 max_k |X[m, k]| (true when
 *     sum_k |L[k, j]| < 2^11).
 * Deterministic: identical inputs (and at M > 32 a workspace that holds the same kernels, see
 * slim_linear_workspace) give identical bits.
 */
#ifndef SLIM_H
#define SLIM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SLIM_ABI_VERSION 2

typedef enum {
  SLIM_OK = 0,
  SLIM_EINVAL = 1,        /* a required pointer is NULL, or an argument is out of range */
  SLIM_ESHAPE = 2,        /* a size breaks a divisibility or range rule */
  SLIM_EDTYPE = 3,        /* unsupported dtype code */
  SLIM_EALIGN = 4,        /* a device array is not 16-byte aligned */
  SLIM_ENONFINITE = 5,    /* W holds a NaN or an infinity */
  SLIM_EWORKSPACE = 6,    /* workspace missing or too small for the call's kernels */
  SLIM_EDEVICE = 7,       /* a HIP runtime call or a kernel launch failed */
  SLIM_EUNSUPPORTED = 8,  /* valid but not supported by this library (e.g. no gfx950 device) */
  SLIM_ERANGE = 9         /* a group scale the packed format or the backward cannot represent */
} slim_status;

/* Element types. Activations (X, dY) are SLIM_F16 or SLIM_BF16; Y and dX are always SLIM_F32. */
typedef enum { SLIM_F16 = 0, SLIM_BF16 = 1, SLIM_F32 = 2 } slim_dtype;

/* Values kept in 8 bits (see "The 8-bit path" below), where an entry point names it among its types. */
typedef enum { SLIM_Q8_E4M3 = 3 } slim_dtype_q8;

/* Activations: x; max(x, 0); x Phi(x) (Phi the normal distribution); x (1 + tanh(sqrt(2/pi) (x + 0.044715 x^3))) / 2;
 * x / (1 + exp(-x)). */
typedef enum {
  SLIM_ACT_NONE = 0,
  SLIM_ACT_RELU = 1,
  SLIM_ACT_GELU = 2,
  SLIM_ACT_GELU_TANH = 3,
  SLIM_ACT_SILU = 4
} slim_act;

/* Human-readable name of a status code (static string, never NULL). */
const char* slim_status_string(int status);

/* SLIM_ABI_VERSION of the built library. */
int slim_abi_version(void);

/*
 * slim_pack - one-time forward pack of a dense fp32 weight.
 * Thesis: 2:4 magnitude pruning along the reduction dimension (SLoPe "Double-pruned Backward
 * Pass"; background "Sparse Tensor Core Acceleration"); symmetric AbsMax quantisation
 * (SLiM preliminaries, eq. symmetric_quantization) with groups of 128 (SLiM setup).
 *
 *   W       fp32 [N, K], device.
 *   N, K    N >= 16 and N % 16 == 0; K >= 128 and K % 128 == 0.
 *   codes   out, uint8 [N/16][K/128][16][32]; meta out, uint8 [N/16][K/128][16][16];
 *   scales  out, uint16 [N/16][K/128][16]. The packed layout keeps rows in blocks of 16 and K in
 *           chunks of 128: row n, chunk c (positions 128c .. 128c+127) owns slot
 *           ((n/16) * (K/128) + c) * 16 + n%16, holding 8 code words (uint32, little-endian;
 *           word i covers positions 16i .. 16i+15 of the chunk: the kept codes, as q + 8, of
 *           its four 2:4 groups, the first kept of group g in nibble g, the second in nibble
 *           g+4), 8 index
 *           half-words (uint16; nibble g = i0 | i1 << 2, the kept positions of group g) and one
 *           fp16 scale (the chunk is one quantisation group). The blocks keep one chunk of 16
 *           rows contiguous (512 B of codes, 256 B of indices, 32 B of scales).
 *   mask    out, optional (NULL to skip): uint8 [N, K], 1 where the weight is kept.
 * Mask rule: in each aligned group of four along K, keep the two largest |w|; on equal
 * magnitude the lower position wins (-0 and +0 are equal). Codes: q = clamp(rint(w / s16), -7, 7)
 * with the division done in double precision and ties rounded to even; q = 0 when s16 == 0.
 * Returns SLIM_ENONFINITE if W holds a NaN/Inf and SLIM_ERANGE if a scale overflows fp16; the
 * outputs are then unspecified. This call synchronises `stream` (it reads back a status word)
 * and allocates 4 bytes of device memory for that word for the duration of the call.
 */
int slim_pack(const float* W, int64_t N, int64_t K, uint8_t* codes, uint8_t* meta,
              uint16_t* scales, uint8_t* mask, void* stream);

/*
 * slim_pack_bwd - one-time backward pack: prune the packed forward weight a second time,
 * 2:4 along N, for the transposed contraction of the input gradient.
 * Thesis: SLoPe "Double-pruned Backward Pass" (W^{R,C}, eq. sparse_backward_input; Lemma
 * sparsity_ratio gives the extra zeros, 9.375% for 2:4).
 *
 *   codes, meta, scales   a forward pack of an [N, K] weight (from slim_pack), device.
 *   N, K                  N >= 128 and N % 128 == 0; K % 128 == 0.
 *   codesT  out, uint8 [K/16][N/128][16][32]; metaT out, uint8 [K/16][N/128][16][16]: the packed
 *           layout of slim_pack with rows k and reduction n (W^{R,C} transposed, pruned 2:4
 *           along n). scalesT out, uint16 [K/128, N]: s16[n, k/128] by 128-group of k.
 *   mask_rc out, optional (NULL to skip): uint8 [N, K], 1 on the support of W^{R,C}.
 * Rule: for each column k and aligned group of four rows, keep two slots ranked by
 * (|Wc| descending, forward-kept descending, row ascending). A kept slot carries its forward
 * code (8, i.e. zero, if the forward mask had dropped it).
 * Returns SLIM_ERANGE if a forward scale is 2048 or more (a group max |w| of about 14336): the
 * M > 32 backward forms dY * s16 in fp16 from row-scaled gradients below 32, which would overflow.
 * The outputs are then unspecified. This call synchronises `stream` (it reads back a status word)
 * and allocates 4 bytes of device memory for that word for the duration of the call.
 */
int slim_pack_bwd(const uint8_t* codes, const uint8_t* meta, const uint16_t* scales, int64_t N,
                  int64_t K, uint8_t* codesT, uint8_t* metaT, uint16_t* scalesT, uint8_t* mask_rc,
                  void* stream);

/*
 * slim_pack_adapter - one-time layout of the adapter factors for slim_linear.
 * Thesis: the rank-r adapter W ~ W^C + L R (SLiM "SLiM-LoRA low-rank adapters"); like the weight
 * pack (set up once, multiply many times), this runs once per layer. The forward reads L along
 * K for each rank (X L) and R along the rank for each output row (T R), so it takes L^T
 * row-major and R^T in tiles of 32 rows x 16 ranks; re-laying them inside every slim_linear call
 * would add a launch and 4 r (K + N) bytes of traffic per call. The backward
 * (slim_linear_bwd_dx) reads L and R as given.
 *
 *   L    fp16 [K, r], device.     R    fp16 [r, N], device.
 *   K, N >= 1; r >= 16, r % 16 == 0.
 *   Lt   out, fp16 [r, K] = L^T, row-major.
 *   Rt   out, fp16 R^T in 32 x 16 tiles: ceil(N/32) * 32 * r elements, element (n, j) of R^T at
 *        ((n / 32) * (r / 16) + j / 16) * 512 + (n % 32) * 16 + j % 16; rows n >= N of the last
 *        tile are zero. One tile is 1 KiB of contiguous memory, the unit the kernels load.
 * Asynchronous on `stream`; a pure data movement (bit-exact).
 */
int slim_pack_adapter(const uint16_t* L, const uint16_t* R, int64_t K, int64_t N, int64_t r, uint16_t* Lt,
                      uint16_t* Rt, void* stream);

/*
 * slim_pack_adapter_q - one-time 4-bit pack of the adapter factors for slim_linear_qa.
 * Thesis: SLiM "Low-rank adapter quantization" (SLiM-LoRA^Q): AbsMax group quantization of the
 * adapters with groups of 128 elements, which cuts their bytes about 4x. The groups run along each
 * factor's input dimension: L^T [r, K] by rows j along K (the reduction of X L) and R^T [N, r] by
 * rows n along r (the reduction of T R); a row's last group holds r % 128 elements when 128 does
 * not divide r. Scale and codes follow the weights' rules: s16 = fp16_RNE(fp32(max |a|) / 7),
 * q = clamp(rint(a / s16), -7, 7) (double-precision division, ties to even; 0 when s16 == 0).
 *
 *   L    fp16 [K, r], device.     R    fp16 [r, N], device.
 *   K % 128 == 0, N >= 1, r >= 32 and r % 32 == 0.
 *   Lq   out, uint8 [r, K/2]: row j holds the codes u = q + 8 of L[:, j], 8 consecutive elements
 *        per little-endian 32-bit word, element 2c in nibble c and element 2c + 1 in nibble c + 4.
 *   Ls   out, fp16 bits [r, ceil(K/128)].
 *   Rq   out, uint8 [N, r/2]: row n holds the codes of R[:, n], same word format.
 *   Rs   out, fp16 bits [N, ceil(r/128)].
 * Bytes: r (K + N) / 2 codes plus 2 (r ceil(K/128) + N ceil(r/128)) scales (4.125 bits per element
 * when 128 divides both). Returns SLIM_ENONFINITE if L or R holds a NaN/Inf. Synchronises `stream`
 * (status read back) and allocates 4 bytes of device memory for the duration of the call.
 */
int slim_pack_adapter_q(const uint16_t* L, const uint16_t* R, int64_t K, int64_t N, int64_t r, uint8_t* Lq,
                        uint16_t* Ls, uint8_t* Rq, uint16_t* Rs, void* stream);

/*
 * slim_linear_workspace - bytes of device workspace with which slim_linear runs its fastest kernels for
 * these sizes (written to *bytes, host pointer). Depends only on the sizes. Pure host function.
 * The figure does not always grow with M: a workspace for calls of several M should have the largest of
 * their figures. At M > 32 a smaller one may still hold the kernels that take the least (512-row tiles);
 * the call then runs those, slower for some hundred rows and with its sums in another order, and returns
 * SLIM_EWORKSPACE only if they do not fit either.
 */
int slim_linear_workspace(int64_t M, int64_t N, int64_t K, int64_t r, size_t* bytes);

/*
 * slim_bwd_dx_workspace - the same for slim_linear_bwd_dx. Pure host function.
 */
int slim_bwd_dx_workspace(int64_t M, int64_t N, int64_t K, int64_t r, size_t* bytes);

/*
 * slim_workspace_init - zero a workspace before its first use (its leading control words must
 * start at zero; every successful call leaves them at zero again). Asynchronous on `stream`.
 */
int slim_workspace_init(void* ws, size_t ws_bytes, void* stream);

/*
 * slim_linear - Y = X * Wc^T + (X * L) * R, fp32 accumulation, fp32 output.
 * Thesis: SLiM "SLiM-LoRA low-rank adapters" (W ~ W^C + L R) and SLoPe eq. sparse_plus_low_rank
 * with the adapter as a parallel path; the adapter product is fused into the same kernels.
 *
 *   X       [M, K] in `xdtype` (SLIM_BF16 or SLIM_F16), device.
 *   M, N, K M >= 1, N >= 16, N % 16 == 0, K % 128 == 0.
 *   codes, meta, scales   forward pack of W (slim_pack).
 *   Lt, Rt  the adapter laid out by slim_pack_adapter: Lt fp16 [r, K] = L^T row-major, Rt fp16 R^T
 *           in 32 x 16 tiles (a plain row-major R^T gives wrong results); both NULL when
 *           r == 0. r % 16 == 0.
 *   Y       out, fp32 [M, N]. Must not alias any input.
 *   ws      device workspace of slim_linear_workspace(M, N, K, r) bytes or more (see there for less), zeroed
 *           once with slim_workspace_init before its first use. Two calls that overlap in time must
 *           not share a workspace.
 * Sizes past the kernels' 32-bit offsets return SLIM_EUNSUPPORTED: for M > 32, K above 2^23, or
 * ceil(M/32)*32*r or ceil(N/32)*32*r of 2^30 or more.
 * Operand precision: see "Precision" above (row-scaled fp16 activations, fp16 dequantised
 * weights, fp32 accumulation). Deterministic: identical inputs give identical bits.
 */
int slim_linear(const void* X, int xdtype, int64_t M, int64_t N, int64_t K, const uint8_t* codes,
                const uint8_t* meta, const uint16_t* scales, const uint16_t* Lt, const uint16_t* Rt,
                int64_t r, float* Y, void* ws, size_t ws_bytes, void* stream);

/*
 * slim_linear_qa - Y = X * Wc^T + (X * L^Q) * R^Q with the 4-bit adapters of slim_pack_adapter_q
 * (L^Q, R^Q their dequantized values (u - 8) * s16). Thesis: SLiM-LoRA^Q, the quantized adapters of
 * SLiM's deployed layer ("Low-rank adapter quantization"; quantized-adapter rows of the SLiM
 * results and speedup tables).
 *
 *   Arguments as slim_linear, with Lq, Ls, Rq, Rs in place of Lt, Rt; r >= 32, r % 32 == 0.
 *   ws      slim_linear_qa_workspace(M, N, K, r) bytes (for less see slim_linear_workspace), zeroed once with
 *           slim_workspace_init.
 * At M <= 32 the kernels dequantize the factors in registers as they stream them; at M > 32 the
 * first launch expands them to fp16 in the workspace. The dequantized factor values are
 * (u - 8) * s16 rounded to fp16 (as for the weights); otherwise precision as slim_linear.
 */
int slim_linear_qa_workspace(int64_t M, int64_t N, int64_t K, int64_t r, size_t* bytes);
int slim_linear_qa(const void* X, int xdtype, int64_t M, int64_t N, int64_t K, const uint8_t* codes,
                   const uint8_t* meta, const uint16_t* scales, const uint8_t* Lq, const uint16_t* Ls,
                   const uint8_t* Rq, const uint16_t* Rs, int64_t r, float* Y, void* ws, size_t ws_bytes,
                   void* stream);

/*
 * slim_linear_bwd_dx - dX = dY * W^{R,C} + (dY * R^T) * L^T, fp32 accumulation, fp32 output.
 * Thesis: SLoPe eq. sparse_backward_input (BWD-2 with the double-pruned weight) plus the adapter
 * path's input gradient.
 *
 *   dY      [M, N] in `dydtype` (SLIM_BF16 or SLIM_F16), device.
 *   M, N, K M >= 1, N % 16 == 0, K % 128 == 0.
 *   codesT, metaT, scalesT   backward pack (slim_pack_bwd).
 *   L, R    fp16 [K, r] and [r, N]; both NULL when r == 0. r % 16 == 0.
 *   dX      out, fp32 [M, K].
 *   ws      workspace of slim_bwd_dx_workspace(M, N, K, r) bytes (for less see slim_linear_workspace), zeroed once.
 * Sizes past the kernels' 32-bit offsets return SLIM_EUNSUPPORTED: for M > 32, N above 2^23, or
 * ceil(M/32)*32*r or ceil(K/32)*32*r of 2^30 or more.
 * Operand precision: the weight codes enter the matrix cores as exact small integers; the fp16
 * scale s16[n, k/128] multiplies the row-scaled gradient and the product is rounded to fp16 once
 * (see "Precision" above). Deterministic.
 */
int slim_linear_bwd_dx(const void* dY, int dydtype, int64_t M, int64_t N, int64_t K,
                       const uint8_t* codesT, const uint8_t* metaT, const uint16_t* scalesT,
                       const uint16_t* L, const uint16_t* R, int64_t r, float* dX, void* ws,
                       size_t ws_bytes, void* stream);

/*
 * slim_linear_noalloc - slim_linear without a caller workspace, for callers that cannot allocate
 * device memory (code under HIP graph capture, tight serving loops, harnesses that forbid
 * allocation). Same arguments, results and precision as slim_linear, minus ws / ws_bytes.
 *
 * The workspace is a fixed array of SLIM_NOALLOC_SCRATCH_BYTES (64 MiB) of device memory that the
 * library holds per device from the first call on that device until the process ends; its first
 * call on a device also enqueues a small kernel that clears the array's counter region. The call
 * allocates nothing (no hipMalloc, hipFree or allocating library routine) and records no timing
 * events. Sizes whose kernels need more than SLIM_NOALLOC_SCRATCH_BYTES return
 * SLIM_EWORKSPACE before touching any device; that covers every M <= 32 layer of the shapes here
 * and the 11008 x 4096 layer at M = 2048, but not, for example, a 5120 x 5120 layer at M = 4096.
 * All calls on one device share its array, so two calls that overlap in time on one device
 * (different streams or threads) race and give undefined results; serialise them.
 */
#define SLIM_NOALLOC_SCRATCH_BYTES (64u << 20)
int slim_linear_noalloc(const void* X, int xdtype, int64_t M, int64_t N, int64_t K, const uint8_t* codes,
                        const uint8_t* meta, const uint16_t* scales, const uint16_t* Lt, const uint16_t* Rt,
                        int64_t r, float* Y, void* stream);

/*
 * ---- The rest of SLoPe's sparse training step (SLoPe, Alg. "Accelerated Sparse Pretraining
 * Algorithm for a Linear Layer": setup of the sparse weight and its transpose, the weight gradient
 * with the weight's mask, the sparse add of the optimizer with weight decay, and the update of both
 * sparse matrices; appendix "Implementation details"). Training weights are kept in half precision,
 * so these calls work on value packs instead of the int4 inference pack:
 *
 *   vals   fp16 bits [rows, len/2], row-major: for aligned group g of four positions of a row,
 *          the values at its two kept positions, the lower position first (2g, 2g + 1);
 *   meta   uint8 [rows, len/8], row-major, the inference pack's index format (little-endian
 *          half-word b covers positions 16b .. 16b+15; its group c holds the kept offsets
 *          i0 < i1 in bits 4c..4c+1 and 4c+2..4c+3).
 *
 * The forward pack of W^R has rows = N, len = K (2:4 along K); its transposed pack W^{R,C} has
 * rows = K, len = N (2:4 along N). Every pointer is device memory, 16-byte aligned, owned by the
 * caller; every call enqueues on `stream` and returns after the launch unless stated otherwise.
 * ----
 *
 * slim_pack16 - setup of W^R from fp32 W [N, K] (row-major): per aligned group of four along K,
 * keep the two largest |w| (ties: lower position), store them rounded to fp16 (nearest, ties to
 * even) in vals [N, K/2] with meta [N, K/8]; mask (optional, uint8 [N, K], 0/1) receives M^R.
 * K % 16 == 0. Synchronous (reads back a status word): SLIM_ENONFINITE if W holds a NaN or Inf.
 */
int slim_pack16(const float* W, int64_t N, int64_t K, uint16_t* vals, uint8_t* meta, uint8_t* mask,
                void* stream);

/*
 * slim_pack16_t - W^{R,C} from a W^R value pack (SLoPe eq. sparse_backward_input's double
 * pruning): for each column k and aligned group of four rows, keep the two entries ranked first by
 * (|v| descending, M^R bit descending, row ascending) and store them (0 for a kept slot M^R had
 * dropped) in valsT [K, N/2] with metaT [K, N/8]. Run at setup and after every update of vals.
 * N % 64 == 0 and K % 64 == 0; the values must be finite.
 */
int slim_pack16_t(const uint16_t* vals, const uint8_t* meta, int64_t N, int64_t K, uint16_t* valsT,
                  uint8_t* metaT, void* stream);

/*
 * slim_grad_w - BWD-1 with the weight's mask (SLoPe eq. sparse_backward_weight and "pruneAndCompress"):
 * gW [N, K/2] fp32 = (dY^T X) at the positions meta (M^R, [N, K/8]) keeps, in the value-pack order.
 * dY [M, N] and X [M, K] row-major, both of `dtype` (SLIM_F16 or SLIM_BF16); products exact in
 * fp32, accumulated in fp32 along M (the order differs from a sequential sum). N % 128 == 0,
 * K % 128 == 0, M >= 1; SLIM_EUNSUPPORTED if M N or M K reaches 2^31 elements.
 */
int slim_grad_w(const void* dY, const void* X, int dtype, int64_t M, int64_t N, int64_t K, const uint8_t* meta,
                float* gW, void* stream);

/*
 * slim_sparse_add - out = beta A + gamma B on `count` compressed values sharing one pattern ("sparseAdd":
 * in the training step, A the masked gradient with beta = 1 / loss scale and B the weight values
 * with gamma = the weight decay). A and out fp32, B fp16 bits; computed in fp32 as
 * fma(gamma, B, beta A). count % 8 == 0; out may alias A.
 */
int slim_sparse_add(const float* A, const uint16_t* B, float beta, float gamma, float* out, int64_t count,
                    void* stream);

/*
 * slim_update_pack16 - write the optimizer's new compressed values Wnew (fp32, `count` of them, the
 * pack's order) into vals, rounded to fp16 (nearest, ties to even); the pattern (meta) is unchanged.
 * Follow with slim_pack16_t to rebuild the transposed pack ("updateSparseMatrix" on both).
 * count % 8 == 0.
 */
int slim_update_pack16(const float* Wnew, int64_t count, uint16_t* vals, void* stream);

/*
 * SLiM-Quant: one symmetric quantisation parameter alpha for a whole weight by minimising the
 * expected squared quantisation error over the distribution of |w| (SLiM chapter, "SLiM-Quant
 * quantization method": eq. error_summation = eq. quantization_error + eq. clipping_error,
 * integrated on a histogram of |w|; Alg. quantization for the candidate grids).
 *
 * slim_quant_bins - the histogram size of the SLiM setup, max(512, min(floor(N K / 1000), 20000)).
 *
 * slim_quant_search - histogram and search.
 *   W       fp32, `count` values (any shape, e.g. a weight [N, K]), device; count % 4 == 0,
 *           16-byte aligned.
 *   bits    quantiser width q, 2..8: codes in [-(2^(q-1) - 1), 2^(q-1) - 1], step alpha / (2^(q-1) - 1).
 *   bins    1..20480 equal bins over [0, max|w|]; |w| falls in bin floor(|w| bins / max|w|) (exact
 *           rational floor; the maximum in the last bin).
 *   hist    out, device uint32 [bins]: the counts.
 *   out     out, device float64 [4 + 2 * 30]: [0] alpha*, [1] E(alpha*), [2] max|w|, [3] the number C
 *           of candidates evaluated, then C pairs (alpha_i, E(alpha_i)) in evaluation order.
 * E(alpha) weighs each bin's count at its centre (b + 1/2) max|w| / bins: a centre c <= alpha
 * contributes (delta rint(c / delta) - c)^2 (delta = alpha / (2^(q-1) - 1), ties to even), one
 * above alpha (alpha - c)^2; E is their count-weighted mean, in float64. Candidates: i max|w| / 10
 * for i = 1..10, then (a - max|w| / 10) + j max|w| / 100 for j = 0..19 around the best of those, a,
 * the positive ones only; alpha* is the first candidate of least error. All-zero W gives alpha* = 0
 * and C = 0. Returns SLIM_ENONFINITE for NaN/Inf in W. This call synchronises `stream` (it reads
 * back a status word) and allocates under 4 KiB of device memory for the duration of the call.
 *
 * slim_pack_alpha - slim_pack with the per-tensor parameter in place of each group's absmax: every
 * group's scale is s16 = fp16_RNE(fp32(alpha) / 7.0f), so weights beyond alpha clip to +-7 (same
 * layout, mask rule, codes, status codes and synchronisation as slim_pack).
 *   alpha   device pointer to one float64 (e.g. `out` of slim_quant_search), 8-byte aligned;
 *           negative or NaN gives SLIM_ERANGE.
 */
int slim_quant_bins(int64_t N, int64_t K);
int slim_quant_search(const float* W, int64_t count, int bits, int64_t bins, uint32_t* hist, double* out,
                      void* stream);
int slim_pack_alpha(const float* W, int64_t N, int64_t K, const double* alpha, uint8_t* codes, uint8_t* meta,
                    uint16_t* scales, uint8_t* mask, void* stream);

/*
 * SLiM-LoRA: saliency-based low-rank adapters fitted to the compression error (SLiM chapter,
 * "SLiM-LoRA low-rank adapters": eq. lora_wanda_objective_function, eq. lora_svd, Alg. lora).
 *
 * slim_lora_workspace - bytes of workspace slim_lora needs for an [N, K] weight, B calibration rows
 * and rank r (float64 buffers: the saliency-weighted error, its d x d Gram matrix and eigenvectors,
 * d = min(N, K) rounded up to 64; about 8 (d max(N, K) + 2 d^2) bytes).
 *
 * slim_lora - the adapters.
 *   W                fp32 [N, K], device: the uncompressed weight.
 *   codes/meta/scales its forward pack (slim_pack or slim_pack_alpha), device: W^C.
 *   X, xdtype, B     calibration activations [B, K] (bf16 or fp16), device.
 *   r                rank, 0 <= r <= min(N, K).
 *   L, R             out, fp32 [K, r] and [r, N], device: W ~ W^C + (L R)^T, i.e. the layer's adapter.
 *   sigma            out, optional (NULL to skip): float64 [r], the r largest singular values of S.
 *   sweeps           out, optional host int: Jacobi sweeps run.
 *   ws, ws_bytes     workspace (slim_lora_workspace), 16-byte aligned; contents undefined after.
 * With x_k = mean_i |X[i, k]| + min_j mean_i |X[i, j]| (the per-channel mean input magnitude shifted
 * by its smallest value) and S = diag(x) (W^C - W)^T [K, N], L = -diag(1/x) U_r Sigma_r^(1/2) and
 * R = Sigma_r^(1/2) V_r^T from the r largest singular triplets of S (ties to the lower index of
 * the Gram side); each row of R has its largest-magnitude entry positive (the first on equal
 * magnitudes), L's column following. The singular vectors come from a float64 two-sided block-
 * Jacobi eigendecomposition (blocks of 32, one inner sweep per pair) of S S^T (K <= N) or S^T S
 * (N < K), run until the off-diagonal norm is
 * below 1e-13 of the Frobenius norm (or stalls at rounding level). Returns SLIM_ERANGE if some x_k is
 * zero (a channel that is zero in every sample and is the smallest), SLIM_ENONFINITE for NaN/Inf
 * inputs and SLIM_EUNSUPPORTED if 40 sweeps do not converge. Synchronises `stream` (the sweep loop
 * reads back the off-diagonal norm); allocates nothing.
 */
int slim_lora_workspace(int64_t N, int64_t K, int64_t B, int64_t r, size_t* bytes);
int slim_lora(const float* W, int64_t N, int64_t K, const uint8_t* codes, const uint8_t* meta,
              const uint16_t* scales, const void* X, int xdtype, int64_t B, int64_t r, float* L, float* R,
              double* sigma, int* sweeps, void* ws, size_t ws_bytes, void* stream);

/*
 * PATCH hybrid tiles: a weight whose 128 x 128 tiles are each dense or 2:4 sparse, in fp16, and its
 * product (PATCH chapter, "Efficient deployment of PATCH": hybrid sparse-dense tiles in one GEMM,
 * 128 x 128 as the tile size; appendix "STOICC Integration").
 *
 * slim_hybrid_layout - host-only: from the tile map `kinds` (host uint8 [N/128, K/128], row-major;
 *   1 = 2:4 sparse, 0 = dense) the payload size in bytes and, if tile_info (host) is not NULL, each
 *   tile's info word: its payload's byte offset, bit 63 set for a sparse tile. Payloads follow each
 *   other in row-major tile order: a dense tile is 128 rows x 128 fp16 (32768 bytes); a sparse tile
 *   is two halves (positions 0..63, then 64..127) of 9216 bytes: 128 rows x 32 fp16 kept values
 *   (group g of the half's 16 groups at 2g, 2g+1, the lower position first), then 128 rows x 4
 *   uint16 index half-words (half-word b covers the half's positions 16b .. 16b+15; group c holds
 *   i0 in bits 4c..4c+1 and i1 in bits 4c+2..4c+3); 18432 bytes.
 *   N, K multiples of 128.
 *
 * slim_pack_hybrid - one-time pack of fp32 W [N, K] (device) with the tile map `kinds` (host):
 *   writes tile_info (device uint64 [N/128, K/128]) and the payload (device, payload_bytes from
 *   slim_hybrid_layout). A sparse tile keeps the two largest |w| of every aligned group of four along
 *   K (the lower position on equal magnitude); all kept values are rounded to fp16 (nearest, ties to
 *   even). Returns SLIM_ENONFINITE for NaN/Inf in W; synchronises `stream` (status read-back) and
 *   allocates 4 bytes of device memory for the call.
 *
 * slim_linear_hybrid_workspace / slim_linear_hybrid - Y = X Wp^T.
 *   X          fp16 [M, K], device.            tile_info, payload   the hybrid pack, device;
 *                                              payload_bytes        its size, below 4 GiB.
 *   Y          out, fp32 [M, N], device.       ws, ws_bytes         workspace (split partials of
 *              small-M calls; 0 bytes when the call needs none), 16-byte aligned.
 * Dense tiles run on v_mfma_f32_32x32x16_f16, sparse tiles on v_smfmac_f32_32x32x32_f16 (half
 * the issue for the same K); fp32 accumulation; the split partials are summed in split order, so
 * results are deterministic. Asynchronous; allocates nothing.
 */
int slim_hybrid_layout(const uint8_t* kinds, int64_t N, int64_t K, uint64_t* tile_info, size_t* payload_bytes);
int slim_pack_hybrid(const float* W, int64_t N, int64_t K, const uint8_t* kinds, uint64_t* tile_info,
                     uint8_t* payload, size_t payload_bytes, void* stream);
int slim_linear_hybrid_workspace(int64_t M, int64_t N, int64_t K, size_t* bytes);
int slim_linear_hybrid(const void* X, int64_t M, int64_t N, int64_t K, const uint64_t* tile_info,
                       const uint8_t* payload, size_t payload_bytes, float* Y, void* ws, size_t ws_bytes,
                       void* stream);

/*
 * ---- The 8-bit path: the norm before a linear layer, activations kept in 8 bits (as the next
 * layer's input and as the backward's checkpoint), the product of two 8-bit operands with a scale
 * for each block of 128, and the weight gradient from an 8-bit checkpoint. The thesis also gives a
 * layer's input 8 bits (SLiM appendix, FP8 input quantization, one scale for a tensor); here every
 * group of 128 has its own, as the thesis's weights have.
 *
 * Format. A value is c 2^e: c an e4m3 code (OCP: sign, 4 exponent bits, 3 mantissa bits, largest
 * 448, NaN 0x7F and 0xFF, no infinities), e one integer for each group of 128 consecutive values of
 * a row (of weights: for each 128 x 128 block), the smallest e >= -126 with (largest finite
 * magnitude of the group) / 2^e <= 448. Codes are value / 2^e rounded to nearest, ties to even. A
 * NaN or an infinity becomes the code NaN and does not count towards its group's e. Exponents are
 * stored as bytes e + 127.
 *   rows      codes uint8 [M][K rounded up to 128], the columns past K zero; exponents uint8
 *             [M][K/128 rounded up to 4], the bytes past the last group zero.
 *   weights   tiles of 16 rows and 128 columns, 2 KiB each: codes uint8
 *             [N/16 up][K/128 up][2][4][16][16], where byte i of [half][block][row] is the code of
 *             row `row`, column 32 block + 16 half + i of the tile, zeros past N and K; exponents
 *             uint8 [N/128 up][K/128 rounded up to 4], the bytes past the last block zero.
 * 16-bit and fp32 operands may have rows of any stride >= their width (in elements) and start at
 * any element; codes and exponents are 16-byte aligned. M = 0 is allowed: nothing is read, and
 * sums over rows are zero. Rows are at most 2^22 columns. What one launch cannot take returns
 * SLIM_EUNSUPPORTED: 2^29 groups in slim_quant8 and slim_dequant8, 2^22 rows of more than 16384 columns
 * in the norms (slim_norm_bwd in fp32: of more than 8192 that are no multiple of 8), 2^36 elements of dY
 * in slim_grad_w8, 2^23 tiles in slim_grad_w8 and 2^24 in slim_linear8 (2^36 results at least) and in the products that end
 * in an activation, 2^32 - 64 groups of dh in slim_act_bwd, 2^26 - 3 rows or 2^24 blocks of 16 rows, 2048 columns
 * and one expert in slim_route, 2^24 tiles of 16 columns of h over the experts that slim_moe8's rows may pick (512 experts: F
 * past 2^19 - 128).
 * Every call is asynchronous, allocates nothing, may be captured into a graph, and gives the same bits for the same
 * inputs.
 * ----
 *
 * slim_quant8 - X [M, K] (`dtype` SLIM_F16, SLIM_BF16 or SLIM_F32, row stride ldx) in 8 bits.
 * slim_dequant8 - the values back in `dtype`, row stride ldy, rounded to nearest: exact in fp32 and, from
 *   2^-130 on, in bf16; in fp16 for values that came from fp16 below 63488. What passes the type's range is
 *   infinite: in fp16 past 65519, in fp32 and bf16 values from 248 2^120 on (within 3 % of their largest),
 *   whose nearest code is 256.
 */
int slim_quant8(const void* X, int dtype, int64_t M, int64_t K, int64_t ldx, uint8_t* codes, uint8_t* exps, void* stream);
int slim_dequant8(const uint8_t* codes, const uint8_t* exps, int64_t M, int64_t K, void* Y, int dtype, int64_t ldy,
                  void* stream);

/*
 * slim_pack8 - W [N, K] (`dtype` SLIM_F16, SLIM_BF16 or SLIM_F32, row stride ldw) as an 8-bit weight:
 *   codes, exps     rows N, columns K: the forward's operand. Both NULL: not wanted.
 *   codesT, expsT   W^T (rows K, columns N), the same values: the input gradient's. Both NULL: not wanted.
 * A weight's NaN or infinity becomes NaN; no status word is read back.
 */
int slim_pack8(const void* W, int dtype, int64_t N, int64_t K, int64_t ldw, uint8_t* codes, uint8_t* exps,
               uint8_t* codesT, uint8_t* expsT, void* stream);

/*
 * slim_linear8 - Y [M, N] = X W^T with an 8-bit weight (rows N, columns K). The input gradient
 * dX = dY W is the same call on the transposed pack: X = dY, N and K exchanged, codesT, expsT.
 *   X, xdtype   [M, K]: SLIM_Q8_E4M3 codes with exponents xexps (ldx is not looked at); or SLIM_F16,
 *               SLIM_BF16 or SLIM_F32 with row stride ldx (xexps is not looked at), which the call
 *               turns into 8 bits first, to the bit as slim_quant8 does.
 *   Y, ydtype   out, SLIM_F16 or SLIM_BF16, row stride ldy.
 *   ws          slim_linear8_workspace(xdtype, M, N, K) bytes (0 when the call needs none); its
 *               contents need not be kept or cleared.
 * Sums are fp32, but for those of each eight consecutive products, which the scaled matrix instructions
 * cut at 2^-13 of the largest of them: together 2e-5 of the result's norm, 4.5e-5 where a hundredth of X's
 * channels is twenty times the rest, before Y is rounded to 16 bits (2e-4 in fp16, 1.7e-3 in bf16). For
 * that reason fp32 is not offered for Y.
 */
int slim_linear8_workspace(int xdtype, int64_t M, int64_t N, int64_t K, size_t* bytes);
int slim_linear8(const void* X, int xdtype, const uint8_t* xexps, int64_t M, int64_t N, int64_t K, int64_t ldx,
                 const uint8_t* codes, const uint8_t* exps, void* Y, int ydtype, int64_t ldy, void* ws, size_t ws_bytes,
                 void* stream);

/*
 * slim_linear8_act - a product that ends in an activation: z = X W^T + bias, Y = act(z) mul + residual, the sums as
 * slim_linear8's and all that follows in fp32, rounded once.
 *   X .. exps   as slim_linear8.                    act        a slim_act.
 *   bias        [N] of `bdtype` (SLIM_F16, SLIM_BF16, SLIM_F32), or NULL.
 *   mul, residual  [M, N] of `dtype` with row strides ldmul, ldres, or NULL: a gate's factor, what Y is added to.
 *   dtype, q8   SLIM_F16 or SLIM_BF16: the type of mul, residual, Y and pre; with q8 nonzero Y and pre leave as 8-bit
 *               rows instead (codes with exponents yexps, preexps; ldy, ldpre are not looked at), rounded from fp32.
 *   Y           out, row stride ldy.
 *   pre         out, NULL if not wanted: z, for the backward; row stride ldpre.
 *               In 16 bits Y and pre may each be mul or residual, in the very place: the same address and row stride. But
 *               for that they and their exponents share no memory with each other, X, bias, mul or residual (SLIM_EINVAL).
 *   ws          slim_linear8_act_workspace(xdtype, M, N, K, dtype, q8) bytes; its contents need not be kept or cleared.
 *
 * slim_bwd_dx8_act - the gradient through the activation in front of a product: dh = dY W, the input gradient of the
 * product that took act(u) mul, then dU = dh mul act'(u), dmul = dh act(u) and dbias = the sum of dU over the rows.
 *   dY .. expsT  M, N, K as in the product's forward (W [N, K], dY [M, N], dh [M, K]), dY of any type that
 *               slim_linear8 takes, codesT and expsT its transposed pack.
 *   U, udtype   [M, K], the kept argument: `dtype` with row stride ldu, or SLIM_Q8_E4M3 with uexps. May be NULL with
 *               SLIM_ACT_NONE where mul is.
 *   mul         [M, K] like U (ldmul or mulexps), the gate's factor, or NULL; then dmul is NULL too.
 *   dtype       SLIM_F16 or SLIM_BF16, of dU, dmul (row strides lddu, lddmul) and dbias.
 *   dU, dmul    out. Each may be U or mul in 16 bits, in the very place: the same address and row stride. But for that dU, dmul and
 *               dbias share no memory with each other, U, mul or an 8-bit dY (SLIM_EINVAL).
 *   dbias       out, [K] of `dtype`, or NULL: sums in fp32, rounded once at the end. That rounding is most of its error (bf16's some
 *               forty times what the product's sums are off, fp16's five times), and past fp16's range it is infinite: where the
 *               bias's gradient is to be fp32, slim_act_bwd gives it, from a dh that is rounded to 16 bits instead.
 *   ws          slim_bwd_dx8_act_workspace(dydtype, M, N, K, dtype, dbias != NULL) bytes, as above.
 *
 * slim_act_bwd - the same from a dh at hand: dH [M, K] of `dtype`, row stride lddh. dU or dmul may be dH, as above. dbias fp32.
 *   ws          slim_act_bwd_workspace(M, K, dbias != NULL) bytes, as above.
 */
int slim_linear8_act_workspace(int xdtype, int64_t M, int64_t N, int64_t K, int dtype, int q8, size_t* bytes);
int slim_linear8_act(const void* X, int xdtype, const uint8_t* xexps, int64_t M, int64_t N, int64_t K, int64_t ldx,
                     const uint8_t* codes, const uint8_t* exps, int act, const void* bias, int bdtype, const void* mul,
                     int64_t ldmul, const void* residual, int64_t ldres, int dtype, int q8, void* Y, int64_t ldy, uint8_t* yexps,
                     void* pre, int64_t ldpre, uint8_t* preexps, void* ws, size_t ws_bytes, void* stream);
int slim_bwd_dx8_act_workspace(int dydtype, int64_t M, int64_t N, int64_t K, int dtype, int sums, size_t* bytes);
int slim_bwd_dx8_act(const void* dY, int dydtype, const uint8_t* dyexps, int64_t M, int64_t N, int64_t K, int64_t lddy,
                     const uint8_t* codesT, const uint8_t* expsT, int act, const void* U, int udtype, const uint8_t* uexps,
                     int64_t ldu, const void* mul, const uint8_t* mulexps, int64_t ldmul, int dtype, void* dU, int64_t lddu,
                     void* dmul, int64_t lddmul, void* dbias, void* ws, size_t ws_bytes, void* stream);
int slim_act_bwd_workspace(int64_t M, int64_t K, int sums, size_t* bytes);
int slim_act_bwd(const void* dH, int dtype, int64_t lddh, int64_t M, int64_t K, int act, const void* U, int udtype,
                 const uint8_t* uexps, int64_t ldu, const void* mul, const uint8_t* mulexps, int64_t ldmul, void* dU, int64_t lddu,
                 void* dmul, int64_t lddmul, float* dbias, void* ws, size_t ws_bytes, void* stream);

/*
 * slim_route - the router in front of a layer of experts: p = softmax(x Wr^T) over E experts for each row x of X, then the `top` largest.
 *   X, xdtype   [M, K]: SLIM_F16, SLIM_BF16 or SLIM_F32 with row stride ldx, or SLIM_Q8_E4M3 with xexps.
 *   Wr, wdtype  [E, K]: SLIM_F16, SLIM_BF16 or SLIM_F32, row stride ldw. E <= 512.
 *   top         1 .. min(E, 16).                    renorm   nonzero: weights are divided by their row's sum.
 *   ids         out, int32 [M, top]: experts by falling logit, the lower number first where two are equal.
 *   weights     out, fp32 [M, top]: their p.
 *   ws          slim_route_workspace(M, E, K) bytes; its contents need not be kept or cleared.
 * Arithmetic is fp32: experts whose logits differ by less than the error of their sums, (K / 256 + 80) 2^-24 of the magnitudes', may
 * change places. A row with a NaN among its logits has weights of NaN, and those experts last that gave it.
 *
 * slim_moe8 - a layer of experts for a few tokens: y_i = sum_j w_ij down_e(act(gate_e x_i) * (up_e x_i)) (+ residual), e = ids_ij.
 *   X, xdtype   [M, D], M <= 64: SLIM_F16 or SLIM_BF16 with row stride ldx, or SLIM_Q8_E4M3 with xexps, whose values stand for x.
 *   gate, up    E weights of rows F, columns D, each as slim_pack8's, one after the other (codes E [F/16 up][D/128 up] tiles, exponents
 *               E [F/128 up] rows). up NULL: h = act(gate x).            down     E weights of rows D, columns F.
 *   act         a slim_act.
 *   ids, weights  [M, top] as slim_route's, E <= 512, top <= 16. A number outside 0 .. E - 1 adds nothing (a row of padding, a dropped
 *               token); one that is twice in a row adds twice.
 *   residual    [M, D] of `dtype`, row stride ldres, or NULL.
 *   Y, dtype    out, SLIM_F16 or SLIM_BF16, row stride ldy; may be X, and the residual in the very place (the same address and row
 *               stride), but share no other memory with the residual, ids or weights (SLIM_EINVAL).
 *   ws          slim_moe8_workspace(M, D, F, E, top) bytes; its contents need not be kept or cleared.
 * x is not rounded to 8 bits, nor is h, which is held to 16 significant bits; sums are fp32, the experts' of a row in order of number.
 */
int slim_route_workspace(int64_t M, int64_t E, int64_t K, size_t* bytes);
int slim_route(const void* X, int xdtype, const uint8_t* xexps, int64_t M, int64_t K, int64_t ldx, const void* Wr, int wdtype, int64_t E,
               int64_t ldw, int top, int renorm, int32_t* ids, float* weights, void* ws, size_t ws_bytes, void* stream);
int slim_moe8_workspace(int64_t M, int64_t D, int64_t F, int64_t E, int top, size_t* bytes);
int slim_moe8(const void* X, int xdtype, const uint8_t* xexps, int64_t M, int64_t D, int64_t ldx, int64_t F, int64_t E, const uint8_t* gate,
              const uint8_t* gate_exps, const uint8_t* up, const uint8_t* up_exps, const uint8_t* down, const uint8_t* down_exps, int act,
              const int32_t* ids, const float* weights, int top, const void* residual, int64_t ldres, void* Y, int dtype, int64_t ldy,
              void* ws, size_t ws_bytes, void* stream);

/*
 * slim_grad_w8 - the weight gradient dY^T X with X [M, K] an 8-bit checkpoint (xcodes, xexps).
 *   dY, dtype   [M, N], SLIM_F16 or SLIM_BF16, row stride lddy. X is widened to the same type: exact in
 *               bf16 from 2^-130 on; in fp16 values below its normal range are rounded to multiples of
 *               2^-24, and in a group of 128 columns with values past 448 2^7 to less than 2^-39 of its
 *               largest over the rows (no value of X is lost to fp16's range). Products are exact, sums
 *               fp32 along M.
 *   meta        NULL: gW fp32 [N, K], all of it. Else the index words of a value pack (slim_pack16,
 *               [N, K/8], K % 16 == 0): gW fp32 [N, K/2] at the positions they keep, as slim_grad_w.
 *   ws          slim_grad_w8_workspace(M, N, K, meta != NULL, aligned) bytes, where `aligned` says that
 *               dY is 16-byte aligned and lddy a multiple of 8 below 2^22 (0 always suffices); its
 *               contents need not be kept or cleared.
 */
int slim_grad_w8_workspace(int64_t M, int64_t N, int64_t K, int masked, int aligned, size_t* bytes);
int slim_grad_w8(const void* dY, int dtype, int64_t lddy, const uint8_t* xcodes, const uint8_t* xexps, int64_t M,
                 int64_t N, int64_t K, const uint8_t* meta, float* gW, void* ws, size_t ws_bytes, void* stream);

/*
 * slim_norm - y = (x - mu) rstd gamma + beta for each row x of X [M, K], rstd = (v + eps)^(-1/2), mu
 * and v the row's mean and variance (divided by K); with rms nonzero mu = 0 and v the mean square.
 *   X, dtype    SLIM_F16, SLIM_BF16 or SLIM_F32, row stride ldx.
 *   gamma, beta [K] of `pdtype` (any of the three); NULL for ones and zeros. No beta with rms.
 *   Y, ydtype   out: `dtype`, row stride ldy; or SLIM_Q8_E4M3: codes with exponents yexps (ldy is not
 *               looked at), rounded to 8 bits from fp32 without a rounding to 16 bits between.
 *   mean, rstd  out, fp32 [M], for the backward; mean may be NULL.
 * eps >= 0. All arithmetic is fp32, the variance taken about the mean.
 *
 * slim_norm_bwd - the gradients, with xh = (x - mean) rstd and t = dy gamma:
 *   dx = rstd (t - mean_k(t) - xh mean_k(t xh)), dgamma = sum over rows of dy xh, dbeta = that of dy.
 *   dY, dtype   [M, K], row stride lddy; dX out, the same type, row stride lddx (may be dY).
 *   X, xdtype   the forward's input: `dtype` with row stride ldx, or SLIM_Q8_E4M3 with xexps: a
 *               checkpoint of it (slim_quant8), whose rounded values stand in for x.
 *   gamma       as in the forward.
 *   mean, rstd  the forward's; mean NULL for the RMS norm (whose dx has no mean_k(t)).
 *   dgamma, dbeta  out, fp32 [K]; NULL if not wanted.
 *   ws          slim_norm_bwd_workspace(M, K) bytes; its contents need not be kept or cleared.
 */
int slim_norm(const void* X, int dtype, int64_t M, int64_t K, int64_t ldx, const void* gamma, const void* beta,
              int pdtype, int rms, float eps, void* Y, int ydtype, int64_t ldy, uint8_t* yexps, float* mean, float* rstd,
              void* stream);
int slim_norm_bwd_workspace(int64_t M, int64_t K, size_t* bytes);
int slim_norm_bwd(const void* dY, int dtype, int64_t lddy, const void* X, int xdtype, const uint8_t* xexps, int64_t ldx,
                  int64_t M, int64_t K, const void* gamma, int pdtype, const float* mean, const float* rstd, void* dX,
                  int64_t lddx, float* dgamma, float* dbeta, void* ws, size_t ws_bytes, void* stream);

/*
 * Per-kernel timing for benchmarks (host-side bookkeeping; not part of the layer's math).
 * slim_timing_enable(1) makes every later kernel launch of this library record a hipEvent
 * before and after itself on the caller's stream. slim_timing_read waits for the recorded
 * events and writes one line per kernel name, "name launches total_ms median_ms\n", into buf (host);
 * it returns 0, or the buffer size needed when buf is NULL or too small. slim_timing_reset
 * clears the totals. These three calls are the library's only process-wide mutable state (a
 * mutex-guarded switch, event pool and totals); with timing off, which is the default, the layer
 * calls read nothing of it but the switch. Thread-safe; timing adds two event records per launch
 * while enabled, and never records inside a stream capture.
 */
int slim_timing_enable(int on);
int slim_timing_reset(void);
int slim_timing_read(char* buf, size_t buf_len);

#ifdef __cplusplus
}
#endif
#endif /* SLIM_H */
