/*
 * attn.h -- C ABI of the MI355X (gfx950) exact-attention library.
 *
 * The library computes, for B*H independent problems of N tokens and head
 * dimension d (paper: Section 2.2 and Appendix B.3),
 *
 *     S = tau * Q K^T,  S_masked = MASK(S),  P = softmax(S_masked) row-wise,
 *     P_dropped = dropout(P, p_drop),        O = P_dropped V,
 *
 * without ever writing S or P to memory (tiling with an online softmax,
 * Section 3.1 / Algorithm 1 and 2), and the gradients dQ, dK, dV of a scalar
 * loss given dO by recomputing S and P tile by tile from Q, K, V and the saved
 * per-row statistic (Appendix B.2 and B.4 / Algorithm 4).  A block mask turns
 * both passes into the block-sparse variant (Section 3.3 / Algorithm 5).
 *
 * General conventions
 *   - Every tensor pointer is a DEVICE pointer owned by the caller.  The
 *     library never allocates, frees, or keeps a pointer after a call returns.
 *   - Q, K, V, O, dO, dQ, dK, dV are [B, H, N, d] arrays of 16-bit floats
 *     (fp16 or bf16, chosen by attn_params.dtype) with d contiguous; the
 *     element strides of the b, h and n axes are given in attn_params and are
 *     shared by all of these tensors (all three 0 = densely packed).
 *   - LSE is a packed [B, H, N] float array: L_i = m_i + ln(l_i), the natural
 *     logsumexp of row i of the scaled, masked logits.  It replaces the pair
 *     (l, m) that Algorithm 2 saves; P_ij = exp(S_ij - L_i).
 *   - Calls are asynchronous on attn_params.stream (a hipStream_t, may be
 *     NULL for the default stream), never synchronise the device, and may be
 *     issued concurrently from several host threads.
 *   - Outputs are fully overwritten; the caller need not clear them.
 *   - A query row that sees no key (through a block mask, or a padded position
 *     under key_lengths) gets O = 0, LSE = -inf and contributes zero gradients.
 *   - All argument checks happen on the host before anything is launched:
 *     sizes, strides (rows 16-byte aligned, non-overlapping: the axes of size
 *     > 1 must nest by stride, as in [B,H,N,d] or a [B,N,H,d] view), tensor
 *     pointers (non-NULL, 16-byte aligned), scale, dropout, mask, workspace.
 *     Functions return ATTN_OK (0) or a negative attn_status; they never
 *     abort, throw, or print.
 *   - Every element of the input tensors must be finite, padded positions
 *     (under key_lengths) included: they enter the matrix products with weight
 *     zero, and 0 * inf is not zero.
 *
 * Supported in this version: d in {16, 32, 64, 128}; any N >= 1 for the dense entry
 * points (a last block of fewer than 128 tokens is handled inside the kernels:
 * nothing outside the [B,H,N,d] tensors is read or written), N a multiple of
 * 128 for the block-sparse ones; tau finite and > 0; 0 <= p_drop < 1;
 * mask_block == 128.
 *
 * Which kernel a call takes depends on head dimension, length, masks and the
 * number of heads; every choice computes the same operation to the same
 * tolerance.  The last bits of a head's results may therefore depend on how many
 * heads share its call (few heads are divided over groups of wavefronts, which
 * sum in an order of their own); for given sizes and options they are the same in
 * every call, but for the block-sparse columns named at attn_blocksparse_bwd.
 * attn_debug_set_variant overrides the choice for comparisons and
 * tests; its initial values come from two environment variables read once, when
 * the first call needs them: ATTN_FWD_VARIANT=base|pp and ATTN_DKV_VARIANT=rs|fr|w64.
 * Unset, the library picks by measurement.
 */
#ifndef ATTN_H_
#define ATTN_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  ATTN_OK = 0,
  ATTN_ERR_NULL = -1,       /* a required pointer is NULL */
  ATTN_ERR_SHAPE = -2,      /* B, H, N out of range, bad strides, misaligned tensor, block-sparse with N % 128 != 0 */
  ATTN_ERR_DTYPE = -3,      /* dtype is neither ATTN_FP16 nor ATTN_BF16 */
  ATTN_ERR_HEADDIM = -4,    /* d not in {16, 32, 64, 128} */
  ATTN_ERR_DROPOUT_P = -5,  /* p_drop not in [0, 1) or NaN */
  ATTN_ERR_SCALE = -6,      /* softmax_scale not finite or <= 0 */
  ATTN_ERR_WORKSPACE = -7,  /* workspace NULL, misaligned (256 B) or too small */
  ATTN_ERR_MASK = -8,       /* mask_block != 128 or negative mask stride */
  ATTN_ERR_LAUNCH = -9,     /* the HIP runtime refused the launch */
  ATTN_ERR_PAGES = -10,     /* page size no power of two in [16, 4096], or a list of page copies that names a page it must not */
  ATTN_ERR_ROTARY = -11,    /* rotary_dim odd or not in [2, d], no frequencies, or a factor that is not finite */
  ATTN_ERR_NORM = -12,      /* no weights, weights that are not aligned to their type, or eps not finite and > 0 */
  ATTN_ERR_WINDOW = -13     /* window < 1, sinks < 0, or not causal */
} attn_status;

enum { ATTN_FP16 = 0, ATTN_BF16 = 1 };

typedef struct {
  int32_t B, H, N, d;        /* problem sizes */
  int32_t dtype;             /* ATTN_FP16 or ATTN_BF16 */
  int64_t stride_b;          /* element strides of the [B,H,N,d] tensors;    */
  int64_t stride_h;          /*   all three zero means packed                */
  int64_t stride_n;          /*   (stride_n >= d, d itself has stride 1)     */
  float softmax_scale;       /* tau: multiplies Q K^T before mask and softmax */
  int32_t causal;            /* != 0: key j is visible to query i iff j <= i */
  float dropout_p;           /* p_drop in [0,1), applied rounded down to a multiple of 1/256;
                                below 1/256 the generator is switched off      */
  uint64_t seed;             /* Philox key   (the saved generator state R)   */
  uint64_t offset;           /* low 32 bits enter the Philox counter         */
  int32_t o_fp32;            /* != 0: O is read/written as float32 [B,H,N,d] packed
                                with the same strides, instead of dtype      */
  void* stream;              /* hipStream_t, borrowed for the call           */
  const int32_t* key_lengths; /* NULL, or device int32 [B]: key-padding mask (the MASK example of
                                Appendix B.3).  Tokens of batch b at positions >= key_lengths[b]
                                are padding: they are not attended to, their O is 0, their LSE
                                -inf and all gradients at those positions are 0.  Lengths are clamped to [0, N].
                                Sequences of any length are run by padding N up to a multiple
                                of 128 and passing the true lengths here.                    */
} attn_params;

/*
 * Dropout mask (bit-exact contract, shared with nothing but this text):
 * Philox-4x32 with 10 rounds (Salmon et al., SC'11), key = (seed low word,
 * seed high word), counter = (j / 16, i, b * H + h, offset low word) for query
 * row i and key column j of head (b, h); element (i, j) takes the 8-bit
 * field f = j % 16 of the 128-bit output (byte f % 4, i.e. bits [8 (f % 4),
 * 8 (f % 4) + 7], of output word f / 4) and is KEPT iff field >= T, with
 * T = floor((double)dropout_p * 2^8).  The dropout applied is therefore the one
 * with probability T / 256, dropout_p rounded down to a multiple of 1/256
 * (0.1 -> 25/256; below 1/256 nothing is dropped), and kept probabilities are
 * multiplied by 256 / (256 - T), the reciprocal of the keep probability, so
 * that the mask has expectation one.  One generator call decides sixteen
 * consecutive keys of a query.  The mask depends on indices only, so the
 * backward pass regenerates it (Appendix B.4, obs. 1).
 */

/*
 * Forward pass (Algorithm 2; Algorithm 1 when causal = 0 and dropout_p = 0).
 *   Q, K, V : in,  [B,H,N,d] dtype
 *   O       : out, [B,H,N,d] dtype (or float32 when o_fp32)
 *   LSE     : out, [B,H,N] float32, packed
 */
int attn_fwd(const attn_params* p, const void* Q, const void* K, const void* V,
             void* O, float* LSE);

/*
 * Bytes of scratch for attn_bwd with these params: two floats per query
 * row (D_i of Eq. (4), Appendix B.2, and the row statistic in base 2), i.e. the
 * O(N) additional memory of Theorem 1; never quadratic in N.  Where the one-launch
 * kernel takes heads of 257 to 512 tokens (d <= 64), a row of dQ in float32 more;
 * attn_bwd takes such problems in two launches if it is given the two floats per
 * row only (the same gradients but for the last bits).  Returns 0 if the
 * params are invalid.
 */
size_t attn_bwd_workspace_bytes(const attn_params* p);

/*
 * Same for attn_blocksparse_bwd (and attn_bwd_timed with a mask): additionally holds the
 * per-column block counts and fp32 dK/dV accumulators used when a mask column keeps so many
 * blocks (a "global token" column) that its work is split over several workgroups.  Still
 * linear in B*H*N*d.  Returns 0 if the params are invalid.
 */
size_t attn_blocksparse_bwd_workspace_bytes(const attn_params* p);

/*
 * Backward pass (Algorithm 4, with D_i = rowsum(dO_i o O_i) from Eq. (4) of
 * Appendix B.2).
 *   Q, K, V, O, dO : in,  [B,H,N,d] (O as written by attn_fwd with the same params)
 *   LSE            : in,  [B,H,N] float32 from attn_fwd
 *   dQ, dK, dV     : out, [B,H,N,d] dtype
 *   workspace      : device scratch, 256-byte aligned, of attn_bwd_workspace_bytes(p) (at least
 *                    two floats per row, rows counted in whole blocks of 128 per head);
 *                    contents on entry are ignored and on exit unspecified
 */
int attn_bwd(const attn_params* p, const void* Q, const void* K, const void* V,
             const void* O, const void* dO, const float* LSE,
             void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes);

/*
 * attn_bwd for callers that can neither allocate device memory nor pass a workspace: code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same
 * arguments and results as attn_bwd with a workspace of ATTN_STATIC_SCRATCH_BYTES (bit-identical), a
 * fixed array inside the library, per GPU, held from the first
 * use on that GPU until the process ends.  The call allocates and frees nothing.  Problems whose
 * two row vectors exceed ATTN_STATIC_SCRATCH_BYTES (more than 2^20 query rows
 * over all heads, counted in whole blocks of 128 per head) return ATTN_ERR_WORKSPACE.  All calls
 * on one GPU share that GPU's array: calls that overlap in time on one GPU (different streams or
 * threads) race and give wrong gradients; calls on one stream, or otherwise ordered, are safe,
 * and no call reads what an earlier one left there.  The device that is current when the call
 * is made must be the one that owns the tensors and the stream.
 */
#define ATTN_STATIC_SCRATCH_BYTES (8u << 20)
int attn_bwd_static(const attn_params* p, const void* Q, const void* K, const void* V,
                    const void* O, const void* dO, const float* LSE,
                    void* dQ, void* dK, void* dV);

/*
 * Block-sparse forward (Section 3.3, Algorithm 5): as attn_fwd, but entry
 * (i, j) is additionally masked out unless
 * block_mask[(i / mask_block) * T + (j / mask_block)] != 0, T = N / mask_block;
 * tiles whose block is zero are skipped, not computed.
 *   block_mask    : in, device uint8 [T, T] row-major (per head if mask_stride_h != 0)
 *   mask_block    : must be 128
 *   mask_stride_h : bytes between the masks of consecutive heads h (0 = one
 *                   mask shared by all heads; batches always share)
 */
int attn_blocksparse_fwd(const attn_params* p, const uint8_t* block_mask, int32_t mask_block,
                         int64_t mask_stride_h, const void* Q, const void* K, const void* V,
                         void* O, float* LSE);

/*
 * Block-sparse backward: Algorithm 4 restricted to the non-zero blocks (the
 * paper states only that the backward skips the same blocks, Section 3.3).
 * Arguments as attn_bwd plus the mask arguments of attn_blocksparse_fwd; the workspace must
 * hold attn_blocksparse_bwd_workspace_bytes(p) bytes.  dK and dV of mask columns that keep more
 * than 24 blocks may be split over several workgroups and summed with fp32 atomics, so their last bits may
 * differ from run to run; everything else is bit-reproducible.
 */
int attn_blocksparse_bwd(const attn_params* p, const uint8_t* block_mask, int32_t mask_block,
                         int64_t mask_stride_h, const void* Q, const void* K, const void* V,
                         const void* O, const void* dO, const float* LSE,
                         void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes);

/*
 * Attention with a sliding window and first tokens that stay visible: as attn_fwd with the causal mask (p->causal must be set), but key j is visible to query i iff
 * j <= i and (i - j < window or j < sinks): a query sees the last `window` keys, its own among them, and the first `sinks` of its sequence.  window >= 1, sinks >= 0.
 * The work is linear in N (window + sinks).  Where nothing is hidden (window + sinks >= N) this is attn_fwd.
 */
int attn_window_fwd(const attn_params* p, int32_t window, int32_t sinks, const void* Q, const void* K, const void* V, void* O, float* LSE);

/*
 * Bytes of scratch for attn_window_bwd: two floats a row (N rounded up to 128), and pieces of dK and dV in float32 for the keys that are sinks, 32 at a time: 256 d bytes each, at least two for
 * every head and 32 sinks, or none.  Where nothing is hidden, attn_bwd_workspace_bytes.  0 if the params are invalid.
 */
size_t attn_window_bwd_workspace_bytes(const attn_params* p, int32_t window, int32_t sinks);

/* Its backward pass: arguments as attn_bwd, O and LSE from attn_window_fwd.  Gradients are the same bits in every call. */
int attn_window_bwd(const attn_params* p, int32_t window, int32_t sinks, const void* Q, const void* K, const void* V, const void* O, const void* dO, const float* LSE,
                    void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes);

/*
 * Profiling aid for the backward pass (Algorithm 4 as attn_bwd / attn_blocksparse_bwd run it):
 * identical to attn_bwd when block_mask is NULL and to attn_blocksparse_bwd otherwise, and in
 * addition records the caller's four hipEvent_t handles on p->stream: events[0] and events[1]
 * before the first launch (two handles for one instant: an earlier version had a preparation
 * launch between them; D = rowsum(dO o O) is now computed inside the dQ kernel), events[2] after
 * the dQ kernel, events[3] after the dK/dV kernel (where one launch does both, both after it).  The
 * events stay owned by the caller.
 */
int attn_bwd_timed(const attn_params* p, const uint8_t* block_mask, int32_t mask_block,
                   int64_t mask_stride_h, const void* Q, const void* K, const void* V,
                   const void* O, const void* dO, const float* LSE,
                   void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes,
                   void* const* events);

/*
 * Test hook: writes the dropout keep mask of the rule above, keep[b][h][i][j] in
 * {0, 1}, as a packed device uint8 [B,H,N,N] array (N*N bytes per head: only
 * for small problems).  Uses B, H, N, dropout_p, seed, offset, stream of p.
 */
int attn_debug_dropout_mask(const attn_params* p, uint8_t* keep);

/*
 * Measurement aid, outside the paper's operation: launches on `stream` a kernel that
 * only issues 32x32x16 matrix instructions of the given dtype on register operands
 * (2048 workgroups of 4 wavefronts, 4 * iters instructions per wavefront), so a
 * benchmark that times the launch can quote the matrix rate this GPU sustains under
 * load next to the published peak.  operand_sets = 1: every instruction reads the same
 * two registers (fewest bits change between instructions: the highest clock the GPU
 * holds); operand_sets = 4: consecutive instructions read four different pseudo-random
 * operand pairs in turn, as the tile products of a real kernel do.  sink: device pointer
 * to at least one float, never written in practice; *flops (host pointer, may be NULL)
 * receives the number of floating-point operations launched.  iters in [1, 2^20].
 * Asynchronous.
 */
int attn_debug_mfma_rate(int32_t dtype, int32_t iters, int32_t operand_sets, float* sink, void* stream,
                         double* flops);

/*
 * Measurement aid: which kernels attn_fwd / attn_bwd (sparse = 0) or the block-sparse
 * entry points (sparse != 0) would launch for these params, without launching anything.
 * *fwd_kernel: 0 = free-running forward kernel, 1 = two-group forward kernel.
 * *dkv_kernel: 0 = role-split dK/dV kernel, 1 = one-wavefront kernel (d <= 64),
 * 2 = one-wavefront kernel for d = 128 (32 keys per wavefront), 3 = the same with 64 keys
 * per wavefront, 4 = short heads at d <= 64, dQ included (one launch).  (The dQ kernel is the same
 * for every other problem.)  The backward's answer is for a workspace of the two row vectors:
 * attn_debug_bwd_kernel says what a call with more runs.
 */
int attn_debug_kernel_choice(const attn_params* p, int32_t sparse, int32_t* fwd_kernel, int32_t* dkv_kernel);

/*
 * Measurement aid: which dK/dV kernel attn_bwd would launch for these params with a workspace of
 * workspace_bytes, without launching anything.  *kernel as *dkv_kernel above, or 5 = heads of 257 to
 * 512 tokens at d <= 64 in two key blocks, dQ included (one launch).  A workspace that attn_bwd would
 * refuse is refused (ATTN_ERR_WORKSPACE).
 */
int attn_debug_bwd_kernel(const attn_params* p, size_t workspace_bytes, int32_t* kernel);

/*
 * Test and comparison hook, outside the paper's operation: which kernel serves the calls that
 * have a choice.  fwd_variant: 0 = by measurement, 1 = free-running forward kernel, 2 = two-group
 * forward kernel (where both exist).  dkv_variant: 0 = by measurement, 1 = role-split dK/dV kernel
 * wherever it exists, 2 = one-wavefront dK/dV kernels with 32 keys per wavefront only, 3 = the
 * 64-keys-per-wavefront dK/dV kernel wherever it exists (d = 128, no dropout, N >= 512, N % 32 == 0).
 * While dkv_variant is not 0, short heads take the two launches too, and no kernel divides the sweep of a work item over groups of wavefronts (which
 * they do where there are few work items).
 * -1 leaves a setting unchanged.  Process-wide and thread-safe; affects calls issued afterwards.
 */
int attn_debug_set_variant(int32_t fwd_variant, int32_t dkv_variant);

/*
 * ---- Rotary positions and the paged key/value cache ----
 *
 * What a program with attention over a growing context calls around it.  The conventions above hold: device
 * pointers of the caller, the caller's stream, all argument checks on the host, nothing allocated or kept.  The device of the
 * tensors must be the current one.
 */

/* Which columns of a row turn, and how fast. */
typedef struct {
  const double* frequencies;  /* device, [rotary_dim / 2]: radians a position                              */
  int32_t rotary_dim;         /* r: the first r columns turn (even, 2 <= r <= d), the others are copied      */
  int32_t interleaved;        /* != 0: pair i is columns (2 i, 2 i + 1); 0: columns (i, i + r / 2)           */
  float magnitude;            /* m: factor of the turned columns                                           */
} attn_rotary_spec;

/* A [B,H,N,d] tensor and where its turned copy goes (y == x with the same strides: in place).  Strides in elements, multiples of 8, the d axis
 * contiguous; pointers 16-byte aligned.  x and y must not overlap otherwise, nor y and what the call's other tensor reads or writes. */
typedef struct {
  const void* x;
  void* y;
  int32_t H;
  int64_t x_stride_b, x_stride_h, x_stride_n;
  int64_t y_stride_b, y_stride_h, y_stride_n;
} attn_rotary_tensor;

typedef struct {
  int32_t B, N, d;             /* d in {16, 32, 64, 128} */
  int32_t dtype;
  attn_rotary_spec rotary;
  int32_t inverse;             /* != 0: by the negative angle (the gradient of the rotation) */
  const int32_t* positions;    /* device, [N] or [B, N]; NULL: 0 .. N - 1.  Any int32 value */
  int64_t position_stride_b;   /* elements from one batch entry to the next (0: all share one row) */
  void* stream;
} attn_rotary_params;

/*
 * Pair i of a row at position p turns by the angle p f_i:  y_a = m (x_a cos - x_b sin),  y_b = m (x_b cos + x_a sin).
 * One or two tensors (Q and K, which may differ in their number of heads) in one launch.  The angle is formed in
 * 64 bits and reduced to a turn before it is rounded: every int32 position is as exact as a near one.
 */
int attn_rotary(const attn_rotary_params* p, const attn_rotary_tensor* tensors, int32_t n_tensors);

/* The norm of every row of Q and K: y = w o x / sqrt(mean(x^2) + eps), with one vector of weights for all heads of a tensor. */
typedef struct {
  const void* q_weight;        /* device, [d]: of the first tensor of a call                                */
  const void* k_weight;        /* device, [d]: of the second                                                */
  int32_t weights_fp32;        /* != 0: float32, else of the tensors' dtype                                 */
  float eps;                   /* finite, > 0                                                               */
} attn_norm_spec;

/*
 * Every row normed, then turned as by attn_rotary, in one pass and with one rounding.  p->rotary.frequencies == NULL with rotary_dim 0: the norm alone.  p->inverse must be 0.
 * Sums are in 32 bits: a row whose squares add up beyond their range (elements near 10^18 in bf16) comes out as zeros.
 */
int attn_norm_rotary(const attn_rotary_params* p, const attn_norm_spec* norm, const attn_rotary_tensor* tensors, int32_t n_tensors);

/* A tensor of its backward pass: x as the forward call read it, dy the gradient of what that wrote, both in; dx and the weights' gradient dw ([d], of the weights' type, NULL: not
 * asked for) out.  Strides as in attn_rotary_tensor.  dx must not overlap what the call reads. */
typedef struct {
  const void* x;
  const void* dy;
  void* dx;
  void* dw;
  int32_t H;
  int64_t x_stride_b, x_stride_h, x_stride_n;
  int64_t dy_stride_b, dy_stride_h, dy_stride_n;
  int64_t dx_stride_b, dx_stride_h, dx_stride_n;
} attn_norm_grad;

/* Bytes of scratch for attn_norm_rotary_bwd at head dimension d; 0 if there is none such. */
size_t attn_norm_rotary_bwd_workspace_bytes(int32_t d);

/*
 * With g = dy turned back and h = g o w:  dx = r (h - x r^2 mean(h o x)),  dw = the sum over all rows of g o x r,  r = 1 / sqrt(mean(x^2) + eps).
 * p and norm as in the forward call.  workspace: 256-byte aligned, needed where a dw is asked for; contents on entry are ignored.  The same inputs give the same bits in every
 * call.  A finite row whose squares add up beyond 32 bits has no gradient, as it has come out as zeros: its dx is 0, and it adds nothing to dw.
 */
int attn_norm_rotary_bwd(const attn_rotary_params* p, const attn_norm_spec* norm, const attn_norm_grad* tensors, int32_t n_tensors, void* workspace,
                         size_t workspace_bytes);

/*
 * A batch of B sequences whose keys and values lie in the pages of a cache.
 *   caches         K and V: [pages, Hk, page_size, d], strides shared by both (multiples of 8 elements, d contiguous); page_stride and
 *                  row_stride * page_size below 2^31 elements
 *   block_table    device int32 [B, table_width]: entry t of row b is the page of positions t * page_size ...
 *   lengths        device int32 [B]: tokens of each sequence, the new ones included
 *   query_starts   device int32 [B + 1], rising: rows query_starts[b] .. query_starts[b + 1] - 1 of the token tensors [T, heads, d] are the
 *                  new tokens of sequence b, its last ones.  NULL: row b is the one new token of sequence b (then T >= B).
 *                  Rows of no sequence (behind the last, in a padded batch) are not read, and are left as they were in the outputs.
 *                  Starts that fall give unspecified outputs.
 * These three are read on the GPU only: a captured graph follows their contents.  Whatever they hold, nothing outside the tensors is
 * read or written: starts are forced into 0 .. T; a sequence has as many keys as its length says, but no more than a row of its table holds, table_width * page_size
 * (its new tokens keep the positions that its length gives them); and a page
 * number outside [0, pages) stands for a page of zeros that nothing is written to.  (Table entries behind a sequence's length are not used.)
 * What stands in the pages at positions < length must be finite; what stands behind is never used.
 */
typedef struct {
  int32_t B, T;
  int32_t Hq, Hk, d;           /* Hq a multiple of Hk: Q head h reads K head h / (Hq / Hk); d in {16, 32, 64, 128} */
  int32_t dtype;
  int32_t pages, page_size, table_width;   /* page_size: a power of two from 16 to 4096 */
  int32_t causal;              /* != 0: a new token sees its own position and those before it; 0: all positions < length */
  float softmax_scale;
  int64_t page_stride, head_stride, row_stride;   /* of the caches */
  int64_t table_stride;        /* elements between rows of the block table */
  int64_t q_stride_t, q_stride_h;      /* Q [T, Hq, d] */
  int64_t o_stride_t, o_stride_h;      /* O (attn_paged_append: the turned Q) */
  int64_t k_stride_t, k_stride_h, v_stride_t, v_stride_h;   /* new K and V [T, Hk, d] (attn_paged_append only) */
  const int32_t* block_table;
  const int32_t* lengths;
  const int32_t* query_starts;
  void* stream;
} attn_paged_params;

/*
 * Writes the new tokens' K and V rows into the pages, token i of the m new ones of sequence b at position lengths[b] - m + i (a position that is negative, or behind
 * the table's last page, is not written).  Where the table gives two tokens of a call the same row, every 16 bytes of it are one or the other's.  What is
 * written must not overlap what else the call reads or writes.  With rotary != NULL K is turned by its position, and so is Q, if one is given, into Qout (in place where
 * Qout == Q with the same strides).  rotary == NULL: K is copied; then Q must be NULL.
 */
int attn_paged_append(const attn_paged_params* p, const attn_rotary_spec* rotary, const void* K, const void* V, void* k_cache, void* v_cache, const void* Q,
                      void* Qout);

/* The same with Q and K normed first, Q with q_weight and K with k_weight (attn_norm_rotary).  rotary == NULL: the norm alone, of Q too if one is given. */
int attn_paged_norm_append(const attn_paged_params* p, const attn_rotary_spec* rotary, const attn_norm_spec* norm, const void* K, const void* V, void* k_cache,
                           void* v_cache, const void* Q, void* Qout);

/* Bytes of scratch for attn_paged_fwd with these params.  The head dimension alone decides: a workspace serves every call at its head dimension.  0 if the params
 * are invalid. */
size_t attn_paged_workspace_bytes(const attn_paged_params* p);

/*
 * O = softmax(tau Q K^T) V and its row statistic for the new tokens of every sequence over its pages.
 *   Q, O       [T, Hq, d] with strides of their own;   LSE  [Hq, T] float32, packed
 *   workspace  256-byte aligned, attn_paged_workspace_bytes(p); contents on entry are ignored, and calls that overlap in time must not share one
 * A row that sees no key (a sequence of length 0, a token whose position is negative) gets O = 0, LSE = -inf.  Results do not depend on timing: for the
 * same sizes and lengths they are the same in every call.
 */
int attn_paged_fwd(const attn_paged_params* p, const void* Q, const void* k_cache, const void* v_cache, void* O, float* LSE, void* workspace,
                   size_t workspace_bytes);

/*
 * The same with a sliding window (p->causal must be set): a new token at position i sees the keys at positions j <= i with i - j < window or j < sinks.  window >= 1, sinks >= 0.  Of a
 * sequence's pages only those are read that hold a key that one of its new tokens sees; the others may belong to another sequence by now, or their numbers be none.  Workspace as
 * for attn_paged_fwd.
 */
int attn_paged_window_fwd(const attn_paged_params* p, int32_t window, int32_t sinks, const void* Q, const void* k_cache, const void* v_cache, void* O, float* LSE,
                          void* workspace, size_t workspace_bytes);

/* Caches of one or more layers, [layers, pages, Hk, page_size, d]. */
typedef struct {
  int32_t layers, pages, Hk, page_size, d;
  int32_t dtype;
  int64_t layer_stride, page_stride, head_stride, row_stride;
  void* stream;
} attn_paged_copy_params;

/*
 * Copies whole pages, K and V, in all layers.  pairs: HOST memory, [n_pairs][2] (source, destination), read during the call.  All copies are
 * independent of their order: a page that is the destination of one copy and the source or the destination of another is
 * refused (ATTN_ERR_PAGES), as is a number outside [0, pages).  A source may be named any number of times.
 */
int attn_paged_copy(const attn_paged_copy_params* p, void* k_cache, void* v_cache, const int32_t* pairs, int64_t n_pairs);

/* Static, human-readable text for a status code. */
const char* attn_strerror(int status);

/* Library version: major * 10000 + minor * 100 + patch. */
int attn_version(void);

#ifdef __cplusplus
}
#endif
#endif /* ATTN_H_ */
