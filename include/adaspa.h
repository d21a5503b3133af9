/*
 * adaspa.h - C ABI of the AdaSpa attention hot path for AMD MI355X (gfx950).
 *
 * AdaSpa (arXiv 2502.21079) accelerates the 3D full attention of video
 * diffusion transformers with blockified sparse attention whose block pattern
 * is found by a precise online search that reuses log-sum-exp values across
 * denoising steps.  This library exposes the three operations of that path:
 *
 *   adaspa_dense_attn_lse     dense softmax attention + per-row LSE
 *                             (Sec. 2.2; first pass of Algorithm 1)
 *   adaspa_block_search       block attention mass W_sum_attn from a given
 *                             LSE (second pass of Algorithm 1 / Algorithm 2,
 *                             Sec. 4.1-4.2) and per-head block selection
 *                             (optimal sparse indices of Sec. 4.1, text sink
 *                             and row-wise uniform selection of Sec. 4.3)
 *   adaspa_block_sparse_attn  blockified sparse attention over the selected
 *                             key blocks (Sec. 4.1, bias form with c -> inf)
 *
 * and adaspa_fused_online_search, the first two in one call as Algorithm 1
 * describes them (dense attention + LSE, then the masses of the same rows),
 * and adaspa_single_pass_online_search, the same results with one pass over
 * Q K^T instead of two.
 *
 * Beside it stand the attentions of the prompt side, with their gradients:
 * adaspa_cross_attn (video tokens over a text encoder's states) and
 * adaspa_rel_bias_attn (the encoder's own, with a learned relative position
 * bias), rotary positions of queries and keys (adaspa_rotary), and a
 * key/value cache in 8 bits with the attention that reads it (adaspa_cache_*).  Their
 * tensors, strides and masks are described at their declarations; what is said
 * below of ownership, streams, errors and determinism holds for them too.
 *
 * Conventions shared by every call
 * --------------------------------
 *  - Tensors are DEVICE pointers, contiguous, 16-byte aligned.
 *    Q, K, V, O: bf16 [B, H, L, D] (D innermost).  LSE: fp32 [B, H, L],
 *    natural logarithm.  W_sum_attn: fp32 [B, H, NB, NB] with NB = ceil(L/Bs).
 *  - Block rows of the sparse pattern are numbered r = (b*H + h)*NB + p for
 *    query block p; the pattern is CSR: row_ptr int32 [B*H*NB + 1] and col_idx
 *    int32, key-block indices strictly ascending within a row.
 *  - A block is a TEXT block when its token range overlaps
 *    [text_start, text_start + text_len).
 *  - Ownership: the caller owns every buffer.  No call allocates device
 *    memory, keeps a pointer after it returns, or synchronises the device:
 *    each call validates its arguments on the host, enqueues kernels on
 *    `stream` (a hipStream_t; NULL means the default stream) and returns.
 *    Counters are cleared by kernels, not memsets, so a sequence of calls
 *    with caller-allocated outputs and workspaces can be captured in a HIP
 *    graph and replayed.
 *  - Results are deterministic: the same inputs and shape give the same bits.
 *    How a row's sums are split over waves follows the whole shape (B * H
 *    among it) and, for block-sparse attention, the whole pattern, so a
 *    (batch, head) pair computed in another batch or in a shard of the heads
 *    agrees within rounding.
 *  - Errors: invalid arguments are reported synchronously with a status code
 *    before anything is enqueued.  A failed launch returns ADASPA_ERR_HIP.
 *    A fault inside a kernel surfaces at the caller's next synchronisation.
 *  - Calls are stateless and may be issued from several host threads on
 *    different streams; calls that share an output buffer must be ordered by
 *    the caller.  (adaspa_block_sparse_attn_noalloc is the exception: its calls
 *    on one GPU share that GPU's counters and must not overlap.)
 */
#ifndef ADASPA_H_
#define ADASPA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  ADASPA_OK = 0,
  ADASPA_ERR_INVALID_ARG = 1,   /* null/misaligned pointer, bad size or range */
  ADASPA_ERR_UNSUPPORTED = 2,   /* head_dim or block outside what is built,
                                   L * D >= 2^30, or B * H >= 65536            */
  ADASPA_ERR_CAPACITY = 3,      /* col_idx capacity too small                 */
  ADASPA_ERR_WORKSPACE = 4,     /* workspace missing or too small             */
  ADASPA_ERR_HIP = 5            /* a HIP launch reported an error             */
} adaspa_status;

/* Shape of one attention call: B batches x H heads of L tokens with head
 * dimension D; square sparse blocks of Bs tokens.  Supported: D in {64, 128},
 * Bs in {64, 128}, L >= 1 (L need not be a multiple of Bs: the last block is
 * ragged and out-of-range keys never contribute), L * D < 2^30 and B * H <
 * 65536 (larger shapes return ADASPA_ERR_UNSUPPORTED).  softmax_scale <= 0 selects
 * 1/sqrt(D) (the attention-weights equation, Sec. 2.2). */
typedef struct {
  int32_t batch, heads, seqlen, head_dim;
  int32_t block;
  int32_t text_start, text_len;   /* text range for the text sink; len may be 0 */
  float softmax_scale;
} adaspa_problem;

/* Selection modes (Sec. 4.1 optimal sparse indices; Sec. 4.2 head-adaptive
 * sparsity; Sec. 4.3 row-wise uniform selection).  In every mode each video
 * query-block row of head h keeps the same count k_h of key blocks: text key
 * blocks first (text sink), then the remaining blocks by mass descending with
 * ties to the lower index.  Text query-block rows keep all NB blocks. */
enum {
  /* k_h = clamp(ceil(head_param_bp[h] * NB / 10000), max(1, #text blocks), NB) */
  ADASPA_SELECT_TOPK = 0,
  /* k_h = smallest count whose head Recall (Sec. 2.3, text rows counted as
   * fully kept) reaches head_param_bp[h] / 10000. */
  ADASPA_SELECT_COVERAGE = 1,
  /* Head-adaptive hierarchical sparsity (Sec. 4.2).  At base sparsity s
   * (base_sparsity_bp) every head keeps k(s) blocks per row; n = number of
   * heads whose Recall there exceeds recall_threshold_bp (strictly), capped at
   * floor(H/2).  The n heads of highest Recall (ties: lower head index) move
   * to sparsity (1+s)/2, the n of lowest Recall to (3s-1)/2 (at least 0);
   * k(x) is the TOPK count of keep fraction 1-x.  Heads are ranked within each
   * batch element; Recall is compared exactly.  head_param_bp is unused. */
  ADASPA_SELECT_HIERARCHICAL = 2
};

/* Flags */
enum {
  ADASPA_F_TEXT_SINK = 1,       /* force text blocks (Sec. 4.3); usually set   */
  ADASPA_F_SCORES_GIVEN = 2     /* block_mass is an INPUT: skip the mass pass  */
};

typedef struct {
  int32_t mode;                 /* ADASPA_SELECT_*                                */
  int32_t flags;                /* ADASPA_F_*                                     */
  const int32_t* head_param_bp; /* HOST array [H]: keep fraction (TOPK) or Recall
                                   target (COVERAGE) in basis points, 0..10000;
                                   applies to every batch element; may be NULL
                                   for HIERARCHICAL                              */
  int32_t base_sparsity_bp;     /* HIERARCHICAL: base sparsity s, 0..10000        */
  int32_t recall_threshold_bp;  /* HIERARCHICAL: Recall threshold, 0..10000       */
} adaspa_select;

/* Human-readable name of a status code (static storage). */
const char* adaspa_status_string(adaspa_status s);

/* Device bytes of the optional workspace of adaspa_dense_attn_lse (0 for
 * invalid arguments). */
size_t adaspa_dense_attn_workspace(const adaspa_problem* prob);

/* Dense attention with LSE (Sec. 2.2; Algorithm 1, first pass).
 *   out[b,h,i,:] = sum_j softmax_j(scale * q_i . k_j) v_j        bf16 (RNE)
 *   lse[b,h,i]   = log sum_j exp(scale * q_i . k_j)             fp32
 * q, k, v, out: bf16 [B,H,L,D]; lse: fp32 [B,H,L] (may be NULL to skip).
 * workspace (optional, caller-owned, 16-byte aligned, at least
 * adaspa_dense_attn_workspace() bytes, contents need not be initialised)
 * holds the counters of a work queue per XCD, so that the XCDs that run
 * faster take more of the work; with NULL, and where a launch is short (up to
 * 1,024 (head, 256-row tile) items), the work is split statically.  The
 * results are bitwise the same either way.  The call clears the counters
 * itself (with a kernel on `stream`); calls that may run concurrently need
 * separate workspaces.  ADASPA_ERR_WORKSPACE if it is too small or
 * misaligned. */
adaspa_status adaspa_dense_attn_lse(const adaspa_problem* prob, const void* q,
                                    const void* k, const void* v, void* out,
                                    float* lse, void* workspace,
                                    size_t workspace_bytes, void* stream);

/* Device bytes of workspace adaspa_block_search needs for this problem and
 * selection (0 for invalid arguments). */
size_t adaspa_block_search_workspace(const adaspa_problem* prob,
                                     const adaspa_select* sel);

/* Number of col_idx entries the selection may write: the exact count for
 * TOPK, an upper bound for HIERARCHICAL (every head at the largest of its
 * three counts), B*H*NB*NB for COVERAGE (the counts depend on the data and
 * the library never synchronises to learn them).  Returns -1 for invalid
 * arguments. */
int64_t adaspa_block_search_capacity(const adaspa_problem* prob,
                                     const adaspa_select* sel);

/* Block search (Sec. 4.1-4.3; Algorithm 1 second pass / Algorithm 2).
 *   1. Unless ADASPA_F_SCORES_GIVEN: block_mass[b,h,p,c] =
 *        sum_{i in block p} sum_{j in block c} exp(scale * q_i . k_j - lse[b,h,i])
 *      with the LSE given by the caller (fresh from adaspa_dense_attn_lse, or
 *      cached from an earlier step); no renormalisation.
 *   2. Per-head count k_h (see the modes) and per-row selection, emitted as CSR
 *      into row_ptr / col_idx.  head_k int32 [B,H] and head_recall fp32 [B,H]
 *      (the head Recall at k_h) are optional outputs (may be NULL).
 * Ranking compares fp32 masses (-0 == +0, NaN last).  Cumulative masses are
 * exact: each mass m >= 0 becomes min(round_half_even(m * 2^32), cap) with
 * cap = floor(2^62 / (NB*NB)) (NaN and m <= 0 give 0); coverage holds when
 * kept * 10000 >= total * tau_bp; recall = (float)((double)kept/(double)total),
 * 1 when total is 0.
 * Supported: NB <= 8192 key blocks, H <= 512 heads and B*H*NB*NB < 2^31
 * (ADASPA_ERR_UNSUPPORTED otherwise).
 * q, k, lse may be NULL with ADASPA_F_SCORES_GIVEN.  col_capacity must be at
 * least adaspa_block_search_capacity(); workspace must hold
 * adaspa_block_search_workspace() bytes, 256-byte aligned. */
adaspa_status adaspa_block_search(const adaspa_problem* prob, const void* q,
                                  const void* k, const float* lse,
                                  const adaspa_select* sel, float* block_mass,
                                  int32_t* row_ptr, int32_t* col_idx,
                                  int64_t col_capacity, int32_t* head_k,
                                  float* head_recall, void* workspace,
                                  size_t workspace_bytes, void* stream);

/* Fused online search (Algorithm 1, Sec. 4.2): dense attention with LSE and
 * the block masses of that fresh LSE in ONE kernel, then the selection.  Each
 * workgroup computes the output and LSE of 256 query rows (first pass) and
 * then the block masses of the same rows (second pass) while their Q and LSE
 * are still in registers, so Q is read once and the LSE is not read back.
 * Where dense attention splits rows' keys over waves (B * H * ceil(L / 64) up
 * to 512, or a few items past a multiple of 256), the two passes are kernels
 * of their own.  It produces exactly (bit for bit) what
 * adaspa_dense_attn_lse followed by adaspa_block_search with that LSE
 * produces:
 *   out, lse          as adaspa_dense_attn_lse (lse may be NULL: the masses
 *                     still use the fresh LSE)
 *   block_mass, row_ptr, col_idx, head_k, head_recall
 *                     as adaspa_block_search (ADASPA_F_SCORES_GIVEN is not
 *                     allowed: ADASPA_ERR_INVALID_ARG)
 * The workspace, its size (adaspa_block_search_workspace), the capacity
 * rule, the alignment rules and the errors are those of the two calls; the
 * workspace also holds the per-XCD work-queue counters of the fused kernel,
 * which the call clears itself. */
adaspa_status adaspa_fused_online_search(const adaspa_problem* prob, const void* q,
                                         const void* k, const void* v, void* out,
                                         float* lse, const adaspa_select* sel,
                                         float* block_mass, int32_t* row_ptr,
                                         int32_t* col_idx, int64_t col_capacity,
                                         int32_t* head_k, float* head_recall,
                                         void* workspace, size_t workspace_bytes,
                                         void* stream);

/* Device bytes of the workspace of adaspa_single_pass_online_search: the
 * workspace of adaspa_block_search plus B*H*NB*L floats of per-row block
 * masses (NB = ceil(L/Bs); 9.1 GB for B=1, H=24, L=110,336, Bs=128), rounded
 * up to 256 bytes.  0 for invalid arguments or ADASPA_F_SCORES_GIVEN. */
size_t adaspa_single_pass_online_search_workspace(const adaspa_problem* prob,
                                                  const adaspa_select* sel);

/* The least workspace adaspa_single_pass_online_search accepts: the
 * search's workspace plus the per-row block masses and row LSEs of ONE
 * (batch, head) pair (NB*L + L floats), each part rounded up to 256 bytes.
 * Given less than adaspa_single_pass_online_search_workspace() but at least
 * this, the call runs the attention pass over groups of as many (batch,
 * head) pairs as fit, one after another, then the selection of all of them;
 * the results are the same as with the full workspace.  0 for invalid
 * arguments or ADASPA_F_SCORES_GIVEN. */
size_t adaspa_single_pass_online_search_min_workspace(const adaspa_problem* prob,
                                                      const adaspa_select* sel);

/* Single-pass online search (Algorithm 1, Sec. 4.1-4.2, with one pass over
 * Q K^T): the outputs of adaspa_fused_online_search, computed differently.
 * The block mass W[p][c] is the sum over rows i of p of exp(s_ij - LSE_i)
 * over the keys j of c.  The attention pass already forms
 * exp(s_ij - m_i) for its softmax (m_i the row's running reference), so it
 * also adds those terms per (row, key block) in fp32 and keeps
 * log2 of each sum plus m_i in the workspace; once a row's LSE is known the
 * kernel turns them into the row's shares exp(y - LSE_i) and sums them over
 * the rows of each query block.  The second recomputation of Q K^T that the
 * two-pass form needs is not taken.
 *   out, lse          bit for bit those of adaspa_dense_attn_lse (lse may be
 *                     NULL: the masses still use the fresh LSE)
 *   block_mass        the masses of the fresh LSE, within 1e-3 relative of
 *                     the exact values.  They are normalised by the LSE of
 *                     the unrounded fp32 row sum; the stored lse normalises
 *                     the bf16-rounded weights of the output, so
 *                     adaspa_block_search given that lse returns masses
 *                     that differ from these by up to 2^-9 relative
 *   row_ptr, col_idx, head_k, head_recall
 *                     the selection of those masses, as adaspa_block_search
 *                     (ADASPA_F_SCORES_GIVEN is not allowed:
 *                     ADASPA_ERR_INVALID_ARG)
 * workspace must hold at least adaspa_single_pass_online_search_min_workspace()
 * bytes, 256-byte aligned (ADASPA_ERR_WORKSPACE otherwise); with
 * adaspa_single_pass_online_search_workspace() bytes all (batch, head) pairs
 * run together.  It holds the selection's scratch, the per-XCD work-queue
 * counters (cleared by the call) and the per-row block masses, and its
 * contents need not be kept between calls.  Capacity, alignment and the other
 * errors as adaspa_block_search. */
adaspa_status adaspa_single_pass_online_search(const adaspa_problem* prob, const void* q,
                                               const void* k, const void* v, void* out,
                                               float* lse, const adaspa_select* sel,
                                               float* block_mass, int32_t* row_ptr,
                                               int32_t* col_idx, int64_t col_capacity,
                                               int32_t* head_k, float* head_recall,
                                               void* workspace, size_t workspace_bytes,
                                               void* stream);

/* Device bytes of the optional workspace of adaspa_block_sparse_attn (0 for
 * invalid arguments). */
size_t adaspa_block_sparse_attn_workspace(const adaspa_problem* prob);

/* Blockified sparse attention (Sec. 4.1, bias -c(1-M) with c -> inf).
 *   out[b,h,i,:] = sum_{j in kept(p(i))} exp(scale*q_i.k_j - lseM_i) v_j
 *   lseM[b,h,i]  = log sum_{j in kept(p(i))} exp(scale * q_i . k_j)
 * where kept(p) are the key blocks col_idx[row_ptr[r] .. row_ptr[r+1]) of
 * row r = (b*H+h)*NB + p.  A row that keeps nothing gives out = 0 and
 * lseM = -inf.  Keeping every block reproduces adaspa_dense_attn_lse bit for
 * bit (both visit a row's keys in the same order and split the same rows over
 * waves).  lse_out may be NULL.  col_count is
 * the number of readable col_idx entries: row bounds are clamped to
 * [0, col_count] and entries outside [0, NB) are skipped, so malformed
 * patterns never read out of bounds.  Rows should be strictly ascending
 * (a repeated block would be counted twice).  prob->text_start/text_len only
 * schedule the work (the text query blocks, which keep every key block under
 * the text sink, are started first, and fewer workgroups share a CU with them)
 * and name the block every row is expected to begin with (its first tiles are
 * loaded before the row's indices are read, and reloaded if the row begins
 * elsewhere).  The results depend on neither them nor col_count beyond the
 * pattern's last entry.
 * Block 64 supports NB <= 8192 key blocks (ADASPA_ERR_UNSUPPORTED otherwise).
 * workspace (optional, caller-owned, 16-byte aligned, at least
 * adaspa_block_sparse_attn_workspace() bytes, contents need not be
 * initialised) holds per-XCD work-queue counters: in launches of more than a
 * few rounds of workgroups the last tenth of the query blocks then goes to the
 * XCDs that run ahead; with NULL all work is split statically.  The results
 * are bitwise the same either way.  The call clears
 * the counters itself (with a kernel on `stream`); calls that may run
 * concurrently need separate workspaces.  ADASPA_ERR_WORKSPACE if it is too
 * small or misaligned. */
adaspa_status adaspa_block_sparse_attn(const adaspa_problem* prob, const void* q,
                                       const void* k, const void* v,
                                       const int32_t* row_ptr,
                                       const int32_t* col_idx, int64_t col_count,
                                       void* out, float* lse_out, void* workspace,
                                       size_t workspace_bytes, void* stream);

/* adaspa_block_sparse_attn without a workspace argument and without any
 * allocation, for callers that cannot allocate device memory (code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc).  It
 * computes exactly what adaspa_block_sparse_attn computes with a workspace
 * (bitwise the same outputs) and takes the same arguments and checks, except
 * that the per-XCD work-queue counters live in a 256-byte array inside the
 * library, one per GPU, held from the library's load until the process ends.
 * The current device must be the one `stream` belongs to.  Every call on a
 * GPU shares that GPU's counters (the call clears them itself with a kernel
 * on `stream`), so calls on one GPU must not overlap: issue them on one
 * stream, or order them; overlapping calls race on the counters.  Returns
 * ADASPA_ERR_WORKSPACE if a problem ever needed more than the 256 bytes (no
 * supported problem does) and ADASPA_ERR_HIP if the array's device address
 * cannot be obtained.  No hipMalloc, hipFree or allocating library routine is
 * called. */
adaspa_status adaspa_block_sparse_attn_noalloc(const adaspa_problem* prob, const void* q,
                                               const void* k, const void* v,
                                               const int32_t* row_ptr,
                                               const int32_t* col_idx, int64_t col_count,
                                               void* out, float* lse_out, void* stream);

/* ---------------------------------------------------------------------------
 * The prompt side: attention of queries over keys of another length (cross
 * attention to an encoder's states), and attention with a learned relative
 * position bias by buckets (the encoder's own), each with its backward pass.
 *
 *   out_i = sum_j exp(S_ij - lse_i) v_j     lse_i = log sum_j exp(S_ij)
 *   S_ij  = scale * q_i . k_j  (+ table[bucket(j - i - offset), h])
 *
 * over the visible keys: j < key_lens[b], key_mask[b, j] != 0 and, with
 * `causal`, j <= i + offset.  A row that sees no key (a dropped prompt) gives
 * out = 0, lse = -inf and no gradient.  Whatever keys past key_lens or with a
 * 0 in key_mask hold, infinities and NaN too, takes no part; keys that only
 * the order hides from a row must be finite, as those that it sees.
 *
 * Tensors are bf16 or fp16 views [B, heads, tokens, D], D contiguous, with
 * strides of their own (elements; multiples of 8, the token stride below 2^23;
 * 16-byte aligned data), so a projection's output is read as it lies and a
 * batch stride of 0 reads one encoder state for every sample.  Outputs must
 * not overlap themselves.  H query heads share Hk key heads, H % Hk == 0, in
 * runs of H / Hk.  Lengths may be 0.  lse: fp32 [B, H, Lq], contiguous.
 * Scores, softmax, sums and gradients are accumulated in fp32; the weights and
 * dS are rounded to the inputs' type for the second products, results once.  In
 * fp16 both are rounded times powers of two that are taken back in fp32, so that
 * neither many keys nor small or large output gradients cost bits.
 * The workspace is scratch, 256-byte aligned, of the size that the matching
 * _workspace call names (0: invalid arguments; 16: the call takes none, NULL
 * will do), not shared by calls that may overlap.  Ownership, streams, errors and
 * determinism are those above: every sum over more than one workgroup is taken
 * in a fixed order. */
enum { ADASPA_BF16 = 0, ADASPA_FP16 = 1 };

typedef struct {
  int32_t batch, heads, kv_heads, q_len, k_len, head_dim;   /* D in {64, 128} */
  int32_t dtype;                  /* ADASPA_BF16 / ADASPA_FP16, of every tensor */
  float softmax_scale;            /* <= 0 selects 1/sqrt(D) */
  /* (batch, head, token) strides in elements; the last four are read by the
   * backward calls only. */
  int64_t q_stride[3], k_stride[3], v_stride[3], out_stride[3];
  int64_t dout_stride[3], dq_stride[3], dk_stride[3], dv_stride[3];
  int64_t key_mask_stride;        /* between the mask's rows, in bytes */
} adaspa_cross_problem;

/* Buckets of the distance between a key and a query.  Bucket m of a direction
 * holds the distances [bucket_start[m], bucket_start[m+1]) (none where the two are
 * equal), the last one all from its start on.  Bidirectional: the first half of the table is for keys
 * at or before the query, the second for keys after it; otherwise keys after
 * the query have distance 0.  A value past -2.3e38 (log2(e) times it leaves fp32)
 * counts as minus infinity and hides its keys; where a row sees nothing but values of
 * a large magnitude, its scores and lse hold 2^-24 of that. */
typedef struct {
  int32_t num_buckets;            /* rows of the table, [num_buckets, H]; at most 256 a direction */
  int32_t bidirectional;
  const int32_t* bucket_start;    /* HOST array of num_buckets / 2 (bidirectional) or num_buckets
                                     distances, ascending from 0, the last at most 1024 */
  int32_t causal;                 /* keys after the query are masked */
  int32_t q_offset;               /* position of query 0 among the keys, |q_offset| < 2^28 */
  int32_t queries_at_end;         /* instead: the queries are their sample's last positions,
                                     offset = key_lens[b] - Lq (decoding with a cache) */
  int32_t table_fp32;             /* the table and its gradient are fp32 (else the tensors' type) */
} adaspa_rel_bias;

/* Cross attention.  key_lens: device int32 [B] or NULL (every key), clamped to
 * [0, Lk]; key_mask: device bytes [B, Lk] (0 = masked) or NULL; lse may be
 * NULL. */
size_t adaspa_cross_attn_workspace(const adaspa_cross_problem* prob);
adaspa_status adaspa_cross_attn(const adaspa_cross_problem* prob, const void* q, const void* k,
                                const void* v, const int32_t* key_lens,
                                const uint8_t* key_mask, void* out, float* lse, void* workspace,
                                size_t workspace_bytes, void* stream);

/* Its backward pass: dq [B, H, Lq, D], dk and dv [B, Hk, Lk, D] (summed over
 * the query heads that share a key head; 0 for masked keys) from the output's
 * gradient and the forward call's out and lse. */
size_t adaspa_cross_attn_bwd_workspace(const adaspa_cross_problem* prob);
adaspa_status adaspa_cross_attn_bwd(const adaspa_cross_problem* prob, const void* dout,
                                    const void* q, const void* k, const void* v,
                                    const int32_t* key_lens, const uint8_t* key_mask,
                                    const void* out, const float* lse, void* dq, void* dk,
                                    void* dv, void* workspace, size_t workspace_bytes,
                                    void* stream);

/* Attention with a learned relative position bias: the bias is added from the
 * table inside the kernels and never written out. */
size_t adaspa_rel_bias_attn_workspace(const adaspa_cross_problem* prob,
                                      const adaspa_rel_bias* bias);
adaspa_status adaspa_rel_bias_attn(const adaspa_cross_problem* prob, const adaspa_rel_bias* bias,
                                   const void* q, const void* k, const void* v, const void* table,
                                   const int32_t* key_lens, const uint8_t* key_mask, void* out,
                                   float* lse, void* workspace, size_t workspace_bytes,
                                   void* stream);

/* Its backward pass; dtable [num_buckets, H] is the sum of dS over samples and
 * over the pairs of each bucket, in fp32, rounded once to the table's type. */
size_t adaspa_rel_bias_attn_bwd_workspace(const adaspa_cross_problem* prob,
                                          const adaspa_rel_bias* bias);
adaspa_status adaspa_rel_bias_attn_bwd(const adaspa_cross_problem* prob,
                                       const adaspa_rel_bias* bias, const void* dout,
                                       const void* q, const void* k, const void* v,
                                       const void* table, const int32_t* key_lens,
                                       const uint8_t* key_mask, const void* out, const float* lse,
                                       void* dq, void* dk, void* dv, void* dtable,
                                       void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Rotary positions of queries and keys, in one call.  Pair i of a head, (u, w), becomes
 *
 *   magnitude * (u cos a - w sin a, u sin a + w cos a),   a = position * freq[i],
 *
 * the elements behind the `pairs` pairs are copied.  The position of token t of
 * sample b is positions[b, t, axis] (without positions, on one axis: t) plus `offset`,
 * plus offsets[b] where that is given; the pairs go by the axes in turn,
 * axis_pairs[a] by axis a.  Angles are formed in fp64, products in fp32, results
 * rounded once.
 *
 * Tensors are bf16 or fp16 views [B, heads, len, D] as those of the prompt side
 * (D contiguous, strides multiples of 8, 16-byte aligned data), D a multiple of 8 up to
 * 256.  kv_heads may be 0 (no keys: k and k_out are not read).  An output may
 * be its input, at the same strides; other overlaps are not allowed, nor is an output
 * that overlaps itself. */
enum { ADASPA_ROTARY_HALF = 0,           /* pair i: elements i and i + pairs */
       ADASPA_ROTARY_INTERLEAVED = 1 };  /* elements 2 i and 2 i + 1 */

typedef struct {
  int32_t batch, heads, kv_heads, len, head_dim;
  int32_t dtype;                  /* ADASPA_BF16 / ADASPA_FP16 */
  int32_t pairs;                  /* 1 to D / 2 */
  int32_t layout;                 /* ADASPA_ROTARY_* */
  int32_t axes;                   /* 1 to 4 */
  int32_t axis_pairs[4];          /* pairs of each axis, `pairs` in all */
  float magnitude;
  const double* freq;             /* HOST array [pairs], radians per position */
  /* (batch, head, token) strides in elements */
  int64_t q_stride[3], k_stride[3], q_out_stride[3], k_out_stride[3];
  int64_t position_stride[2];     /* (batch, token) strides of positions; axes lie side by side */
} adaspa_rotary_problem;

/* positions: device int32 or NULL; offset: below 2^40 in magnitude; offsets:
 * device int32 [B] or NULL. */
adaspa_status adaspa_rotary(const adaspa_rotary_problem* prob, const void* q, const void* k,
                            const int32_t* positions, int64_t offset, const int32_t* offsets,
                            void* q_out, void* k_out, void* stream);

/* Its backward pass: the results' gradients turned the other way, by the same
 * magnitude.  The strides of q and k are those of the given gradients, q_out's and
 * k_out's those of dq and dk. */
adaspa_status adaspa_rotary_bwd(const adaspa_rotary_problem* prob, const void* dq_out,
                                const void* dk_out, const int32_t* positions, int64_t offset,
                                const int32_t* offsets, void* dq, void* dk, void* stream);

/* ---------------------------------------------------------------------------
 * A key/value cache in 8 bits: a pool of pages, each `page` tokens of one sequence
 * for every key head.
 *
 *   k        e4m3 (OCP) [pages, Hk, page, D]
 *   v        e4m3 [pages, Hk, page / 16, D, 16]: sixteen tokens of a channel side by
 *            side, the order in which attention takes them
 *   k_scale, v_scale   fp32 [pages, Hk], powers of two (2^-126 to 2^127): a value is its
 *            code times its page's and head's scale
 *   page_table         int32 [B, max_pages] (row stride table_stride): the pages of each
 *            sequence in order.  Entries outside [0, pages) name no page: what would be
 *            written there is dropped, what would be read there is not there.
 *
 * All are device memory of the caller's; k and v 16-byte aligned.  New keys and values,
 * queries and outputs are bf16 or fp16 views [B, heads, len, D] as those of the prompt
 * side (D in {64, 128}, strides multiples of 8, 16-byte aligned data, outputs that do not
 * overlap themselves).  H query heads share Hk key heads in runs; read and write have
 * H = Hk.  Lengths are device int32 [B]. */
typedef struct {
  void *k, *v;
  float *k_scale, *v_scale;
  const int32_t* page_table;
} adaspa_cache;

typedef struct {
  int32_t batch, heads, kv_heads;
  int32_t len;                    /* new tokens, rows to read, or queries, of a sample */
  int32_t head_dim, dtype;        /* ADASPA_BF16 / ADASPA_FP16 */
  int32_t pages, page, max_pages; /* page in {16, 32, 64, 128}; max_pages * page < 2^28 */
  int32_t causal;                 /* attention: a query sees the tokens up to its own place */
  float softmax_scale;            /* attention: <= 0 selects 1/sqrt(D) */
  int64_t table_stride;
  /* (batch, head, token) strides in elements; attention reads the first two, read and
   * write the last two */
  int64_t q_stride[3], out_stride[3], k_stride[3], v_stride[3];
} adaspa_cache_problem;

/* Quantises k and v [B, Hk, len, D] into the pages behind the lens[b] tokens that a
 * sequence has; new_lens (may be NULL: len) leaves sample b its first new_lens[b] tokens.
 * A page and head gets the least power of two s >= 2^-126 with amax <= 448 s over the
 * finite values, values the nearest code, ties to even; infinities and NaN are kept as NaN.  A
 * page that holds tokens before lens[b] keeps the larger of its scale and the new tokens', and
 * where that grows their codes are brought to it.  What lies behind the last token stays as it
 * was.  A sample with lens[b] < 0 is left out; one without new tokens writes nothing, whatever
 * pages the table names for it.  No two sequences may write the same page. */
adaspa_status adaspa_cache_write(const adaspa_cache_problem* prob, const adaspa_cache* cache,
                                 const void* k, const void* v, const int32_t* lens,
                                 const int32_t* new_lens, void* stream);

/* Rows t of k and v [B, Hk, len, D] are the tokens at positions starts[b] + t (starts may be
 * NULL: t) of sequences of lens[b] tokens; rows that are no token's are zeros.  k and v must
 * not overlap. */
adaspa_status adaspa_cache_read(const adaspa_cache_problem* prob, const adaspa_cache* cache,
                                const int32_t* lens, const int32_t* starts, void* k, void* v,
                                void* stream);

/* Attention of q [B, H, len, D] over the first lens[b] tokens of each sequence (clamped to
 * [0, max_pages * page]):
 *   out_i = sum_j exp(S_ij - lse_i) v_j,  lse_i = log sum_j exp(S_ij),  S_ij = scale q_i . k_j
 * The queries are their sequence's last tokens: sample b has q_lens[b] of them (NULL: len;
 * clamped to [0, len]), query i stands at lens[b] - q_lens[b] + i and, with `causal`, sees no
 * token behind that.  Rows without a token, and those from q_lens[b] on, give 0 and -inf.  What lies
 * behind lens[b], on pages that are not there, or in queries from q_lens[b] on takes no part,
 * infinities and NaN too; tokens that only the order hides from a row must be finite.  lse:
 * fp32 [B, H, len] or NULL.  The workspace is that of the prompt side's calls: scratch, 256-byte
 * aligned, of the size that the _workspace call names for the same problem, `causal` included. */
size_t adaspa_cache_attn_workspace(const adaspa_cache_problem* prob);
adaspa_status adaspa_cache_attn(const adaspa_cache_problem* prob, const adaspa_cache* cache,
                                const void* q, const int32_t* lens, const int32_t* q_lens, void* out,
                                float* lse, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* ADASPA_H_ */
