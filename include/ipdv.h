/*
 * ipdv.h -- C ABI of the verifier-side window scoring library (libipdv.so)
 * for AMD Instinct MI355X (gfx950).
 *
 * The entry points are the verifier's calls in one propose-and-verify
 * step of Interactive-Policy Distillation (Section 3.2.3, "Fused Inference
 * Engine", and Eq. (9)):
 *
 *   verify_attn_paged        -- the verification stage's attention: append the
 *                               proposer's window to the verifier's own paged
 *                               KV cache and score every window row in one
 *                               prefill pass over the resident prefix;
 *   lmhead_logsoftmax_verify -- the verifier's next-token distribution at each
 *                               window row (LM head + log-softmax at
 *                               temperature 1): proposal log-prob, LSE, argmax,
 *                               top-K support (Eq. (5)) and entropy;
 *   accept_scan              -- the verdict stage: the top-K coverage rule of
 *                               Eq. (9) applied as a first-event scan over each
 *                               window, with the EOS and length rules and the
 *                               rollback length shared by both caches;
 *   accept_scan_rule         -- the same scan with the rule variants named
 *                               after Eq. (9) (entropy thresholds, asymmetric
 *                               rules, SKD's fixed one-token handback);
 *   sample_takeover          -- the teacher's replacement token at each
 *                               takeover (Eq. (9), second case), drawn from
 *                               the verifier's distribution at that row;
 *   lmhead_sample            -- the proposer's per-row draw (temperature 1)
 *                               from the same records;
 *   lmhead_pack_w            -- W repacked once into 1 KB blocks (optional
 *                               layout for the calls that read W);
 *   lmhead_logp_gather       -- a model's log-probs at listed vocabulary
 *                               indices (the other model's top-K), which
 *                               complete the union support of Eq. (6);
 *   source_split_kl          -- the per-position values of the source-split
 *                               objective (Eqs. (6), (10), (11));
 *   rope_window              -- rotary positions of a window's queries and keys
 *                               (and their gradient);
 *   kv_append_q8, kv_read_q8 -- the window quantised into an 8-bit paged cache,
 *                               and cached rows read back;
 *   verify_attn_q8           -- the verification stage's attention over the
 *                               8-bit cache;
 *   sample_logits            -- a draw per row from logits, filtered by
 *                               temperature, top-k, top-p and min-p;
 *   verify_attn_masked       -- the verification stage's attention with capped
 *                               scores, a distance bias, sliding windows and
 *                               ranges of keys per row;
 *   attn_mass, kv_evict      -- the attention weight that each cached key gathers,
 *                               and the cache cut to the keys of the largest;
 *   verify_drafts            -- the verdict on drafts by both models' probabilities,
 *                               with the replacement drawn from what is left.
 *
 * Conventions common to every entry point:
 *   - All array arguments are DEVICE pointers owned by the caller (except the
 *     host-side shape arguments of the *_workspace_size queries).  The library
 *     allocates no device memory and keeps no state besides a thread-local
 *     error message and the optional thread-local timing hook below.
 *   - Every call only enqueues work on `hip_stream` (a hipStream_t; NULL = the
 *     default stream) and returns; it never synchronises.
 *   - Arrays are dense, row-major, with the shapes given below.  Floating
 *     inputs are IPDV_F32 (float) or IPDV_BF16 (bfloat16) as `dtype` says;
 *     arithmetic accumulates in fp32.
 *   - Return value: IPDV_OK, or a negative ipdv_status when host-side
 *     validation fails (nothing is launched) or a HIP launch fails.
 *     ipdv_last_error() then describes the failure.  Nothing is printed and
 *     nothing aborts.
 *   - Device data that break the documented contract (page ids, lengths that
 *     do not fit the page table) give unspecified outputs; the kernels clamp
 *     every index they read so that no access leaves the caller's buffers.
 *
 * Window convention.  Sequence b has L_b = ctx_lens[b] tokens in this
 * verifier's cache and k_b = cu_q[b+1] - cu_q[b] window rows.  Row i
 * (0 <= i < k_b, batch row cu_q[b] + i) is the token at absolute position
 * L_b + i; its output distribution predicts position L_b + i + 1 and scores
 * proposed token prop_tok[cu_q[b] + i].
 */
#ifndef IPDV_H
#define IPDV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  IPDV_OK = 0,
  IPDV_EINVAL = -1,        /* null required pointer or out-of-range argument  */
  IPDV_EUNSUPPORTED = -2,  /* a shape / dtype combination not implemented      */
  IPDV_EWORKSPACE = -3,    /* workspace null or smaller than the size query    */
  IPDV_EHIP = -4           /* a HIP launch or runtime call failed              */
} ipdv_status;

typedef enum { IPDV_F32 = 0, IPDV_BF16 = 1 } ipdv_dtype;

/* OR'ed into the `dtype` argument of the calls that read the LM-head weight
 * W (lmhead_logsoftmax_verify, sample_takeover, lmhead_sample,
 * lmhead_logp_gather): W is in the tiled layout written by lmhead_pack_w
 * instead of row-major [V, Hd].  bf16 only.  Results are bit-identical to the
 * row-major call; the GEMM's operand loads then read whole cache lines. */
#define IPDV_W_TILED 0x10

/* Driver codes (accept_scan): who proposed the window. */
#define IPDV_DRIVER_S 0   /* the student drives; the teacher verifies */
#define IPDV_DRIVER_T 1   /* the teacher drives; the student verifies */

/* Takeover and handback rules (accept_scan_rule), Section 3.2.1 after
 * Eq. (9): top-K coverage is the paper's rule for both; an entropy threshold
 * may replace either test, and the two may differ.  SKD is coverage takeover
 * with a fixed one-token handback. */
#define IPDV_TAKE_COVERAGE 0   /* take over when the draft is outside the verifier's top-K */
#define IPDV_TAKE_ENTROPY 1    /* take over when ent[row] > tau_take */
#define IPDV_HAND_COVERAGE 0   /* hand back when the draft is inside the verifier's top-K */
#define IPDV_HAND_FIXED_ONE 1  /* the teacher emits one token, then hands back (SKD) */
#define IPDV_HAND_ENTROPY 2    /* hand back when ent[row] <= tau_hand */

/* Distillation support S_t (source_split_kl), Eq. (5) and the text after
 * it; the union is the paper's default (Appendix B.2). */
#define IPDV_SUPPORT_UNION 0
#define IPDV_SUPPORT_STUDENT 1
#define IPDV_SUPPORT_TEACHER 2
#define IPDV_SUPPORT_INTERSECTION 3

/* KL direction per token source (source_split_kl): Eq. (10) is the default;
 * Section 4.3 ablates the other three. */
#define IPDV_LOSS_IPD_SPLIT 0      /* reverse KL where src = S, forward where src = T */
#define IPDV_LOSS_PURE_REVERSE 1
#define IPDV_LOSS_PURE_FORWARD 2
#define IPDV_LOSS_INVERSE_SPLIT 3  /* forward KL where src = S, reverse where src = T */

/* Largest index list per row of lmhead_logp_gather. */
#define IPDV_MAX_GATHER 64

/* Source labels (accept_scan `src`). */
#define IPDV_SRC_S 0
#define IPDV_SRC_T 1
#define IPDV_SRC_DISCARDED 255

/* Largest supported top-K (the paper sweeps K in {4, 8, 16, 32}). */
#define IPDV_MAX_K 32

/*
 * Workspace bytes verify_attn_paged needs for these host-side shape values
 * (0 if the arguments are invalid).  max_q is an upper bound of k_b over the
 * sequences of the call; max_pages_per_seq and page_size as passed to
 * verify_attn_paged.
 */
size_t ipdv_attn_workspace_size(int n_seq, int Hq, int Hkv, int D, int max_q,
                                int max_pages_per_seq, int page_size);

/*
 * verify_attn_paged -- verification-stage attention over the paged cache
 * (Section 3.2.3: the verifier evaluates all unverified drafts of its
 * sub-batch in one prefill pass, computing only the newly appended tokens
 * while the prefix cache stays resident; the proposer's tokens are appended
 * to the verifier's live cache).
 *
 * For every handled sequence b and window row i, in place:
 *   1. append: k_cache/v_cache at position L_b + i  <-  k_new/v_new[cu_q[b]+i];
 *   2. attend: for query head h and KV head g = h / (Hq/Hkv),
 *        out[cu_q[b]+i, h, :] = softmax_j( scale * q[cu_q[b]+i, h, :] . K_j )
 *                               . V_j   over keys j = 0 .. L_b + i (inclusive).
 * Q and K are taken as already position-encoded; no other mask or softcap.
 *
 * q       [T, Hq, D]    window queries (dtype)
 * k_new   [T, Hkv, D]   window keys    (dtype)
 * v_new   [T, Hkv, D]   window values  (dtype)
 * k_cache [num_pages, Hkv, D/32, page_size, 32]
 *                       key pages: per KV head and 32-channel slice, the
 *                       slice of each slot in turn (channel d of a slot at
 *                       [page][g][d/32][slot][d%32]); 16-key MFMA operand
 *                       loads then read whole cache lines (dtype, in/out)
 * v_cache [num_pages, Hkv, D, page_size]   value pages, channel-major: per
 *                                          KV head and channel, one value per
 *                                          slot (dtype, in/out)
 * page_table [B, max_pages_per_seq] int32  pages of sequence b in order;
 *                                          position p lives in page
 *                                          page_table[b][p / page_size], slot
 *                                          p % page_size.  Entries up to
 *                                          (L_b + k_b - 1) / page_size must be
 *                                          valid page ids < num_pages.
 * ctx_lens [B] int32    L_b (>= 0)
 * cu_q    [B+1] int32   window row offsets (non-decreasing, cu_q[0] = 0 for the
 *                       batch; T = cu_q[B])
 * seq_ids [n_seq] int32 the sequences this call handles (the verifier's
 *                       sub-batch, Section 3.2.3 groups requests by verifier);
 *                       NULL = sequences 0 .. n_seq-1.  Rows of other
 *                       sequences are neither read nor written.
 * max_q                 >= k_b for every handled sequence (host-side bound)
 * out     [T, Hq, D]    attention output (dtype)
 * Hq, Hkv, D            Hq % Hkv == 0; D in {64, 128} for bf16, D = 64 for fp32
 * page_size             16, 32 or 64
 * scale                 softmax scale, > 0 (normally 1/sqrt(D))
 * workspace             device buffer of >= ipdv_attn_workspace_size(...)
 *                       bytes (split-KV partial results); contents on entry
 *                       are ignored.
 *
 * Errors: IPDV_EINVAL (null pointer, n_seq < 0, max_q < 1, bad head counts,
 * scale not positive and finite), IPDV_EUNSUPPORTED (D, page_size, dtype),
 * IPDV_EWORKSPACE, IPDV_EHIP.
 */
int verify_attn_paged(const void* q, const void* k_new, const void* v_new,
                      void* k_cache, void* v_cache,
                      const int32_t* page_table, int max_pages_per_seq,
                      const int32_t* ctx_lens, const int32_t* cu_q,
                      const int32_t* seq_ids, int n_seq, int max_q,
                      void* out,
                      int Hq, int Hkv, int D, int page_size, int num_pages, float scale,
                      int dtype, void* workspace, size_t workspace_bytes,
                      void* hip_stream);

/*
 * ipdv_check_page_table -- host-side check of the device-data contract of
 * verify_attn_paged (the kernels clamp every index they read, so a table
 * that breaks the contract gives wrong outputs, not faults).  Takes HOST
 * copies of the call's arrays (page_table [B, max_pages_per_seq], ctx_lens
 * [B], cu_q [B+1], seq_ids [n_seq] or NULL) and checks, for every handled
 * sequence b:
 *   - L_b >= 0 and k_b = cu_q[b+1] - cu_q[b] >= 0, with cu_q[0] = 0 and cu_q
 *     non-decreasing;
 *   - k_b <= max_q, and L_b + k_b <= max_pages_per_seq * page_size;
 *   - every page id that holds a position 0 .. L_b + k_b - 1 lies in
 *     [0, num_pages);
 *   - no page the window writes (positions L_b .. L_b + k_b - 1) is also
 *     visible to another handled sequence (a shared prefix page must be
 *     copied before a sequence appends to it);
 *   - seq_ids entries lie in [0, B) and are distinct.
 * B is the number of rows of page_table / entries of ctx_lens.  Returns
 * IPDV_OK, or IPDV_EINVAL with ipdv_last_error() naming the first violation
 * and *bad_seq (if not NULL) set to its sequence (-1 when none applies).
 * Allocates host memory for the page-ownership map; launches nothing.
 */
int ipdv_check_page_table(const int32_t* page_table, int B, int max_pages_per_seq,
                          const int32_t* ctx_lens, const int32_t* cu_q,
                          const int32_t* seq_ids, int n_seq, int max_q,
                          int page_size, int num_pages, int32_t* bad_seq);

/*
 * verify_attn_paged_noalloc -- verify_attn_paged without a workspace
 * argument, for callers that cannot allocate device memory (code under HIP
 * graph capture, tight serving loops, harnesses that forbid allocation).
 * Same arguments, contract and results as verify_attn_paged (the same
 * kernels and split plan); the split-KV partials go to a scratch array of
 * IPDV_NOALLOC_SCRATCH_BYTES that the library holds on each GPU it runs on
 * until the process ends.  The call allocates nothing.
 *
 * Limit: calls whose workspace (ipdv_attn_workspace_size) exceeds
 * IPDV_NOALLOC_SCRATCH_BYTES return IPDV_EUNSUPPORTED before launching.
 * Every call on one GPU uses the same scratch: calls that may overlap on one
 * GPU (different streams without ordering, or other threads) race and must
 * be serialised by the caller.  Nothing in the scratch needs to start at
 * zero.
 *
 * Errors: those of verify_attn_paged except IPDV_EWORKSPACE; IPDV_EUNSUPPORTED
 * for a call above the limit.
 */
#define IPDV_NOALLOC_SCRATCH_BYTES (128u << 20)
int verify_attn_paged_noalloc(const void* q, const void* k_new, const void* v_new,
                              void* k_cache, void* v_cache,
                              const int32_t* page_table, int max_pages_per_seq,
                              const int32_t* ctx_lens, const int32_t* cu_q,
                              const int32_t* seq_ids, int n_seq, int max_q,
                              void* out,
                              int Hq, int Hkv, int D, int page_size, int num_pages, float scale,
                              int dtype, void* hip_stream);

/* Workspace bytes lmhead_logsoftmax_verify needs (0 if invalid). */
size_t ipdv_lmhead_workspace_size(int M, int Hd, int V, int K);

/*
 * One query for both workspaces, dispatching to the two typed queries above:
 *   which = IPDV_WS_ATTN:   host_shape_args = {n_seq, Hq, Hkv, D, max_q,
 *                           max_pages_per_seq, page_size}, n = 7;
 *   which = IPDV_WS_LMHEAD: host_shape_args = {M, Hd, V, K}, n = 4.
 * host_shape_args is a HOST array.  Returns 0 for an unknown `which`, a NULL
 * array, a count other than the one listed, or shape values the typed query
 * rejects (ipdv_last_error() then says which).
 */
#define IPDV_WS_ATTN 0
#define IPDV_WS_LMHEAD 1
size_t ipdv_workspace_size(int which, const int32_t* host_shape_args, int n);

/*
 * lmhead_logsoftmax_verify -- the verifier's next-token distribution at each
 * window row (temperature 1, as in the paper's rollouts, Appendix A), without
 * writing the logits to memory.
 *
 * For row m: logits l = hidden[m] . W^T (W is the [V, Hd] nn.Linear /
 * tied-embedding layout), LSE = log sum_v exp(l_v), and
 *   lse[m]        = LSE                                   (fp32)
 *   logp_prop[m]  = l[prop_tok[m]] - LSE  (the log q or log pi term of Eq. (4))
 *   argmax[m]     = the first index of the top-K order
 *   topk_idx[m,:] = Top_K of Eq. (5): the K largest logits, sorted by logit
 *                   descending, lower index first on equal logits
 *   topk_logp[m,:]= l[topk_idx] - LSE
 *   entropy[m]    = -sum_v p_v log p_v  (optional; NULL skips it)
 * Row m's outputs go to row out_rows[m] of each output array when out_rows is
 * non-NULL (scatter into batch-wide arrays), else to row m.
 *
 * hidden  [M, Hd]   (dtype);   W [V, Hd] (dtype);   prop_tok [M] int32 in [0, V)
 * out_rows [M] int32 or NULL
 * lse, logp_prop, entropy: float [rows];  argmax int32 [rows];
 * topk_idx int32 [rows, K];  topk_logp float [rows, K]
 * Requirements: M >= 0, Hd % 64 == 0 and Hd <= 4096, 1 <= V <= 262144,
 * 1 <= K <= min(IPDV_MAX_K, V).
 *
 * A row's results do not depend on the other rows' values, but their last bits
 * can depend on how many rows share the call: the order of the fp32 sums goes
 * by M, Hd and V (for instance, above 256 rows at Hd = 2048 it is another).  A
 * near-tie of the top-K, or a draw near an interval's end, can then fall the
 * other way.  The same call repeats bit for bit, and both layouts of W give
 * the same bits.
 *
 * Errors: IPDV_EINVAL, IPDV_EUNSUPPORTED (dtype, Hd), IPDV_EWORKSPACE, IPDV_EHIP.
 */
int lmhead_logsoftmax_verify(const void* hidden, const void* W,
                             const int32_t* prop_tok, const int32_t* out_rows,
                             int M, int Hd, int V, int K,
                             float* lse, float* logp_prop, int32_t* argmax,
                             int32_t* topk_idx, float* topk_logp, float* entropy,
                             int dtype, void* workspace, size_t workspace_bytes,
                             void* hip_stream);

/*
 * accept_scan -- the verdict stage (Section 3.2.3) with the top-K coverage
 * rule of Eq. (9), one window per sequence.
 *
 * Row i of sequence b scores draft i = prop_tok[cu_q[b]+i], proposed by the
 * driver; covered_i = the draft appears in topk_idx[cu_q[b]+i, 0..K-1] (the
 * verifier's support).
 *   driver S: drafts are accepted (src S) while covered; the first uncovered
 *     draft is a takeover (rejected; the teacher emits the replacement later;
 *     next driver T).
 *   driver T: drafts are accepted (src T); the first covered draft is a
 *     handback (kept; later drafts discarded; next driver S).
 *   EOS: a student EOS ends the request only if covered (else takeover); a
 *     teacher EOS is accepted and ends it.
 *   length: draft i needs seq_lens[b] + i < max_len; a request whose accepted
 *     drafts reach max_len is finished.
 * Outputs per sequence: n_acc (accepted drafts), event_row (row of the
 * takeover / handback, -1 if none), next_driver, finished (0/1),
 * new_cache_len = L_b + n_acc (+1 after a takeover: the rejected row's input
 * stays cached and the replacement becomes the last token) -- the common
 * boundary both models' caches roll back to; per row: src (IPDV_SRC_*).
 *
 * cu_q [B+1] int32, prop_tok [T] int32, topk_idx [T, K] int32 (K = 0 allowed:
 * nothing is covered), driver [B] uint8, ctx_lens [B] int32, seq_lens [B]
 * int32.  Outputs: n_acc, event_row, new_cache_len int32 [B]; next_driver,
 * finished uint8 [B]; src uint8 [T].
 *
 * Errors: IPDV_EINVAL (null pointer, B < 0, K < 0 or K > IPDV_MAX_K), IPDV_EHIP.
 */
int accept_scan(const int32_t* cu_q, const int32_t* prop_tok,
                const int32_t* topk_idx, int K,
                const uint8_t* driver, const int32_t* ctx_lens, const int32_t* seq_lens,
                int32_t eos_id, int32_t max_len, int B,
                int32_t* n_acc, int32_t* event_row, uint8_t* next_driver,
                uint8_t* finished, int32_t* new_cache_len, uint8_t* src,
                void* hip_stream);

/*
 * accept_scan_rule -- accept_scan with the rule variants named after Eq. (9)
 * in Section 3.2.1 (SKD's behaviour as described in Section 2).
 *
 * take_rule (IPDV_TAKE_*) replaces the "uncovered" test of a student-driven
 * window and hand_rule (IPDV_HAND_*) the "covered" test of a teacher-driven
 * one; every other rule of accept_scan (first event ends the window, EOS,
 * length cap, cache lengths, source labels) is unchanged, with "covered"
 * read as "passes the takeover test" for a student EOS.
 *   IPDV_TAKE_ENTROPY: row i takes over when ent[row] > tau_take.
 *   IPDV_HAND_ENTROPY: row i hands back when ent[row] <= tau_hand.
 *     ent [T] float32 is a per-row entropy chosen by the caller (the paper
 *     allows the student's or the teacher's; e.g. the `entropy` output of
 *     lmhead_logsoftmax_verify for the verifier's).  Comparisons are IEEE: a
 *     NaN entropy passes neither test.
 *   IPDV_HAND_FIXED_ONE: a teacher-driven window keeps its first draft and
 *     hands back at row 0; a takeover's next driver stays S, since the
 *     replacement is the teacher's only token (SKD: the teacher resamples the
 *     rejected position and the student resumes).
 * With IPDV_TAKE_COVERAGE and IPDV_HAND_COVERAGE it equals accept_scan.
 *
 * ent may be NULL unless an entropy rule is selected; topk_idx may be NULL
 * when K = 0 or no coverage rule is selected.
 *
 * Errors: those of accept_scan, and IPDV_EINVAL for an unknown rule or a
 * NULL ent under an entropy rule.
 */
int accept_scan_rule(const int32_t* cu_q, const int32_t* prop_tok,
                     const int32_t* topk_idx, int K,
                     const uint8_t* driver, const int32_t* ctx_lens, const int32_t* seq_lens,
                     int32_t eos_id, int32_t max_len, int B,
                     int take_rule, int hand_rule, const float* ent,
                     float tau_take, float tau_hand,
                     int32_t* n_acc, int32_t* event_row, uint8_t* next_driver,
                     uint8_t* finished, int32_t* new_cache_len, uint8_t* src,
                     void* hip_stream);

/*
 * sample_takeover -- the teacher's replacement token at a takeover (Eq. (9),
 * second case: the uncovered student draft is discarded and the teacher
 * samples a replacement from its own distribution q(. | c_t) at that position;
 * Section 3.2.3: the rejected token is regenerated by the teacher).  The
 * verifier's logits at the takeover row are that distribution, so the draw
 * reuses the preceding lmhead_logsoftmax_verify call instead of a decode step.
 *
 * The call handles the sequences b = seq_ids[i], i < n_seq (seq_ids NULL: b =
 * i), and writes token / finished of those only, so that the calls of two
 * verifiers (two models, each with its own rows) compose.  For each such b
 * with driver[b] == IPDV_DRIVER_S and event_row[b] >= 0 (accept_scan's
 * outputs: a takeover at row j = event_row[b]) the row is r = cu_q[b] + j and
 * its hidden row m = row_local ? row_local[r] : r; then
 *   token[b] = the first vocabulary index v (index order) with
 *              sum_{w <= v} softmax(l_m)_w > u[b]      (temperature 1)
 * -- the inverse-CDF draw with the caller's uniform u[b] in [0, 1) -- and
 * finished[b] is set to 1 when token[b] == eos_id (a teacher EOS is accepted
 * directly).  The other handled sequences, and those whose m is negative or
 * not below M, get token -1 and keep their finished flag.
 *
 * hidden, W, M, Hd, V, K, dtype and workspace must be those of the preceding
 * lmhead_logsoftmax_verify call over the rows of hidden, with the workspace
 * unchanged since (its group records hold the mass of each 32-entry quarter
 * of each 128-entry group; the chosen quarter's 32 logits are recomputed
 * exactly).  seq_ids [n_seq] int32
 * or NULL; cu_q [B+1] int32, driver [B] uint8, event_row [B] int32, row_local
 * [T] int32 or NULL, u [B] float (B = the batch's sequences).  Outputs: token
 * int32 [B]; finished uint8 [B] (updated in place).
 * The draw agrees with the exact one whenever u[b] is farther than the fp32
 * rounding of the cumulative probabilities from an interval end (typically
 * about 1e-6 of the total mass; at most 1.2e-4 at V = 262144).
 *
 * Errors: IPDV_EINVAL (null pointer, n_seq < 0, the LM-head shape rules),
 * IPDV_EUNSUPPORTED, IPDV_EWORKSPACE, IPDV_EHIP.
 */
int sample_takeover(const void* hidden, const void* W, int M, int Hd, int V, int K,
                    const void* workspace, size_t workspace_bytes,
                    const int32_t* seq_ids, int n_seq,
                    const int32_t* cu_q, const uint8_t* driver, const int32_t* event_row,
                    const int32_t* row_local, const float* u, int32_t eos_id,
                    int32_t* token, uint8_t* finished, int dtype, void* hip_stream);

/*
 * lmhead_sample -- one draw per row from the model's distribution at
 * temperature 1, top-p 1 (Appendix A), reusing the preceding
 * lmhead_logsoftmax_verify call's group records: the proposer's sampling step
 * of the propose stage (Section 3.2.3: the driver proposes its next tokens
 * autoregressively; Eq. (9): x~ ~ pi(. | c_t) when the student drives, q when
 * the teacher does).
 *
 *   token[m] = the first vocabulary index v (index order) with
 *              sum_{w <= v} softmax(l_m)_w > u[m]
 * -- the inverse-CDF draw with the caller's uniform u[m] in [0, 1).
 *
 * hidden, W, M, Hd, V, K, dtype and workspace as in the preceding
 * lmhead_logsoftmax_verify call over these rows, the workspace unchanged
 * since.  u [M] float, token [M] int32.  The same rounding note as
 * sample_takeover applies.
 *
 * Errors: IPDV_EINVAL (null pointer, the LM-head shape rules),
 * IPDV_EUNSUPPORTED, IPDV_EWORKSPACE, IPDV_EHIP.
 */
int lmhead_sample(const void* hidden, const void* W, int M, int Hd, int V, int K,
                  const void* workspace, size_t workspace_bytes, const float* u,
                  int32_t* token, int dtype, void* hip_stream);

/*
 * lmhead_pack_w -- W [V, Hd] row-major bf16 -> the tiled layout of IPDV_W_TILED:
 * [ceil(V/16)][Hd/32][16][32], i.e. element (v, c) at
 * ((v/16) * (Hd/32) + c/32) * 512 + (v%16) * 32 + c%32, with rows V..16*ceil(V/16)-1
 * zero.  Each 16-row x 32-channel block is 1 KB contiguous, one pipeline
 * stage of the LM-head GEMM for 16 vocabulary rows.  Done once per weight
 * (at load time in an engine); the packed copy then replaces W in the calls
 * above with dtype IPDV_BF16 | IPDV_W_TILED.
 *
 * W_tiled: device buffer of ipdv_lmhead_packed_w_size(V, Hd) bytes, not
 * aliasing W.  V and Hd follow the LM-head shape rules.
 *
 * Errors: IPDV_EINVAL (null or aliasing pointers, shape rules),
 * IPDV_EUNSUPPORTED (dtype other than IPDV_BF16), IPDV_EHIP.
 */
size_t ipdv_lmhead_packed_w_size(int V, int Hd);
int lmhead_pack_w(const void* W, int V, int Hd, void* W_tiled, int dtype, void* hip_stream);

/*
 * lmhead_logp_gather -- log-softmax of a model's logits at listed vocabulary
 * indices: logp[m, j] = hidden[m] . W[idx[m, j]] - lse[m].  The union support
 * of Eq. (6) needs each model's log-probs at the other model's top-K indices
 * (S^pi u S^q, Eq. (5)); each model's own top-K log-probs come from
 * lmhead_logsoftmax_verify.
 *
 * hidden [M, Hd], W [V, Hd] (dtype), lse [M] float (that call's LSE for these
 * rows), idx [M, n_idx] int32, n_idx <= IPDV_MAX_GATHER.  Output logp [M,
 * n_idx] float; an index outside [0, V) gives -inf.  The dot product is
 * accumulated in fp32 in a different order from the GEMM's, so a value can
 * differ from the same index's top-K log-prob by fp32 rounding (about 1e-6
 * of the logit's magnitude).
 *
 * Errors: IPDV_EINVAL (null pointer, n_idx out of range, the LM-head shape
 * rules with K = 1), IPDV_EUNSUPPORTED, IPDV_EHIP.
 */
int lmhead_logp_gather(const void* hidden, const void* W, int M, int Hd, int V,
                       const float* lse, const int32_t* idx, int n_idx,
                       float* logp, int dtype, void* hip_stream);

/*
 * source_split_kl -- the per-position values of the source-split objective
 * (Section 3.2.2).  For each row m (a position c_t seen by both models):
 *   S^pi = s_idx[m, 0..K-1] (student top-K), S^q = t_idx[m, 0..K-1] (teacher);
 *   S_t  = the support (IPDV_SUPPORT_*; Eq. (5));
 *   pi_bar, q_bar = both distributions renormalised on S_t (Eq. (6));
 *   kl_rev[m] = D(pi_bar || q_bar), kl_fwd[m] = D(q_bar || pi_bar) (Eq. (10));
 *   loss[m]   = by src[m] and loss_mode (IPDV_LOSS_*): with the default,
 *               kl_rev where src = IPDV_SRC_S, kl_fwd where src = IPDV_SRC_T,
 *               0 where src = IPDV_SRC_DISCARDED;
 *   overlap[m] = |S^pi n S^q| / K (the top-K overlap ratio, Section 4.2).
 * An empty support (a disjoint intersection) gives 0 for both KLs.
 * With cu (segment offsets [B+1], one segment per trajectory), also
 *   seq_loss[b] = the mean of loss over the segment's emitted rows (src S or
 *                 T) -- the length-normalised inner term of Eq. (11);
 *   t_ratio[b]  = the share of teacher tokens among them (the intervention
 *                 ratio, Section 4.3); both 0 for a segment with none.
 *
 * Inputs, each [M, K] (float or int32): s_idx, s_logp (the student's top-K
 * and its log-probs, from its lmhead_logsoftmax_verify), s_at_t (the
 * student's log-probs at t_idx, from lmhead_logp_gather), t_idx, t_logp, t_at_s
 * (the same for the teacher); src [M] uint8.  Log-probs must be finite.  An
 * index in both lists takes its two log-probs from the list that defines the
 * support: the student's (s_logp, t_at_s) for the union, S^pi and the
 * intersection, the teacher's (s_at_t, t_logp) for S^q.  Outputs kl_rev,
 * kl_fwd, loss, overlap [M] and seq_loss, t_ratio [B] float are each
 * optional (NULL: not written); src is required with loss or cu, and loss
 * with cu and B > 0.  Computed in fp32.
 *
 * Errors: IPDV_EINVAL (null pointer, M < 0, K outside [1, IPDV_MAX_K], an
 * unknown support or loss mode, B < 0), IPDV_EHIP.
 */
int source_split_kl(int M, int K,
                    const int32_t* s_idx, const float* s_logp, const float* s_at_t,
                    const int32_t* t_idx, const float* t_logp, const float* t_at_s,
                    const uint8_t* src, int support, int loss_mode,
                    float* kl_rev, float* kl_fwd, float* loss, float* overlap,
                    const int32_t* cu, int B, float* seq_loss, float* t_ratio,
                    void* hip_stream);

/* Pairs of channels that rope_window turns. */
#define IPDV_ROPE_HALF 0          /* channels p and p + rot/2 */
#define IPDV_ROPE_INTERLEAVED 1   /* channels 2p and 2p + 1 */

/* Frequencies of long contexts (ipdv_rope_inv_freq). */
#define IPDV_ROPE_PLAIN 0    /* f_p = base^(-2p/rot) */
#define IPDV_ROPE_LINEAR 1   /* f_p / factor: positions interpolated */
#define IPDV_ROPE_NTK 2      /* base * factor^(rot/(rot-2)): the lowest frequency is divided by factor */
#define IPDV_ROPE_YARN 3     /* f_p / factor where a pair turns less than beta_slow times over
                                original_len, f_p where more than beta_fast times, a ramp over p between (its
                                ends, rounded outwards to whole p, lie within 0 .. rot - 1) */

/*
 * ipdv_rope_inv_freq -- the inverse frequencies of rope_window for a head of
 * `rot` rotary channels.  Host arithmetic in double, rounded once: inv_freq
 * [rot/2] is a HOST array.  *rope_factor (not NULL) becomes the factor to
 * multiply the rotation with: 0.1 ln(factor) + 1 for IPDV_ROPE_YARN, else 1.
 *
 * Errors: IPDV_EINVAL (null pointer, rot odd or < 2, base not > 1 and finite,
 * factor not >= 1 and finite, unknown kind; IPDV_ROPE_NTK with rot = 2;
 * IPDV_ROPE_YARN with original_len < 1 or not beta_fast > beta_slow > 0).
 */
int ipdv_rope_inv_freq(int rot, double base, int kind, double factor, int original_len,
                       double beta_fast, double beta_slow, float* inv_freq, float* rope_factor);

/*
 * rope_window -- rotary positions.  For row i of handled sequence b (position
 * L_b + i), every head of q and k, and every pair (x, y) of its first `rot`
 * channels:
 *   x' = factor (x cos a - y sin a),  y' = factor (x sin a + y cos a),
 *   a = (L_b + i) inv_freq[pair], in double; `inverse` turns by -a
 * (with the same factor the transposed map: the gradient of q and k from that
 * of q' and k').  Channels from `rot` on are copied.
 *
 * q [T, Hq, D], k [T, Hkv, D], q_out, k_out of the same shapes (dtype).  Heads
 * and channels are dense; *_row_stride is the number of ELEMENTS from one row
 * to the next (>= heads * D), so that q and k may be slices of one projection's
 * output.  q_out == q and k_out == k (with equal strides) work in place; any
 * other overlap does not.
 * inv_freq [rot/2] float (device); ctx_lens, cu_q, seq_ids, n_seq, max_q as in
 * verify_attn_paged.  Rows of other sequences are neither read nor written.
 * Requirements: 2 <= rot <= D <= 512, rot even; n_seq <= 65535; max_q * (Hq +
 * Hkv) * D < 2^32.
 *
 * Errors: IPDV_EINVAL, IPDV_EUNSUPPORTED (dtype, D, n_seq), IPDV_EHIP.
 */
int rope_window(const void* q, int64_t q_row_stride, const void* k, int64_t k_row_stride,
                void* q_out, int64_t q_out_row_stride, void* k_out, int64_t k_out_row_stride,
                const float* inv_freq, const int32_t* ctx_lens, const int32_t* cu_q,
                const int32_t* seq_ids, int n_seq, int max_q, int Hq, int Hkv, int D, int rot,
                int layout, float factor, int inverse, int dtype, void* hip_stream);

/*
 * kv_append_q8 -- the window's keys and values quantised into the 8-bit cache:
 * rows i of every handled sequence go to positions L_b + i.
 *
 * One row of one KV head, keys and values apart, is stored in 8-bit floats
 * (e4m3: 4 exponent, 3 mantissa bits, no infinities, largest 448) with a
 * power-of-two scale:
 *   e = the least integer >= -126 with max|x| <= 448 * 2^e  (0 if all are 0)
 *   stored = x * 2^-e rounded to nearest even; scale byte = e + 127
 * so that a stored value stands for stored * 2^e.  A row with an entry that is
 * not finite is stored as NaN as a whole (scale byte 255).
 *
 * k_new, v_new [T, Hkv, D] (dtype), *_row_stride elements from one row to the
 *                       next (>= Hkv * D)
 * k_pages [num_pages, Hkv, D/16, page_size, 16]  e4m3 bytes: per KV head and 16
 *                       channels, those of each slot in turn (channel d of a
 *                       slot at [page][g][d/16][slot][d%16])
 * v_pages [num_pages, Hkv, D, page_size]         e4m3 bytes, channel-major
 * scales  [num_pages, Hkv, 2, page_size]         scale bytes: keys, values
 * page_table, ctx_lens, cu_q, seq_ids, n_seq, max_q as in verify_attn_paged.
 * Slots of other positions are left as they are.
 * Requirements: D in {64, 128}, page_size 16, 32 or 64, n_seq * Hkv <= 65535,
 * num_pages * Hkv < 2^31, max_q < 2^27; pages, scales and the rows of k_new and
 * v_new start on 16-byte boundaries.
 *
 * Errors: IPDV_EINVAL, IPDV_EUNSUPPORTED (D, page_size, dtype, alignment), IPDV_EHIP.
 */
int kv_append_q8(const void* k_new, int64_t k_row_stride, const void* v_new, int64_t v_row_stride,
                 void* k_pages, void* v_pages, void* scales,
                 const int32_t* page_table, int max_pages_per_seq,
                 const int32_t* ctx_lens, const int32_t* cu_q, const int32_t* seq_ids,
                 int n_seq, int max_q, int Hkv, int D, int page_size, int num_pages,
                 int dtype, void* hip_stream);

/*
 * kv_read_q8 -- rows of the 8-bit cache as values: positions L_b + i, i < k_b,
 * of every handled sequence to rows cu_q[b] + i of k_out and v_out [T, Hkv, D]
 * (dense, dtype; T at least where the last handled window ends).  With ctx_lens
 * = 0 and the cached lengths in cu_q, whole sequences.  An e4m3 value times its scale is exact in fp32, and in bf16 down
 * to 2^-133 (below, it is rounded); rows of scale byte 255 are NaN.  The other
 * arguments, requirements and errors are those of kv_append_q8.
 */
int kv_read_q8(const void* k_pages, const void* v_pages, const void* scales,
               const int32_t* page_table, int max_pages_per_seq,
               const int32_t* ctx_lens, const int32_t* cu_q, const int32_t* seq_ids,
               int n_seq, int max_q, void* k_out, void* v_out,
               int Hkv, int D, int page_size, int num_pages, int dtype, void* hip_stream);

/* Workspace bytes verify_attn_q8 needs (0 if the arguments are invalid). */
size_t ipdv_attn_q8_workspace_size(int n_seq, int Hq, int Hkv, int D, int max_q);

/*
 * verify_attn_q8 -- verification-stage attention over the 8-bit cache: with
 * K_j and V_j the values that positions j = 0 .. L_b + i of KV head g stand for,
 *   out[cu_q[b]+i, h, :] = softmax_j( scale * q[cu_q[b]+i, h, :] . K_j ) . V_j
 * as in verify_attn_paged, but the window must already be in the cache
 * (kv_append_q8 on the same stream).  A NaN row of the cache makes the rows
 * that see it NaN, and no others; slots behind a sequence's last position may
 * hold anything.
 * Sums, maxima and the normalisation are fp32.  A bf16 call holds a probability
 * to 16 bits before its product with V where max_q * Hq / Hkv is at most 16, else
 * rounds it to bf16 once; and a query's channels to 8 bits down to 2^-14 of its
 * largest, below that to 2^-21 of the largest.  An fp32 call keeps 24 bits of both.
 *
 * q [T, Hq, D] (dtype), q_row_stride elements from one row to the next (>= Hq *
 * D); out [T, Hq, D] dense (dtype).  bf16 and fp32, D in {64, 128}.  The pages
 * as in kv_append_q8, the other arguments as in verify_attn_paged.  q's rows,
 * out, the pages, scales and workspace start on 16-byte boundaries.
 * The workspace is written by the call; two calls that may overlap need one each.
 *
 * Errors: IPDV_EINVAL, IPDV_EUNSUPPORTED (D, page_size, dtype, alignment, sizes
 * as in verify_attn_paged), IPDV_EWORKSPACE, IPDV_EHIP.
 */
int verify_attn_q8(const void* q, int64_t q_row_stride,
                   const void* k_pages, const void* v_pages, const void* scales,
                   const int32_t* page_table, int max_pages_per_seq,
                   const int32_t* ctx_lens, const int32_t* cu_q, const int32_t* seq_ids,
                   int n_seq, int max_q, void* out,
                   int Hq, int Hkv, int D, int page_size, int num_pages, float scale,
                   int dtype, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Workspace bytes sample_logits needs (0 if the arguments are invalid). */
size_t ipdv_sample_logits_workspace_size(int M, int V);

/*
 * sample_logits -- one draw per row from logits, each row with its own filters.
 *
 * For row m let p = softmax(l / T), and order the vocabulary by logit
 * descending, lower index first on equal logits.  Each filter keeps a prefix:
 *   top-k: the first top_k[m] entries                      (<= 0: off)
 *   top-p: as many of those as it takes for their mass to reach top_p[m] times
 *          the mass that top-k left                        (>= 1 or NaN: off)
 *   min-p: the entries with (l - max l) / T >= ln(min_p[m]) (<= 0 or NaN: off)
 * and the shortest, of one entry at least, is drawn from:
 *   token[m] = the first kept index v (index order) whose cumulative kept mass
 *              exceeds u[m] times the kept mass
 *   logp[m]  = ln of token[m]'s share of the kept mass (optional; NULL)
 * Entries with less than e^-31.9 of the largest probability count as of
 * probability zero.  Masses are fp32 exponentials (relative error about 1e-7
 * each), summed exactly for the cuts and for the part of 16384 entries that the
 * draw falls in; inside it 32 neighbours at a time are summed in fp32, and an entry
 * of a small mass m (the largest 1) is off by 2^-24 |ln m| of it, so by less than
 * 1e-7 of the row's.  A cut or a draw closer than that to a border may fall on the
 * border's other side.  The same call repeats bit for bit.
 * T = 0 draws the first entry of the order; 0 < T < 2^-124 is taken as 2^-124.
 * Entries of -inf are never drawn.  A row that holds NaN or +inf, or nothing
 * above -inf, and a row whose T is negative or NaN, gets token -1 and logp NaN.
 *
 * logits [M, V] (dtype), row_stride elements from one row to the next (>= V);
 * u [M] float in [0, 1); temperature, top_p, min_p [M] float and top_k [M]
 * int32, each NULL for off (temperature: 1).  Requirements: 0 <= M < 2^22, 1 <=
 * V <= 262144, M * V < 2^35; workspace on a 16-byte boundary.
 * The workspace is written by the call; two calls that may overlap need one each.
 *
 * Errors: IPDV_EINVAL, IPDV_EUNSUPPORTED (dtype, V, M), IPDV_EWORKSPACE, IPDV_EHIP.
 */
int sample_logits(const void* logits, int64_t row_stride, int M, int V, const float* u,
                  const float* temperature, const int32_t* top_k, const float* top_p,
                  const float* min_p, int32_t* token, float* logp, int dtype,
                  void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * What a score is before the softmax (verify_attn_masked, attn_mass).  For row r
 * = cu_q[b] + i at position p = L_b + i, head h and key j:
 *   x = scale * q . K_j
 *   x = softcap * tanh(x / softcap)              (softcap > 0; 0: off.  At most 2^127, with
 *                                                scale / softcap in [2^-126, 2^125])
 *   x = x - slopes[h] * |p - j|                  (slopes [Hq] float; NULL: off)
 * over the keys  max(first_key[r], p - window + 1, 0) <= j < end_key[r]  and
 * j < L_b + k_b:
 *   window            keys that a row sees at most, its own the last of them (0: off)
 *   first_key [T] int32   e.g. where the row's document begins (NULL: 0)
 *   end_key [T] int32     e.g. the end of a prefix that sees itself whole (NULL: p + 1)
 * A row may be left without keys.  Scores are fp32; up to a softcap of 64 bf16 calls hold a
 * capped one to 2^-22 of softcap, with larger ones to 2^-20 of itself.
 */

/* Workspace bytes verify_attn_masked needs (0 if the arguments are invalid).
 * `window` as in the call, has_end_key whether it has an end_key. */
size_t ipdv_attn_masked_workspace_size(int n_seq, int Hq, int Hkv, int D, int max_q,
                                       int max_pages_per_seq, int page_size,
                                       int window, int has_end_key);

/*
 * verify_attn_masked -- verify_attn_paged with modified scores x (see above):
 * appends the window, then
 *   out[r, h, :] = sum_j softmax_j(x) V_j,   lse[r, h] = ln sum_j e^x
 * over the keys that the row sees; a row that sees none gets 0 and -inf.  Keys and
 * values of slots that a row does not see may hold anything, NaN and infinities
 * included; a value that is not finite makes the rows that see it not finite.
 * Maxima, sums and lse are fp32; a bf16 call holds a probability to 16 bits before its
 * product with V where max_q * Hq / Hkv is at most 16, else rounds it to bf16 once.
 *
 * q [T, Hq, D] (dtype), q_row_stride elements from one row to the next (>= Hq *
 * D); k_new, v_new [T, Hkv, D] (dtype; both NULL: the window is in the cache
 * already); lse [T, Hq] float or NULL.  bf16 and fp32, D in {64, 128}.  The cache and the
 * other arguments as in verify_attn_paged.  q's rows, k_new, v_new, the caches, out and
 * workspace start on 16-byte boundaries.
 * The workspace is written by the call; two calls that may overlap need one each.
 * max_q * Hq / Hkv may be 2^20 in any case, and more where the keys are few.
 *
 * Errors: IPDV_EINVAL (also: softcap negative or not finite, window < 0),
 * IPDV_EUNSUPPORTED (D, page_size, dtype, softcap, alignment, sizes), IPDV_EWORKSPACE, IPDV_EHIP.
 */
int verify_attn_masked(const void* q, int64_t q_row_stride, const void* k_new, const void* v_new,
                       void* k_cache, void* v_cache,
                       const int32_t* page_table, int max_pages_per_seq,
                       const int32_t* ctx_lens, const int32_t* cu_q, const int32_t* seq_ids,
                       int n_seq, int max_q, float softcap, int window, const float* slopes,
                       const int32_t* first_key, const int32_t* end_key, void* out, float* lse,
                       int Hq, int Hkv, int D, int page_size, int num_pages, float scale,
                       int dtype, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * attn_mass -- the attention weight that every cached key gathers from a window: for
 * position j of handled sequence b and KV head g, at its place in the pages,
 *   mass_out = decay * mass_in + sum over rows r and heads h of g of e^(x - lse[r, h])
 * with x and the rows' keys as in verify_attn_masked, whose lse the call takes.  j runs
 * over all positions below L_b + k_b, also those that no row sees; those of the window
 * itself (j >= L_b) start at 0, and so do all where mass_in is NULL.  Slots of other
 * positions are left as they are.  The window must be in the cache.  q and lse may both be
 * NULL: no sequence has rows then, whatever cu_q holds.
 *
 * q, k_cache, the scores' and the batch's arguments as in verify_attn_masked; lse [T,
 * Hq] float; mass_in, mass_out [num_pages, Hkv, page_size] float, the same array or
 * two that do not overlap; 0 <= decay, finite.  Requirement:
 * max_pages_per_seq * page_size + max_q <= 2^22.  A page that two handled sequences
 * share gets the mass of one of them (with mass_in == mass_out, of both in either order
 * or of one): let them have pages of their own, or take them in calls of their own.
 *
 * Errors: IPDV_EINVAL, IPDV_EUNSUPPORTED, IPDV_EHIP.
 */
int attn_mass(const void* q, int64_t q_row_stride, const void* k_cache, const float* lse,
              const int32_t* page_table, int max_pages_per_seq,
              const int32_t* ctx_lens, const int32_t* cu_q, const int32_t* seq_ids,
              int n_seq, int max_q, float softcap, int window, const float* slopes,
              const int32_t* first_key, const int32_t* end_key,
              const float* mass_in, float decay, float* mass_out,
              int Hq, int Hkv, int D, int page_size, int num_pages, float scale,
              int dtype, void* hip_stream);

/*
 * kv_evict -- sequences cut to their heaviest keys.  Of handled sequence b's L_b positions
 * every KV head keeps
 *   n = min(max(keep[b], 0), L_b, max_dst_pages * page_size):
 * the first min(n_sink, n), the last n_recent (as far as n reaches), and of the others
 * those of the largest mass; equal masses: the lower position; NaN below everything.
 * In ascending order they become positions 0 .. n - 1 of dst_table's pages, keys, values
 * and masses.  new_lens[b] = n; kept[b, g, i] = the position that i was, -1 for i >= n.
 * The heads of a sequence keep positions of their own, so that a slot no longer stands
 * for one position: distance biases and sliding windows then count slots.
 *
 * k_cache, v_cache as in verify_attn_paged (dtype, in/out), mass [num_pages, Hkv,
 * page_size] float (in/out); page_table [B, max_pages_per_seq], dst_table [B,
 * max_dst_pages] int32; ctx_lens, keep [B] int32; seq_ids [n_seq] int32 or NULL;
 * new_lens [B], which may be ctx_lens or keep itself, kept [B, Hkv, max_dst_pages * page_size]
 * int32 (entries of other sequences are left).  The pages that dst_table names for positions 0 .. n - 1 must belong to no
 * other sequence and hold nothing that the call reads: not the sequence's own, either.
 * Slots behind position n - 1 are left as they are.
 * Requirements: D in {64, 128}; both tables times page_size <= 2^22; num_pages *
 * page_size and num_pages * Hkv below 2^31; the caches, mass on 16-byte boundaries.
 *
 * Errors: IPDV_EINVAL (also: n_sink or n_recent < 0), IPDV_EUNSUPPORTED, IPDV_EHIP.
 */
int kv_evict(void* k_cache, void* v_cache, float* mass,
             const int32_t* page_table, int max_pages_per_seq,
             const int32_t* dst_table, int max_dst_pages,
             const int32_t* ctx_lens, const int32_t* keep, const int32_t* seq_ids, int n_seq,
             int n_sink, int n_recent, int32_t* new_lens, int32_t* kept,
             int Hkv, int D, int page_size, int num_pages, int dtype, void* hip_stream);

/* Workspace bytes verify_drafts needs (0 if the arguments are invalid): whether the target's
 * and the draft's filters have more than a temperature. */
size_t ipdv_verify_drafts_workspace_size(int T, int V, int B, int target_filtered,
                                         int draft_filtered);

/*
 * verify_drafts -- the verdict on drafted tokens by the two models' probabilities.  With p
 * and q the target's and the draft's distributions at a row (softmax of the logits at the
 * row's temperature over what its filters keep, as in sample_logits), x = prop_tok[r], for
 * the rows r = cu_q[b] + i of sequence b in turn:
 *   x >= 0: accepted if u_accept[r] * q(x) < p(x).  The first draft that is not ends the
 *           window, and token[b] is drawn from max(0, p - q), normalised (from p, should
 *           nothing be left of it);
 *   x < 0:  no draft, e.g. the row behind the last: the window ends, token[b] is drawn from p;
 *   an accepted x == eos_id ends the window, without a token.
 * Tokens are drawn in index order by u_draw[b], as sample_logits does.  What a sequence
 * emits, its n_acc[b] accepted drafts and the token, is distributed as the target's own draws
 * are, if x was drawn from q.
 *   n_acc[b]     accepted drafts
 *   token[b]     the token behind them, -1 for none (all accepted, or the window ended by EOS
 *                or by a row that cannot be drawn from)
 *   finished[b]  1 if the last of these is eos_id
 *   p_accept[r]  min(1, p(x) / q(x)), of every row of a window, also behind the one that ends it;
 *                0 where x < 0, and where p(x) = q(x) = 0.  Rows outside every window are left
 *   logp[b]      ln p(token[b]), NaN without one (optional; NULL)
 * A row whose target logits (or, with a draft, its draft logits) hold NaN or +inf or nothing
 * above -inf, or whose temperature is negative or NaN, ends its window without a token; its
 * p_accept is NaN.  A draft at or beyond V has p(x) = 0 and is rejected.  draft_logits NULL:
 * q(x) = 1, as of drafts looked up or taken greedily; the draft's filters are then not read.
 * Probabilities are 64-bit floats (relative error below 1e-9), except that top-p's cut is found
 * as in sample_logits.  An entry 694 T or more below its row's maximum, less than 2^-1000 of the
 * maximum's probability (a fill of -1e4, say), has none; T from 2^100 on is taken as 2^100.  (A u_draw
 * of 0 may pass over entries of less than 2^-900, too.)  The same call repeats bit for bit.
 *
 * target_logits, draft_logits [T, V] (dtype), *_row_stride elements from one row to the next
 * (>= V); prop_tok [T], cu_q [B+1] int32 (cu_q[B] <= T); u_accept [T], u_draw [B] float in [0,
 * 1); temperature ... draft_min_p [T], each NULL for off (as in sample_logits).  Outputs and
 * inputs may not overlap, except that logp may be u_draw.
 * Requirements: 0 <= T < 2^22, 0 <= B < 2^22, 1 <= V <= 262144, T * V and B * V < 2^35;
 * workspace on a 16-byte boundary, written by the call: two calls that may overlap need one each.
 *
 * Errors: IPDV_EINVAL, IPDV_EUNSUPPORTED (dtype, V, T), IPDV_EWORKSPACE, IPDV_EHIP.
 */
int verify_drafts(const void* target_logits, int64_t target_row_stride,
                  const void* draft_logits, int64_t draft_row_stride, int T, int V,
                  const int32_t* prop_tok, const int32_t* cu_q, int B,
                  const float* u_accept, const float* u_draw,
                  const float* temperature, const int32_t* top_k, const float* top_p,
                  const float* min_p, const float* draft_temperature,
                  const int32_t* draft_top_k, const float* draft_top_p, const float* draft_min_p,
                  int32_t eos_id, int32_t* n_acc, int32_t* token, uint8_t* finished,
                  float* p_accept, float* logp, int dtype,
                  void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Optional timing hook for profilers and benchmarks (thread-local).  While
 * set, each kernel an entry point launches is bracketed by hipEventRecord of
 * the caller's events (hipEvent_t handles cast to void*), taken from
 * `events` in order: the first kernel of a call records one event before and
 * one after it, every further kernel one after it.  Recording stops when
 * `capacity` events are used.  NULL / 0 turns it off.  Returns IPDV_OK.
 * ipdv_trace_count() returns how many events have been recorded since the
 * hook was last set.  Intervals per call: verify_attn_paged 3 (append,
 * attention, split combine; where the attention kernel appends the window
 * itself the append interval is empty, and where it does not split, the
 * combine interval), lmhead_logsoftmax_verify 3 (the hidden rows' copy into the tiled
 * layout, empty where none is made; GEMM + epilogue; merge), accept_scan 1,
 * accept_scan_rule 1, sample_takeover 1, lmhead_sample 1, lmhead_pack_w 1,
 * lmhead_logp_gather 1, source_split_kl 1 (+1 with cu), rope_window 1,
 * kv_append_q8 1, kv_read_q8 1, verify_attn_q8 2 (attention, merge of cut
 * items), sample_logits 2 (chunks, rows), verify_attn_masked 3 (append, attention, merge;
 * empty where there is none), attn_mass 1, kv_evict 2 (selection, move), verify_drafts 3
 * (the rows' masses, with their cuts; verdicts and what is left of rejected rows; draws).
 */
int ipdv_trace_events(void* const* events, int capacity);
int ipdv_trace_count(void);

/* Thread-local description of the last non-OK status ("" if none). */
const char* ipdv_last_error(void);

/* Library version string. */
const char* ipdv_version(void);

#ifdef __cplusplus
}
#endif

#endif /* IPDV_H */
