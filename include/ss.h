/*
 * ss.h -- C ABI of the MI355X fused LLM sampler (libss.so).
 *
 * Operations (SonicSampler, arXiv 2607.20475):
 *   ss_sample          singular-mode sampling: prologue (Appendix C.1), top-k /
 *                      top-p / min-p truncation in Alg. 11 order (Appendix C.2),
 *                      greedy or stochastic selection (Section 3.5, Appendix C.3)
 *   ss_sample_full     the same with top-p / min-p over the whole row for
 *                      requests without a top-k cut (Appendix C.2)
 *   ss_sample_gumbel   the same with the Gumbel-max draw over the kept set and
 *                      caller-drawn noise (Appendix C.3; the Stage-2 selection)
 *   ss_verify          multistep speculative verification (Section 3.1,
 *                      Appendix C.4): accept when u*q(d) <= p(d), else resample
 *                      from normalize(max(0, p - q)); bonus token on full acceptance
 *   ss_verify_sparse   the same against sparse draft distributions: the
 *                      (id, probability) lists a singular-mode draft step
 *                      emits over its candidate set (Section 3.2)
 *   ss_verify_tree     one path through a draft tree, its positions mapped to
 *                      the target rows of the tree (Appendix C.4)
 *   ss_topk            exact top-k (value, index) per row (Section 3.4)
 *   ss_process_logits  materialised processed logits and final probabilities
 *   ss_logprobs        top-k log-probabilities under the full-row distribution
 *                      (indicator bit 0x400, Section 3.5)
 * and the operators at the two ends of the vocabulary, which make the logits
 * that these read and take up the tokens that they give (what such a call writes
 * overlaps no other array of the call, unless it says so):
 *   ss_head_w4         logits of hidden states under a 4-bit vocabulary table
 *   ss_embed, ss_embed_w4   rows of the vocabulary table by token
 *   ss_embed_grad      the gradient of such a lookup, by sorted tokens
 *   ss_quant_w4        the 4-bit form of a vocabulary table
 *
 * Conventions (all functions):
 *   - Every array argument is a DEVICE pointer owned by the caller, except
 *     `const ss_params*` and `const ss_w4*`, host structs whose members are device
 *     pointers, read during the call.  The library never allocates, frees or
 *     synchronises; every launch goes to `stream` (a hipStream_t, NULL = default
 *     stream).
 *   - Row-major layouts with an explicit row stride `ld` (elements).
 *   - Per-request parameter arrays have B entries.  A NULL parameter array
 *     disables the indicator bits that need it (e.g. temperature == NULL
 *     clears SS_TEMP for every request), so a call never reads it.
 *   - Host-side validation happens before any launch; on error nothing is
 *     launched and a negative ss_status is returned.  Data-dependent
 *     conditions never stop the call: they are reported per row in `flags`.
 *   - Launch shapes depend only on (B, V, L, k_max, dtype): every call can be
 *     captured in a HIP graph.  Per-call values (seed, position, params) are
 *     read from device memory.  (The vocabulary operators': on sizes, types,
 *     strides and alignment, never on tokens; their `scale` is a host value, which a
 *     captured call keeps.)
 *   - The workspace needs no initialisation: every call writes what it reads
 *     (its contents between calls are unspecified), so one workspace of the
 *     largest size may serve calls of any operation and shape.  Calls that
 *     share one workspace must not overlap in time.
 *   - Processed logits are float32 (one correctly rounded operation per
 *     prologue step).  Each kept token's weight exp((y - M)/tau) has its
 *     exponent formed in double and the exponential taken in float32 (about
 *     1 ulp, relative error below 2e-7; exponents below about -87 give float32
 *     subnormals and below about -104 zero, i.e. weights under 1e-38 of the
 *     row maximum's).  Weights are summed exactly as 2^-50 fixed-point
 *     integers; probabilities, cuts and draws are then taken in double.
 */
#ifndef SS_H_
#define SS_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t ss_status;
#define SS_OK 0
#define SS_ERR_INVALID_ARG (-1)
#define SS_ERR_UNSUPPORTED (-2)
#define SS_ERR_WORKSPACE (-3)
#define SS_ERR_HIP (-4)

/* Logit element types. */
#define SS_F32 0
#define SS_BF16 1

/* Per-request indicator bits: the paper's bit-level encoding table (Section 3.5). */
#define SS_GRAMMAR 0x001u  /* grammar bit-mask                                   */
#define SS_REP 0x002u      /* multiplicative repetition penalty                  */
#define SS_FREQ 0x004u     /* frequency penalty                                  */
#define SS_PRES 0x008u     /* presence penalty                                   */
#define SS_BIAS 0x010u     /* logit bias                                         */
#define SS_TEMP 0x020u     /* temperature scaling (tau <= 0 means greedy)        */
#define SS_GREEDY 0x040u   /* greedy selection                                   */
#define SS_TOPK 0x080u     /* top-k filtering                                    */
#define SS_TOPP 0x100u     /* top-p filtering                                    */
#define SS_MINP 0x200u     /* min-p filtering                                    */
#define SS_LOGPROBS 0x400u /* top-k log-probabilities (ss_logprobs)              */

/* Per-row result flags (int32 flags[rows]). */
#define SS_FLAG_EMPTY 1      /* every token masked: token -1                       */
#define SS_FLAG_FALLBACK 2   /* exact slow path used (skewed or tied row)          */
#define SS_FLAG_OUT_TRUNC 4  /* kept set longer than k_out                         */
#define SS_FLAG_KCAP 8       /* candidate set bounded by k_max (no or large top-k) */

/* Operations, for ss_workspace_bytes. */
#define SS_OP_TOPK 0
#define SS_OP_SAMPLE 1
#define SS_OP_VERIFY 2
#define SS_OP_PROCESS 3
#define SS_OP_LOGPROBS 4

/* Limits. */
#define SS_MAX_K 4096      /* k_max upper bound                                    */
#define SS_MAX_L 16        /* draft length upper bound                             */
#define SS_MAX_V (1 << 20) /* vocabulary upper bound                               */
#define SS_MAX_T (1 << 20) /* rows of a head, lookup or gradient call              */
#define SS_MAX_H (1 << 16) /* columns of a vocabulary table                        */

/*
 * Per-request parameters (host struct of device pointers), read at call time.
 *
 * mode          uint32[B]  indicator bits above.
 * temperature   float[B]   tau (Appendix C.1); tau <= 0 with SS_TEMP means greedy.
 * top_k         int32[B]   k (Appendix C.2); k <= 0 means no top-k cut.
 * top_p         float[B]   p; p >= 1 means no cut.
 * min_p         float[B]   theta; theta <= 0 means no cut.
 * rep_penalty   float[B]   alpha (> 0, finite).
 * freq_penalty  float[B]   beta (finite).
 * pres_penalty  float[B]   gamma (finite).
 * hist_offsets  int32[B+1], hist_ids int32[nnz]: CSR of decoded token ids per request
 *               (multiplicity = occurrence count; ids outside [0,V) ignored).
 * bias_offsets  int32[B+1], bias_ids int32[nnz], bias_vals float[nnz]: CSR of sparse
 *               logit-bias entries; duplicate ids are summed in list order.
 * bitmask       uint32[rows, bitmask_ld], bitmask_ld >= ceil(V/32): allow bits,
 *               bit (i & 31) of word (i >> 5), 1 = allowed.  rows = B for
 *               ss_sample / ss_process_logits, B*(L+1) for ss_verify.
 * seed          uint64[B]  Philox4x32-10 key.
 * position      int64[B]   Philox counter position of this step.
 */
typedef struct ss_params {
  int32_t B;
  int32_t V;
  const uint32_t *mode;
  const float *temperature;
  const int32_t *top_k;
  const float *top_p;
  const float *min_p;
  const float *rep_penalty;
  const float *freq_penalty;
  const float *pres_penalty;
  const int32_t *hist_offsets;
  const int32_t *hist_ids;
  const int32_t *bias_offsets;
  const int32_t *bias_ids;
  const float *bias_vals;
  const uint32_t *bitmask;
  int64_t bitmask_ld;
  const uint64_t *seed;
  const int64_t *position;
} ss_params;

/* Workspace bytes for one call of `op` (host only, pure).  L is used by
 * SS_OP_VERIFY only; dtype is SS_F32 or SS_BF16.  Returns 0 for invalid sizes. */
size_t ss_workspace_bytes(int op, int B, int V, int L, int k_max, int dtype);

/* Zero-fills a workspace with a kernel on `stream` (no memset node).  Not
 * required before use; kept for callers that want deterministic contents. */
ss_status ss_workspace_init(void *ws, size_t ws_bytes, void *stream);

/*
 * Exact top-k per row on raw values (no prologue; Section 3.4 ordering:
 * value descending, lower index first on ties; NaN ranks as -inf and is never
 * returned; -0 returns as +0).
 *   x        [B, ld] logits of `dtype`, ld >= V.
 *   k        int32[B] per-row k (NULL: k_max for every row); clamped to [0, k_max].
 *   out_val  float[B, k_max], out_idx int32[B, k_max]: the first min(k, valid)
 *            entries, padded with (-inf, -1).
 *   flags    int32[B] or NULL.
 */
ss_status ss_topk(const void *x, int dtype, int B, int V, int64_t ld, const int32_t *k, int k_max,
                  float *out_val, int32_t *out_idx, int32_t *flags, void *ws, size_t ws_bytes,
                  void *stream);

/*
 * Singular-mode sampling (one token per request).
 *   logits      [B, ld] of `dtype`.
 *   k_max       candidate bound, 1..SS_MAX_K: the top-k cut is min(k, k_max);
 *               rows with no top-k use k_max (flag SS_FLAG_KCAP).
 *   out_token   int32[B]: sampled id; -1 if every token is masked.
 *   out_logprob float[B] or NULL: ln P(token) under the final truncated
 *               distribution (0 for greedy rows).
 *   out_idx, out_prob  int32[B, k_out], float[B, k_out] or NULL: the kept set in
 *               canonical order with its probabilities, padded (-1, 0).
 *   flags       int32[B] or NULL.
 */
ss_status ss_sample(const void *logits, int dtype, int64_t ld, const ss_params *p, int k_max,
                    int32_t *out_token, float *out_logprob, int32_t *out_idx, float *out_prob,
                    int k_out, int32_t *flags, void *ws, size_t ws_bytes, void *stream);

/*
 * Singular-mode sampling with full-row truncation (Appendix C.2 defines top-p
 * and min-p over the whole vocabulary; ss_sample bounds requests without a
 * top-k cut to their k_max leading tokens, the bounded regime of Section
 * 3.3).  For a stochastic request whose top-k bit is off (or k <= 0), top-p
 * takes its boundary against the normaliser of every valid token of the row
 * (computed in the same pass over the logits) and min-p is as ever; that
 * result is returned when the kept set holds fewer than k_max tokens.  A
 * longer kept set gives ss_sample's bounded result with SS_FLAG_KCAP.  Other
 * requests, arguments and outputs are as for ss_sample (workspace
 * ss_workspace_bytes(SS_OP_SAMPLE, ...)).
 */
ss_status ss_sample_full(const void *logits, int dtype, int64_t ld, const ss_params *p, int k_max,
                         int32_t *out_token, float *out_logprob, int32_t *out_idx, float *out_prob, int k_out,
                         int32_t *flags, void *ws, size_t ws_bytes, void *stream);

/*
 * Singular-mode sampling with the Gumbel-max draw (Appendix C.3: the argmax
 * of the perturbed logits is distributed as the categorical; the Stage-2
 * selection takes pre-drawn noise).  Everything is as for ss_sample except the
 * draw: a stochastic request's token is the kept id i with the largest
 *     (y_i - M) / tau - g_i        (in double; 0 - g_i for y_i = M),
 * the lower id on equal scores, where g = ln z, z ~ Exp(1), is drawn by the
 * caller (so results are reproducible and calls capture in graphs without an
 * RNG state).  Greedy requests ignore the noise; out_logprob is ln P(token)
 * under the truncated distribution, as for ss_sample.
 *   noise     float[B, ld_noise] (ld_noise >= V), g per token; read at the
 *             kept ids only.  NaN noise is outside the contract.
 */
ss_status ss_sample_gumbel(const void *logits, int dtype, int64_t ld, const ss_params *p, int k_max,
                           const float *noise, int64_t ld_noise, int32_t *out_token, float *out_logprob,
                           int32_t *out_idx, float *out_prob, int k_out, int32_t *flags, void *ws,
                           size_t ws_bytes, void *stream);

/*
 * Multistep speculative verification.
 *   target_logits  [B, L+1, V] rows of `dtype`, row stride ld_row (row (b, l) at
 *                  (b*(L+1) + l) * ld_row); row l is the target for draft position l+1.
 *                  Its penalty history is the request history plus drafts d_1..d_l.
 *   draft_probs    float[B, L, ld_q] draft probabilities q (used as given).
 *   draft_tokens   int32[B, L]; an id outside [0, V) ends the draft (that position
 *                  then samples the target).
 *   out_tokens     int32[B, L+1]: accepted drafts, then one correction or bonus
 *                  token, then -1.
 *   out_num_accepted int32[B] in [0, L].
 *   flags          int32[B] or NULL (OR over the request's rows).
 */
ss_status ss_verify(const void *target_logits, int dtype, int64_t ld_row, const float *draft_probs,
                    int64_t ld_q, const int32_t *draft_tokens, int L, const ss_params *p, int k_max,
                    int32_t *out_tokens, int32_t *out_num_accepted, int32_t *flags, void *ws,
                    size_t ws_bytes, void *stream);

/*
 * Multistep speculative verification against sparse draft distributions
 * (Section 3.1 with the draft probabilities a singular-mode draft step emits
 * over its candidate set, Section 3.2): position l of request b lists kq
 * (id, probability) entries, e.g. the out_idx / out_prob rows of ss_sample.
 * q_l(j) is the sum of the entries naming j; unlisted ids have q = 0, and ids
 * outside [0, V) (the padding -1 among them) are ignored.  Everything else,
 * results included, is as for ss_verify.
 *   draft_idx   int32[B, L, kq], draft_q float[B, L, kq] (used as given).
 *   kq          1..SS_MAX_K entries per draft position.
 *   ws          ss_workspace_bytes(SS_OP_VERIFY, B, V, L, k_max, dtype) bytes.
 */
ss_status ss_verify_sparse(const void *target_logits, int dtype, int64_t ld_row, const int32_t *draft_idx,
                           const float *draft_q, int kq, const int32_t *draft_tokens, int L,
                           const ss_params *p, int k_max, int32_t *out_tokens, int32_t *out_num_accepted,
                           int32_t *flags, void *ws, size_t ws_bytes, void *stream);

/*
 * Verification of one path through a draft tree (the draft-to-target mapping
 * of Appendix C.4, as tree speculation needs): the target evaluated Lt rows
 * per request for the tree's nodes, and path position l (0-based, l = L being
 * the bonus / correction position after L acceptances) is verified against
 * target row row_map[b, l].  A map entry outside [0, Lt) gives a target row
 * with every token masked (SS_FLAG_EMPTY: the path ends there with no
 * correction token).  Draft lists are sparse, as for ss_verify_sparse.  The
 * penalty history, the grammar rows (bitmask rows B*(L+1), one per path
 * position), the uniforms and the outputs follow the path, as for ss_verify.
 *   target_logits  [B, Lt, V] rows of `dtype`, row stride ld_row (request b's
 *                  row t at (b*Lt + t) * ld_row).
 *   Lt             target rows per request, >= 1.
 *   row_map        int32[B, L+1].
 *   ws             ss_workspace_bytes(SS_OP_VERIFY, B, V, L, k_max, dtype) bytes.
 */
ss_status ss_verify_tree(const void *target_logits, int dtype, int64_t ld_row, int Lt, const int32_t *row_map,
                         const int32_t *draft_idx, const float *draft_q, int kq, const int32_t *draft_tokens,
                         int L, const ss_params *p, int k_max, int32_t *out_tokens, int32_t *out_num_accepted,
                         int32_t *flags, void *ws, size_t ws_bytes, void *stream);

/*
 * Materialised pipeline (unfused reference path).
 *   out_logits float[B, V] (row stride V): processed logits y before temperature
 *              (-inf where masked).  May be NULL.
 *   out_probs  float[B, V] (row stride V): final truncated distribution (zero
 *              outside the kept set; one-hot at the argmax for greedy rows).  May be NULL.
 */
ss_status ss_process_logits(const void *logits, int dtype, int64_t ld, const ss_params *p, int k_max,
                            float *out_logits, float *out_probs, int32_t *flags, void *ws,
                            size_t ws_bytes, void *stream);

/*
 * Top-k log-probabilities (indicator bit SS_LOGPROBS = 0x400 of the
 * bit-level encoding table, Section 3.5; the log-probability output of
 * Alg. 11).  For every request whose mode has the bit: the n_lp leading
 * tokens of the canonical order of its processed logits y (the Appendix C.1
 * prologue: grammar mask, penalties, bias; value descending, lower index
 * first) and their log-probabilities under the untruncated distribution
 * softmax(y / tau) over all valid tokens of the row:
 *     lp_i = (y_i - M) / tau - ln sum_j exp((y_j - M) / tau),   M = max_j y_j,
 * tau being the request's temperature when SS_TEMP is set, tau > 0 and the
 * request is not greedy, else 1.  Top-k, top-p and min-p do not apply.
 *   logits    [B, ld] of `dtype`.
 *   n_lp      1..SS_MAX_K entries per request.
 *   out_idx   int32[B, n_lp], out_lp float[B, n_lp]: padded with (-1, -inf)
 *             beyond the valid tokens and for requests without the bit.
 *   flags     int32[B] or NULL.
 *   ws        ss_workspace_bytes(SS_OP_LOGPROBS, B, V, 0, n_lp, dtype) bytes.
 * The normaliser's terms are float32 exponentials, summed in double: a term e^-x
 * of its 2048-token unit's largest has a relative error of up to about
 * (1 + 1.5 x) 1.2e-7, so the sum's is a few 1e-7 (2.6e-8 measured on model-like
 * rows) and stays below 3e-6 where most of the mass lies in the tail.
 */
ss_status ss_logprobs(const void *logits, int dtype, int64_t ld, const ss_params *p, int n_lp,
                      int32_t *out_idx, float *out_lp, int32_t *flags, void *ws, size_t ws_bytes,
                      void *stream);

/*
 * ss_sample with no workspace argument, for callers that cannot allocate
 * device memory (code under HIP graph capture, serving loops and harnesses
 * that forbid allocation).  The workspace is an SS_NOALLOC_BYTES array in the
 * library's device memory, one copy per GPU, held until the process ends;
 * this call allocates and frees nothing.  Arguments and results are those of
 * ss_sample.  SS_ERR_WORKSPACE when ss_workspace_bytes(SS_OP_SAMPLE, B, V, 0,
 * k_max, dtype) exceeds SS_NOALLOC_BYTES (B = 64, V = 2^17, k_max = 1024
 * fits).  Every call on one GPU uses that GPU's single array: calls that
 * overlap in time on one GPU (other streams, other threads) race.
 */
#define SS_NOALLOC_BYTES (48u << 20)
ss_status ss_sample_noalloc(const void *logits, int dtype, int64_t ld, const ss_params *p, int k_max,
                            int32_t *out_token, float *out_logprob, int32_t *out_idx, float *out_prob,
                            int k_out, int32_t *flags, void *stream);

/*
 * A vocabulary table in 4 bits (host struct of device pointers, read at call
 * time): V rows of H columns, a scale for each `group` columns.
 *   fmt     SS_W4_INT: integers -7..7 with a bfloat16 scale for each 32, 64 or 128
 *           columns.  SS_W4_MX: E2M1 numbers (0, .5, 1, 1.5, 2, 3, 4, 6 and their
 *           negatives) with a scale 2^(x - 127), x one byte (255: NaN), for
 *           each 32 columns.  H is a multiple of `group`.
 *   codes   ceil(H / 128) blocks of 64 bytes a row.  Dword 4 g + j of a block (g, j
 *           = 0..3, little-endian) holds its columns 32 j + 8 g + e, e = 0..7.
 *           SS_W4_MX: column e in bits 4 e .. 4 e + 3.  SS_W4_INT: with bytes
 *           s0000mmm (sign and magnitude), A those of e = 0..3 and B those of e =
 *           4..7, lowest byte first: A | rotl32(B, 4).
 *   scales  ceil(H / 128) * 128 / group a row, in column order.
 * What stands for columns beyond H in a row's last block takes no part in
 * any result.  Both pointers are aligned to 16 bytes, rows follow one another.
 * The value of a column is code * scale.  Group scales of SS_W4_MX below 2^-125
 * give weights that are subnormal in bfloat16; ss_head_w4 may take those as zero.
 */
#define SS_W4_INT 0
#define SS_W4_MX 1
typedef struct ss_w4 {
  int32_t V;
  int32_t H;
  int32_t fmt;
  int32_t group;
  const void *codes;
  const void *scales;
} ss_w4;

/* Bytes of a table's two arrays (host only, pure; the pointers are not looked
 * at).  0 for sizes or formats that are not offered. */
size_t ss_w4_codes_bytes(const ss_w4 *t);
size_t ss_w4_scales_bytes(const ss_w4 *t);

/*
 * The 4-bit form of a table, for serving what was trained: writes the codes and
 * scales that `t` points to, for each group of a row from its largest
 * magnitude a:
 *   SS_W4_INT  s = a / 7 rounded to float32 and then to bfloat16, code = w / s rounded
 *              to the nearest integer (ties to even) of -7..7; s = 0 gives magnitudes 0.
 *   SS_W4_MX   2^e with e = floor(log2 a) - 2, not below -127; code = w / 2^e
 *              rounded to the nearest E2M1 number (ties to the even code), at most 6.
 * Quotients are rounded once, as if exact.  A code keeps its weight's sign, at magnitude 0 too.
 * A group that holds a NaN or an infinity gets a NaN scale and codes 0 without signs.  Columns
 * beyond H are filled with zeros.
 *   w       [V, ld] of `dtype`, ld >= H.
 *   values  NULL, or [V, ld_values] of `values_dtype`: the numbers that the codes stand for
 *           (code * scale, rounded once), as training against the quantised table needs.  May be
 *           w itself, with its type and stride.
 */
ss_status ss_quant_w4(const void *w, int dtype, int64_t ld, const ss_w4 *t, void *values, int values_dtype,
                      int64_t ld_values, void *stream);

/* Workspace bytes of ss_head_w4 (host only, pure).  0 for invalid sizes. */
size_t ss_head_w4_bytes(int T, int H, int dtype);

/*
 * Logits of hidden states under a 4-bit table:
 *     logits[t, v] = sum_k h[t, k] * W[v, k]
 * with products exact and sums in float32 (float32 hidden states are taken whole, as three
 * bfloat16 parts), rounded once to `out_dtype`.  The sampler's entry points read the result.
 * SS_W4_INT: a group's products with the integers are summed before the group's scale, so hidden states
 * beyond 2^116 may overflow where the scaled sum would not.  Bits of hidden states below 2^-126 may be
 * taken as zero.
 * A row does not depend on the values of the other rows.
 *   h       [T, ld_h] of `dtype` (SS_F32 or SS_BF16), 0 <= T <= SS_MAX_T, ld_h >= t->H.
 *   logits  [T, ld] of `out_dtype`, ld >= t->V; columns beyond V are left as they were.
 *   ws      ss_head_w4_bytes(T, t->H, dtype) bytes, 16-byte aligned.
 * An infinite or NaN hidden state makes its whole row non-finite or NaN; other rows are not touched.
 */
ss_status ss_head_w4(const void *h, int dtype, int T, int64_t ld_h, const ss_w4 *t, void *logits, int out_dtype,
                     int64_t ld, void *ws, size_t ws_bytes, void *stream);

/*
 * Rows of a vocabulary table by token: out[t, :] = scale * table[tokens[t], :], in
 * float32 and rounded once.  A token outside [0, V) (the padding -1 of
 * ss_verify, the token -1 of an empty row) gives a row of zeros.
 *   tokens  int32[T], 0 <= T <= SS_MAX_T.
 *   table   [V, ld] of `dtype`, ld >= H, 1 <= H <= SS_MAX_H; for ss_embed_w4 a 4-bit table.
 *   out     [T, ld_out] of `out_dtype`, ld_out >= H.
 */
ss_status ss_embed(const int32_t *tokens, int T, const void *table, int dtype, int V, int H, int64_t ld, float scale,
                   void *out, int out_dtype, int64_t ld_out, void *stream);
ss_status ss_embed_w4(const int32_t *tokens, int T, const ss_w4 *t, float scale, void *out, int out_dtype,
                      int64_t ld_out, void *stream);

/* Workspace bytes of ss_embed_grad (host only, pure).  0 for invalid sizes. */
size_t ss_embed_grad_bytes(int T, int V, int H);

/*
 * The gradient of a lookup with respect to its table:
 *     dtable[v, :] = scale * sum over t with tokens[t] = v of dout[t, :]
 * for all V rows (zeros where no token names the row).  With `accumulate`, it
 * is added to what dtable holds, and rows that no token names are left as they
 * were.  Tokens outside [0, V) are passed over.  Sums are taken in float32 in an
 * order that the tokens alone determine, and rounded once to `out_dtype`: the
 * same call gives the same bits.
 *   dout    [T, ld] of `dtype`, 0 <= T <= SS_MAX_T, ld >= H.
 *   dtable  [V, ld_out] of `out_dtype`, ld_out >= H.
 *   ws      ss_embed_grad_bytes(T, V, H) bytes, 16-byte aligned.
 */
ss_status ss_embed_grad(const void *dout, int dtype, int T, int64_t ld, const int32_t *tokens, int V, int H,
                        float scale, void *dtable, int out_dtype, int64_t ld_out, int accumulate, void *ws,
                        size_t ws_bytes, void *stream);

const char *ss_status_string(ss_status s);

#ifdef __cplusplus
}
#endif
#endif /* SS_H_ */
