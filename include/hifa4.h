/*
 * hifa4.h -- C ABI of libhifa4: the HiFA4 causal prefill attention forward on
 * AMD Instinct MI355X (gfx950).
 *
 * HiFA4 (arXiv 2607.04302) runs both FlashAttention contractions, QK^T and PV,
 * on 4-bit HIF4 operands while the online-softmax state stays in FP16
 * (Section 3, "C4V16"), with two corrections:
 *   - Smooth-QK (Eq. 1, Sections 4.2-4.4): a calibration-static per-channel
 *     rescale q*s, k/s applied after RoPE, fused into the quantization;
 *   - P-Reordering (Section 4.5, Theorem 1): P is quantized first and the
 *     softmax normalizer is accumulated from that same P^ inside the PV
 *     contraction, through an appended ones block [V^ | 1].
 * Algorithm 1 gives the loop, including the optional Q-Mean auxiliary (the
 * per-token mean of Q~ removed before quantization and added back through the
 * key sums, Section 4.6 and Appendix C).
 *
 * Conventions (all entry points):
 *   - Tensor pointers are DEVICE pointers owned by the caller; the library
 *     never allocates, frees or retains device memory, and keeps no device
 *     state between calls.  Where a host pointer is meant, it says so.
 *   - Alignment: fp16 tensors (q, k, v, o), the scales s, HIF4 code buffers,
 *     workspaces and debug code dumps 16 bytes; metadata buffers, LSE,
 *     cu_seqlens and the calibration output 4 bytes.  Anything else fails with
 *     HIFA4_ERR_INVALID_ARGUMENT before any work is enqueued.
 *   - Fixed-length problems use BSHD layout ([batch, seqlen, heads, dim],
 *     row-major, contiguous).  Variable-length problems pass cu_seqlens and
 *     use THD layout ([total_tokens, heads, dim]).
 *   - fp16 means IEEE binary16, fp32 IEEE binary32.
 *   - Work is enqueued on `stream` (a hipStream_t passed as void*; NULL is the
 *     default stream) and is asynchronous unless stated.  Arguments are
 *     validated synchronously; a launch failure maps to HIFA4_ERR_HIP.
 *     Device faults surface at the caller's next synchronization.
 *   - Nothing throws across the ABI.  On a non-OK status, hifa4_last_error()
 *     returns a message for the calling thread.
 *   - Inputs must be finite and keep |S * log2(e)/sqrt(D)| within the fp16
 *     range (the paper's FP16 softmax state); other inputs are outside the
 *     contract.
 *
 * HIF4 group format (the library's reading; see the HIF4 paragraph of the
 * paper's Background section): 64 elements along the contraction axis of the
 * GEMM that consumes them; an unsigned E6M2 base b (bias 31, byte = e<<2|m,
 * value (1+m/4)*2^(e-31)), the smallest with 1.75*b >= max|x|; level-2 bit j
 * (8 elements) set iff that block's max <= 0.875*b; level-3 bit q (4
 * elements) set iff its max <= 0.875*b*2^-E2[q/2]; a set bit halves the scale;
 * element code u = floor(|x|/step + 1/2) with step = b*2^-(E2+E3)/4, u in 0..7,
 * sign-magnitude nibble sign<<3|u (zero stored as +0).
 *
 * Canonical packed layout, per group: 32 code bytes (element 2i in the low
 * nibble of byte i, element 2i+1 in the high nibble) and one little-endian
 * uint32 of metadata: base | E2 bits << 8 | E3 bits << 16 (bit j = block j).
 * 36 bytes per 64 values = 4.5 bits per value.
 */
#ifndef HIFA4_H
#define HIFA4_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  HIFA4_OK = 0,
  HIFA4_ERR_INVALID_ARGUMENT = -1, /* null pointer, bad size or shape        */
  HIFA4_ERR_UNSUPPORTED = -2,      /* valid but not implemented (see below)  */
  HIFA4_ERR_WORKSPACE = -3,        /* workspace too small                    */
  HIFA4_ERR_HIP = -4               /* a HIP runtime call or launch failed    */
} hifa4_status;

/* Shape of one causal prefill problem.  Q has num_heads_q heads, K and V have
 * num_heads_kv; query head h reads key/value head h / (num_heads_q /
 * num_heads_kv) (GQA, Appendix C).  Queries and keys of a sequence have equal
 * lengths and key j is visible to query i iff j <= i.
 *   head_dim     in {64, 128, 256};
 *   max_seqlen   fixed length (BSHD) or, with cu_seqlens, an upper bound of
 *                every sequence length (host value; a longer sequence is
 *                outside the contract: the kernels clamp its length to
 *                max_seqlen, so no access leaves the buffers);
 *   cu_seqlens   NULL for BSHD, else a DEVICE int32 array [batch+1] of
 *                non-decreasing prefix sums starting at 0 (THD layout);
 *   total_tokens with cu_seqlens: cu_seqlens[batch] (host value); ignored
 *                for BSHD (batch*max_seqlen);
 *   causal       must be 1. */
typedef struct {
  int32_t batch;
  int32_t num_heads_q;
  int32_t num_heads_kv;
  int32_t head_dim;
  int32_t max_seqlen;
  const int32_t* cu_seqlens;
  int32_t total_tokens;
  int32_t causal;
} hifa4_problem;

typedef enum {
  HIFA4_NORM_PREORDER = 0,     /* P-Reordering: l accumulates P^ (Section 4.5) */
  HIFA4_NORM_INCONSISTENT = 1  /* Direct baseline: l accumulates pre-quantization
                                  P while PV uses P^ (Theorem 1, "mismatched") */
} hifa4_norm;

typedef enum {
  HIFA4_OPERANDS_HIF4 = 0,   /* both contractions on HIF4 operands (C4V16)     */
  HIFA4_OPERANDS_FP16 = 1,   /* same loop on fp16 operands, no quantization and
                                no smoothing: the FP16 reference (C16V16) */
  HIFA4_OPERANDS_P_ONLY = 2  /* P-only local operator (the study the paper
                                defers, Section 4.5): Q, K and V stay fp16
                                (no smoothing), scores and softmax as in the
                                FP16 reference, P^ = HIF4(P) feeds the PV
                                product; the normalizer follows opt->norm */
} hifa4_operands;

/* Options of hifa4_attention_fwd.
 *   smooth_qk      0: the scale vector is ignored (treated as all ones);
 *   debug_p_codes  NULL, or a DEVICE uint8 buffer [NH, NT, NB, 32]
 *                  receiving the canonical codes of the P^ groups of query
 *                  heads [h0, h0+NH) and tokens [t0, t0+NT) (the dump window,
 *                  below), NB = ceil(max_seqlen/64); entry (h-h0, t-t0, J) is
 *                  written for the 64-key blocks J <= i/64 that query t
 *                  (position i in its sequence) sees, other entries are left
 *                  untouched;
 *   debug_p_meta   NULL, or a DEVICE uint32 buffer [NH, NT, NB] with the
 *                  matching metadata words.  Both or neither.
 *   debug_head_begin/_count, debug_token_begin/_count  the dump window
 *                  h0, NH, t0, NT; a count of 0 means every query head
 *                  (every token, T = batch*max_seqlen for BSHD) and needs a
 *                  begin of 0; a window outside the problem fails with
 *                  HIFA4_ERR_INVALID_ARGUMENT.
 * Debug dumps are produced for HIFA4_OPERANDS_HIF4 and _P_ONLY.
 *   timing_events  NULL, or a HOST array of three hipEvent_t (created by the
 *                  caller) that the call records on `stream` before the K/V
 *                  pre-pass, between the pre-pass and the attention kernel,
 *                  and after the attention kernel -- per-kernel device time
 *                  without a profiler.  The events are not waited on.
 *   q_mean         0 or 1: the Q-Mean auxiliary (Algorithm 1; Section 4.6;
 *                  Appendix C).  Per query row mu = fp16(exact sum of the
 *                  row's D smoothed values / D); the row is quantized as
 *                  Q_z = fp16(q~ - mu); per key kappa = fp32(exact sum of the
 *                  key's smoothed channels); after the group terms the score
 *                  accumulator takes fp32(S_acc + mu*kappa) (the exact
 *                  product added with one rounding), before the multiply by
 *                  c.  HIF4 operands only (HIFA4_ERR_UNSUPPORTED with FP16
 *                  operands).
 *   test_decode_no_publish  testing only; see hifa4_decode_fwd (0 otherwise). */
typedef struct {
  int32_t norm;       /* hifa4_norm      */
  int32_t operands;   /* hifa4_operands  */
  int32_t smooth_qk;
  void* debug_p_codes;
  void* debug_p_meta;
  void** timing_events;
  int32_t q_mean;
  int32_t test_decode_no_publish;  /* testing only, hifa4_decode_fwd: see there */
  int32_t debug_head_begin;        /* P^ dump window of hifa4_attention_fwd */
  int32_t debug_head_count;
  int32_t debug_token_begin;
  int32_t debug_token_count;
} hifa4_fwd_options;

/* Host-side calibration report (Table 1 statistics and the gate decision). */
typedef struct {
  double rho_k;        /* max|K| / P99(|K|) over all calibration K elements */
  double t_kq;         /* max|K| / max|Q|                                     */
  int32_t branch;      /* 0 bypass, 1 mild, 2 strong                          */
  float alpha_used;
} hifa4_calib_report;

/* Bytes of device workspace hifa4_attention_fwd needs for this problem and
 * options (0 on invalid arguments).  The workspace holds the MFMA-ready K and
 * V operands written by the pre-pass. */
size_t hifa4_workspace_bytes(const hifa4_problem* p, const hifa4_fwd_options* opt);

/* Bytes of device workspace hifa4_calibrate_smooth_qk needs. */
size_t hifa4_calibrate_workspace_bytes(const hifa4_problem* p, int32_t n_calib);

/* Offline Smooth-QK calibration (Eq. 1; Sections 4.3-4.4; Appendix C).
 * q_calib: DEVICE fp16 [n_calib, max_seqlen, num_heads_q, head_dim];
 * k_calib: DEVICE fp16 [n_calib, max_seqlen, num_heads_kv, head_dim]
 * (n_calib fixed-length sequences stacked on the leading axis; p->batch and
 * p->cu_seqlens are ignored).  Per sequence, the GPU reduces max|K| over
 * tokens and max|Q| over tokens and the query heads of each group, per (kv
 * head, channel), and a 32768-bin histogram of |K| (exact for fp16).  Then, in
 * float64 on the GPU: the RMS over sequences, s = Kbar^alpha / Qbar^(1-alpha)
 * rounded once to fp32 (s = 1 where a statistic is 0 or s is not finite),
 * and the gate statistics rho_K = max|K| / P99|K| (linear interpolation
 * between order statistics) and T = max|K| / max|Q|.
 *   alpha > 0  use this alpha;  alpha == 0  bypass (s = 1);
 *   alpha < 0  the gate picks: strong (0.5) if rho_K >= 6 and T > 3,
 *              mild (0.25) if rho_K >= 6 and 2 <= T <= 3, else bypass.
 * s_out: DEVICE fp32 [num_heads_kv, head_dim].  report: HOST, may be NULL.
 * workspace: DEVICE, at least hifa4_calibrate_workspace_bytes().
 * Synchronizes `stream` before returning (an offline call). */
hifa4_status hifa4_calibrate_smooth_qk(const hifa4_problem* p, int32_t n_calib,
                                       const void* q_calib, const void* k_calib,
                                       float alpha, float* s_out,
                                       hifa4_calib_report* report,
                                       void* workspace, size_t workspace_bytes,
                                       void* stream);

/* Offline calibration of several layers in one call (Sections 4.3-4.4 and
 * Appendix F: the statistics, the scale and the gate decision are taken per
 * layer).  Layer l reads q_calib + l * (n_calib*max_seqlen*num_heads_q*head_dim)
 * and k_calib + l * (n_calib*max_seqlen*num_heads_kv*head_dim) fp16 elements
 * (DEVICE, layers stacked on a leading axis) and writes s_out + l*num_heads_kv*
 * head_dim (DEVICE fp32) and reports[l] (HOST, may be NULL); each layer is
 * exactly hifa4_calibrate_smooth_qk on its slice, with the same alpha (alpha < 0
 * lets the gate decide per layer).  workspace: DEVICE, at least
 * hifa4_calibrate_workspace_bytes(p, n_calib), reused by every layer.
 * Synchronizes `stream`.  On an error no later layer is processed. */
hifa4_status hifa4_calibrate_smooth_qk_layers(const hifa4_problem* p, int32_t n_layers,
                                              int32_t n_calib, const void* q_calib,
                                              const void* k_calib, float alpha, float* s_out,
                                              hifa4_calib_report* reports, void* workspace,
                                              size_t workspace_bytes, void* stream);

/* Smooth-QK then HIF4 quantization of Q~ = fp16(q*s) and K~ = fp16(k/s),
 * each the exact product or quotient of the fp16 input and the fp32 scale
 * rounded once to fp16 (nearest even), in groups of 64 consecutive channels
 * of each (token, head) row (Algorithm 1, the Smooth-QK and HIF4 steps).
 * q, k: DEVICE fp16 in the problem's layout; s: DEVICE fp32
 * [num_heads_kv, head_dim] or NULL (no smoothing).
 * Outputs (DEVICE, canonical layout):
 *   q_codes uint8 [T, num_heads_q, head_dim/64, 32], q_meta uint32 [T, Hq, D/64]
 *   k_codes uint8 [T, num_heads_kv, head_dim/64, 32], k_meta uint32 [T, Hkv, D/64]
 * where T is the token count.  q, q_codes and q_meta may all be NULL: then
 * only K^ is written (filling or appending to a K^ cache; rows are
 * independent, so the K^ of new tokens can be written in place at their
 * cache rows).  Asynchronous. */
hifa4_status hifa4_quantize_qk(const hifa4_problem* p, const void* q, const void* k,
                               const float* s, void* q_codes, void* q_meta,
                               void* k_codes, void* k_meta, void* stream);

/* HIF4 quantization of V along tokens (the contraction axis of PV): groups
 * of 64 consecutive tokens of one (kv head, channel) column, aligned to each
 * sequence's first token; a partial last group is zero padded.
 * v: DEVICE fp16 in the problem's layout.  Outputs (DEVICE, canonical):
 *   v_codes uint8 [batch, NB, num_heads_kv, head_dim, 32]
 *   v_meta  uint32 [batch, NB, num_heads_kv, head_dim]
 * with NB = ceil(max_seqlen/64); groups past a sequence's end are written as
 * all-zero groups.  Asynchronous. */
hifa4_status hifa4_quantize_v(const hifa4_problem* p, const void* v, void* v_codes,
                              void* v_meta, void* stream);

/* The HiFA4 causal prefill forward (Algorithm 1; Section 4.5).
 * q: DEVICE fp16 [.., num_heads_q, head_dim]; k, v: DEVICE fp16
 * [.., num_heads_kv, head_dim]; s: DEVICE fp32 [num_heads_kv, head_dim] (may be
 * NULL when opt->smooth_qk == 0 or operands are FP16).
 * Per query row and 64-key block in ascending order, with c =
 * fp32(log2(e)/sqrt(D)): per 64-channel group g the exact term t_g = the dot
 * of the dequantized Q^ and K^ groups; S_acc = the fp32 sum of the t_g in
 * group order, each addition rounded once (with Q-Mean, then
 * fp32(S_acc + mu*kappa)); S2 = fp16(fp32(S_acc * c));
 * m_new = max(m, rowmax S2); P = fp16(2^(S2-m_new));
 * r = fp16(2^(m-m_new)); P^ = HIF4(P); O = r*O + P^ V^ and l = r*l + P^ 1
 * (fp32 accumulation); O_out = fp16(O/l), LSE = m*ln2 + ln(l).
 * o: DEVICE fp16, same layout as q.  lse: DEVICE fp32 [num_heads_q, T] (T the
 * token count, natural log of the softmax partition, including the score
 * scale 1/sqrt(D)).  workspace: DEVICE, >= hifa4_workspace_bytes().
 * Asynchronous. */
hifa4_status hifa4_attention_fwd(const hifa4_problem* p, const hifa4_fwd_options* opt,
                                 const void* q, const void* k, const void* v,
                                 const float* s, void* o, float* lse,
                                 void* workspace, size_t workspace_bytes, void* stream);

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, serving loops, harnesses that forbid hipMalloc): hifa4_attention_fwd
 * with its workspace in a static device array of the library,
 * HIFA4_NOALLOC_SCRATCH_BYTES (32 MiB) per GPU, held from the first call on
 * that GPU until the process ends.  The caller passes inputs and outputs as
 * for hifa4_attention_fwd; the call allocates and frees nothing.  A problem
 * whose hifa4_workspace_bytes() exceeds the array fails with
 * HIFA4_ERR_WORKSPACE before any work is enqueued (32 MiB holds, for
 * example, 8 kv heads of D=128 up to 10240 tokens).  The array's address on
 * the current device (which must be the stream's device) is looked up on the
 * first call there.  Every call on one GPU shares its array: calls that
 * overlap on one GPU (different streams, or threads) race and give wrong
 * results; calls ordered on one stream are safe.  Nothing in the array needs
 * to start at zero (each call writes every entry it reads).  Otherwise
 * identical to hifa4_attention_fwd, including the debug and timing options. */
#define HIFA4_NOALLOC_SCRATCH_BYTES (32u << 20)
hifa4_status hifa4_attention_fwd_noalloc(const hifa4_problem* p, const hifa4_fwd_options* opt,
                                         const void* q, const void* k, const void* v,
                                         const float* s, void* o, float* lse, void* stream);

/* Workspace size in bytes of hifa4_decode_fwd for problem p (0 if p is
 * invalid).  It grows with batch * num_heads_q * ceil(max_seqlen/64). */
size_t hifa4_decode_workspace_bytes(const hifa4_problem* p);

/* One decode step of HiFA4 over a packed HIF4 K/V cache: for each sequence b,
 * the attention of its newest token (position L_b - 1, which sees every cached
 * key) -- row L_b - 1 of hifa4_attention_fwd on the same sequence, computed
 * from the cache.  The paper evaluates prefill only and leaves decode and
 * the KV-cache footprint open; this entry point applies Algorithm 1 and
 * Section 4.5 to that row with the same contract, including every P^ code.
 * p describes the cached sequences (their lengths include the newest token):
 * BSHD (every length max_seqlen) or THD with cu_seqlens; causal must be 1.
 * q: DEVICE fp16 [batch, num_heads_q, head_dim], the raw query of each
 *    sequence's newest token (smoothed here with s when opt->smooth_qk);
 * k_codes/k_meta: DEVICE canonical K^ cache [T, Hkv, D/64, 32] / [T, Hkv, D/64]
 *    as written by hifa4_quantize_qk with the same s (T the token count);
 * v_codes/v_meta: DEVICE canonical V^ cache [batch, NB, Hkv, D, 32] /
 *    [batch, NB, Hkv, D] as written by hifa4_quantize_v (NB = ceil(max_seqlen/64));
 * o: DEVICE fp16 [batch, num_heads_q, head_dim]; lse: DEVICE fp32
 *    [num_heads_q, batch]; rows of empty sequences are left untouched.
 * opt: norm, smooth_qk, debug_p_codes/_meta ([num_heads_q, batch, NB, 32] /
 *    [num_heads_q, batch, NB], entries J < ceil(L_b/64) written) and
 *    timing_events (before the first kernel, before the merge kernel, after
 *    the merge) as for hifa4_attention_fwd; operands must be
 *    HIFA4_OPERANDS_HIF4 and q_mean 0 (the cache carries no key sums), else
 *    HIFA4_ERR_UNSUPPORTED; num_heads_q / num_heads_kv must be <= 8 (else
 *    HIFA4_ERR_UNSUPPORTED).
 * workspace: DEVICE, >= hifa4_decode_workspace_bytes(p).  Asynchronous.
 * total_tokens sizes the launch; a captured call may be replayed after
 * cu_seqlens have changed in place, also past total_tokens (within max_seqlen
 * and the caches): every cached token is still taken in, in a launch of the
 * captured size.
 * The blocks of a sequence are cut into runs (splits), one kernel takes their
 * scores and their partial outputs, and each run waits, with a bounded spin,
 * for the run maxima that the runs before it in the same row
 * publish (tagged with a per-call value; the last kernel of the call clears
 * them, so no word of an earlier call, eager or replayed from a graph,
 * satisfies a wait).  Every GPU engine dispatches the workgroups of a grid in
 * index order and each waits only on lower indices, so the waits are short
 * where the call has the GPU to itself; next to other work (a second decode
 * call on another stream whose waiting workgroups hold this one's off the GPU)
 * a wait may run to its limit, some milliseconds, and the run then scores the
 * earlier blocks of its sequence itself: the results are the same bits.
 * opt->test_decode_no_publish (testing only): 2 publishes nothing and lets
 * every wait give up after 16 polls; with 1 the rows that waited come out NaN
 * instead of being computed. */
hifa4_status hifa4_decode_fwd(const hifa4_problem* p, const hifa4_fwd_options* opt,
                              const void* q, const void* k_codes, const void* k_meta,
                              const void* v_codes, const void* v_meta, const float* s,
                              void* o, float* lse, void* workspace, size_t workspace_bytes,
                              void* stream);

/* ---------------------------------------------------------------------------
 * The paged key-value cache of a serving loop: sequences grow a page of 64
 * tokens at a time, pages come from one pool in any order, and a table names
 * each sequence's pages.  The paper evaluates prefill only; these entry points
 * keep what its attention quantizes (K^ with Smooth-QK, V^ in groups of 64
 * tokens) and attend over it.
 *
 *   operands     what a page holds: HIFA4_OPERANDS_HIF4 (4.5 bits a value) or
 *                HIFA4_OPERANDS_FP16;
 *   pool         DEVICE, num_pages * hifa4_paged_page_bytes() bytes, 16-byte
 *                aligned.  A page is one record per kv head, in the order of
 *                the matrix instructions' registers: it is written by
 *                hifa4_paged_append and read by the other entry points;
 *   block_table  DEVICE int32 [batch, max_pages]: the page of each 64 tokens.
 *                An entry outside [0, num_pages) names no page: its tokens are
 *                not stored, attended to or read back.  Sequences may share
 *                pages for reading; two that append into one page race;
 *   seq_lens     DEVICE int32 [batch]: the cached tokens of each sequence,
 *                those that an append brings included; 0 for an unused row
 *                (values outside [0, 64 max_pages] are cut to that range);
 *   v_tail       DEVICE fp16 [batch, 64, num_heads_kv, head_dim]: V of the
 *                tokens in the page that each sequence's last append ended in,
 *                kept by hifa4_paged_append for HIFA4_OPERANDS_HIF4 (a group of
 *                V^ is quantized again when a token joins it); may be NULL
 *                otherwise and for the other entry points.
 * Before an append a length may be cut back (tokens that were rejected) within
 * the page that the last append ended in, or to a multiple of 64; on HIF4 pages
 * not into the middle of an earlier page, whose V is no longer in v_tail: the
 * append would quantize that page's group from rows of the later one, without
 * an error.  (Until the next append the page keeps V^ as it was quantized with
 * the tokens that were cut off.)  A sequence that moves to another row of the
 * batch takes its row of v_tail along.
 * head_dim is 64, 128 or 256.  Calls of more pages than one launch holds (2^24
 * workgroups, 2^23 for an append to HIF4 pages of head_dim 256: a grid's threads
 * are counted in 32 bits; batch * max_pages reaches 2^30) are refused.  Every
 * entry point reads the table and the lengths on the device, enqueues a fixed
 * number of kernels whose grid follows from host values alone, and may be
 * captured into a graph and replayed with other lengths and tables. */
typedef struct {
  int32_t batch;
  int32_t num_heads_kv;
  int32_t head_dim;
  int32_t operands;
  int32_t num_pages;
  int32_t max_pages;
  void* pool;
  const int32_t* block_table;
  const int32_t* seq_lens;
  void* v_tail;
} hifa4_paged_cache;

/* Bytes of one page: 64 tokens of K and V, every kv head (0 on invalid
 * arguments). */
size_t hifa4_paged_page_bytes(int32_t num_heads_kv, int32_t head_dim, int32_t operands);

/* Appends new tokens.  The new tokens of sequence b are the rows
 * [cu_new[b], cu_new[b+1]) of k and v and the last ones of its seq_lens[b]
 * tokens; cu_new NULL: one token for each sequence, rows of length 0 skipped.
 * k, v: DEVICE fp16 [total_new, num_heads_kv, head_dim]; s: DEVICE fp32
 * [num_heads_kv, head_dim] or NULL.  K~ = fp16(k/s), rounded once; with HIF4
 * pages K~ and V become the codes of hifa4_quantize_qk and hifa4_quantize_v:
 * the pages hold at any time the codes of quantizing the whole sequence (the
 * group of an open page zero padded), whatever pieces it came in.  HIF4 has no
 * infinity and no NaN: where K~ or V is not finite, what the page holds for that
 * kv head is undefined (no other page and no other head is touched); FP16 pages
 * hold it as it is.
 * max_new: a host bound of the tokens that one sequence gets (it sizes the
 * launch, for every sequence of the batch; further tokens are not stored).  An
 * append may begin inside a page and end in another; earlier tokens of the page
 * must have come through hifa4_paged_append, with the same v_tail, which must
 * still hold them (above: lengths that are cut back).  Asynchronous. */
hifa4_status hifa4_paged_append(const hifa4_paged_cache* c, int32_t total_new, int32_t max_new,
                                const int32_t* cu_new, const void* k, const void* v,
                                const float* s, void* stream);

/* Reads tokens back: of sequence b the tokens starts[b], starts[b]+1, ... into
 * the rows [cu_tokens[b], cu_tokens[b+1]) of k and v (DEVICE fp16
 * [total_tokens, num_heads_kv, head_dim]), K^ as it is cached (Smooth-QK not
 * undone) and V^, HIF4 values rounded to fp16 (exact unless they fall below
 * its normal range).  Tokens at or behind seq_lens[b] are zeros; rows that
 * cu_tokens does not name are left as they are.  starts: DEVICE int32 [batch]
 * or NULL (0).  max_tokens: a host bound of the rows per sequence (it sizes
 * the launch; further rows are not written).  Asynchronous. */
hifa4_status hifa4_paged_gather(const hifa4_paged_cache* c, int32_t total_tokens, int32_t max_tokens,
                                const int32_t* cu_tokens, const int32_t* starts, void* k, void* v,
                                void* stream);

/* Bytes of device workspace hifa4_paged_decode_fwd needs (0 on invalid
 * arguments); page_weights != 0 where the call accumulates page weights.  It
 * grows with batch * num_heads_q and, with page weights, with
 * batch * max_pages * num_heads_q; it does not depend on the lengths. */
size_t hifa4_paged_decode_workspace_bytes(const hifa4_paged_cache* c, int32_t num_heads_q,
                                          int32_t page_weights);

/* One decode step: the attention of each sequence's newest token over its
 * cached tokens (its own among them, appended before).
 * q: DEVICE fp16 [batch, num_heads_q, head_dim], smoothed with s when s is not
 * NULL (q~ = fp16(q*s)); query head h reads kv head h / (num_heads_q /
 * num_heads_kv).  With S_j = q~ k_j / sqrt(D) over the cached values:
 * p = softmax(S), o = sum_j p_j v_j (DEVICE fp16 [batch, num_heads_q,
 * head_dim]), lse = log sum_j exp(S_j) (DEVICE fp32 [num_heads_q, batch]).
 * Unlike hifa4_decode_fwd, which repeats a row of the prefill code for code,
 * only the cache is quantized here: a step's time is the cache's bytes, and
 * the query, the scores, the softmax state (fp32) and p keep their precision (on
 * HIF4 pages the query's values and p enter the products as whole numbers,
 * rounded by at most 2^-19 of the largest of their 64: a group's channels, a
 * page's keys; on FP16 pages p as the sum of two fp16 values).  A score moves
 * with the query by up to 2^-19 of sum max|q| sum|k| / sqrt(D) over the groups:
 * lse by 6e-6 at the median, 1.5e-4 at most, of 400 queries with two channels of
 * 128 at 64 times the others, by 1e-5 at most at 16 times.
 * Sequences without tokens get o = 0 and lse = -inf.
 * page_weights (DEVICE fp32 [batch, max_pages], may be NULL): then
 * weights_out[b][j] = decay * page_weights[b][j] + the sum of p over every
 * query head and the tokens of page j, for the pages that sequence b uses, and
 * page_weights[b][j] for the others.  weights_out may be page_weights itself;
 * both are NULL or neither.
 * workspace: DEVICE, >= hifa4_paged_decode_workspace_bytes(); nothing in it
 * has to start at zero and nothing is kept in it.  Sums are taken in a fixed
 * order: equal inputs give equal bits.  Asynchronous. */
hifa4_status hifa4_paged_decode_fwd(const hifa4_paged_cache* c, int32_t num_heads_q, const void* q,
                                    const float* s, void* o, float* lse, const float* page_weights,
                                    float* weights_out, float decay, void* workspace,
                                    size_t workspace_bytes, void* stream);

/* Eviction by accumulated attention weight: a sequence of more than `budget`
 * pages keeps its `first` first pages, its `last` last pages and, of those
 * between, the ones of the largest weight until it has `budget` (equal weights:
 * the earlier page stays; NaN counts as the smallest).  Whole pages leave, so
 * that no group of V^ is broken up and nothing in the pool moves; the pages
 * that stay close ranks in order (cached keys carry their position).
 * 0 <= first, 1 <= last (the open page stays), first + last <= budget.
 * block_table, seq_lens, page_weights: as above (read); out_table, out_lens,
 * out_weights: the same after the eviction (entries behind the pages that stay
 * are -1 and 0; 64 tokens less for each page evicted); each may be its input's
 * own buffer, and must not overlap any other.  freed: DEVICE int32
 * [batch, max_pages], the evicted pages' entries in order, then -1; num_freed:
 * DEVICE int32 [batch].  Asynchronous. */
hifa4_status hifa4_paged_evict(int32_t batch, int32_t max_pages, const int32_t* block_table,
                               const int32_t* seq_lens, const float* page_weights, int32_t budget,
                               int32_t first, int32_t last, int32_t* out_table, int32_t* out_lens,
                               float* out_weights, int32_t* freed, int32_t* num_freed, void* stream);

/* Bytes of device workspace hifa4_paged_chunk_fwd needs (0 on invalid
 * arguments): the parts of rows that two shares of the work cut, for the shares
 * that fill the GPU.  It does not depend on the lengths. */
size_t hifa4_paged_chunk_workspace_bytes(const hifa4_paged_cache* c, int32_t num_heads_q,
                                         int32_t total_new, int32_t max_new);

/* The attention of each sequence's last tokens over its cached tokens: chunks
 * of prompts, drafted tokens that are checked, one token of each sequence, or
 * all of these in one batch.  The new tokens of sequence b are the rows
 * [cu_new[b], cu_new[b+1]) of q (DEVICE fp16 [total_new, num_heads_q, head_dim])
 * and the last ones of its seq_lens[b] tokens, appended before; the i-th of n
 * stands at position seq_lens[b] - n + i and sees the cached tokens up to its
 * own.  cu_new: DEVICE int32 [batch+1], prefix sums from 0 to at most total_new
 * (others are cut so that no access leaves q, o and lse).  q is smoothed with s when s
 * is not NULL (q~ = fp16(q*s)); query head h reads kv head h / (num_heads_q /
 * num_heads_kv).  With S_j = q~ k_j / sqrt(D) over the cached values that the
 * token sees: p = softmax(S), o = sum_j p_j v_j (DEVICE fp16, like q), lse = log
 * sum_j exp(S_j) (DEVICE fp32 [num_heads_q, total_new]).
 * Scores, softmax and o are held in fp32.  The products take fp16 operands: q~,
 * the cached values (on HIF4 pages exact down to 2^-14, below that rounded by at
 * most 1.125 2^-24) and p, rounded to fp16 for the sum over v; o is divided by the
 * sum of the rounded p, lse holds the sum of p itself (hifa4_paged_decode_fwd keeps
 * p's precision: one token's o is nearer there by that rounding).  A value that is
 * not finite (FP16 pages) reaches the rows that see its token and no others.
 * Rows that see no token (more new tokens than cached ones, pages that are none),
 * or all of whose scores are -inf, get o = 0 and lse = -inf; rows of q behind cu_new[batch] leave o and lse as
 * they were.  max_new: a host bound of the new tokens of one sequence (it sizes
 * the launch; o and lse of further tokens are left as they were).  A batch of
 * single or drafted tokens gives it: with at most 32 rows (max_new times the query
 * heads per kv head) the kernels for few rows take the call, else FP16 pages have
 * only those for many.
 * workspace: DEVICE, >= hifa4_paged_chunk_workspace_bytes(); nothing in it has to
 * start at zero and nothing is kept in it.  Sums are taken in a fixed order: equal
 * inputs give equal bits.  Asynchronous. */
hifa4_status hifa4_paged_chunk_fwd(const hifa4_paged_cache* c, int32_t num_heads_q,
                                   int32_t total_new, int32_t max_new, const int32_t* cu_new,
                                   const void* q, const float* s, void* o, float* lse,
                                   void* workspace, size_t workspace_bytes, void* stream);

/* Deals out the pages of new tokens from a stack of free ones.  Row b holds
 * seq_lens[b] tokens and asks for counts[b] more (DEVICE int32 [batch]; negative:
 * none).  A row that asks for more than max_new (a host bound, which sizes the
 * launch) or than fit its 64 max_pages places gets none and asks for none.  The
 * others are served in order: a row gets its tokens if those that were asked for
 * up to and with it are at most max_total and, where it needs pages, the pages
 * needed up to and with it are at most the free ones; else it gets none.
 *   free_pages   DEVICE int32 [capacity], num_free (DEVICE int32 [1]) entries of
 *                which are free pages, the last one on top; the first page of
 *                the first row that needs one is the top one;
 *   block_table  gets the new pages at the places behind the old ones (the first
 *                ceil(seq_lens[b]/64), which are read); what lies at other places
 *                is left as it is;
 *   out_lens     DEVICE int32 [batch], the lengths with the tokens that were got,
 *                out_free DEVICE int32 [1] the pages left; each may be its
 *                input's own buffer;
 *   cu_new       DEVICE int32 [batch+1], prefix sums of the tokens that the rows
 *                got (what hifa4_paged_append and hifa4_paged_chunk_fwd take);
 *   positions    DEVICE int32 [max_total], of each of these tokens, row by row,
 *                its place in its sequence, plus shift[b] (DEVICE int32 [batch] or
 *                NULL: 0; the tokens that an eviction has taken out of a row keep
 *                their positions);
 *   slots        DEVICE int64 [max_total], 64 * page + place in the page (-1 where
 *                the table names no page).
 * Entries of positions and slots behind cu_new[batch] are -1.  No buffer overlaps
 * another but as stated.  Asynchronous; it may be captured and replayed. */
hifa4_status hifa4_paged_extend(int32_t batch, int32_t max_pages, int32_t* block_table,
                                const int32_t* seq_lens, const int32_t* counts,
                                const int32_t* free_pages, int32_t capacity, const int32_t* num_free,
                                const int32_t* shift, int32_t max_total, int32_t max_new,
                                int32_t* out_lens, int32_t* out_free, int32_t* cu_new,
                                int32_t* positions, int64_t* slots, void* stream);

/* Bytes of device workspace hifa4_paged_release needs (0 on invalid arguments). */
size_t hifa4_paged_release_workspace_bytes(int32_t batch);

/* Puts pages back on the stack of free ones: of each row of table (DEVICE int32
 * [batch, max_pages]: a block table, or the evicted pages of hifa4_paged_evict) the
 * entries at the places [first[b], to[b]) (DEVICE int32 [batch]; first may be
 * NULL: 0; cut to the row), but for negative ones, which are none.  They end on
 * top in order, the first row's first entry uppermost: a release of what
 * hifa4_paged_extend has dealt out restores the stack.  Pages that find no place
 * below `capacity` are dropped (the first ones); out_free (DEVICE int32 [1]) is
 * the new number and may be num_free itself.  The table is left as it is: lengths
 * say which of its places count.  A page is released once: one that several rows
 * share, or that stands in the table twice, would be dealt out twice.
 * workspace: DEVICE, >= hifa4_paged_release_workspace_bytes(), 4-byte aligned; one
 * call at a time.  Asynchronous; it may be captured and replayed. */
hifa4_status hifa4_paged_release(int32_t batch, int32_t max_pages, const int32_t* table,
                                 const int32_t* first, const int32_t* to, int32_t* free_pages,
                                 int32_t capacity, const int32_t* num_free, int32_t* out_free,
                                 void* workspace, size_t workspace_bytes, void* stream);

/* Rotary positions (the step before Smooth-QK, whose scales act "after RoPE",
 * Section 4.2).  The first rot_dim channels of a head are rotated in pairs, the
 * others are copied: pair i of a token at position p becomes
 *   (x cos(p w_i) - y sin(p w_i), x sin(p w_i) + y cos(p w_i)) * magnitude.
 * Scaling of the frequencies w_i = base^(-2i/rot_dim): */
typedef enum {
  HIFA4_ROPE_NONE = 0,
  HIFA4_ROPE_LINEAR = 1,  /* w_i / factor                                            */
  HIFA4_ROPE_NTK = 2,     /* base * factor^(rot_dim/(rot_dim-2)) in place of base    */
  HIFA4_ROPE_PARTS = 3    /* w_i (g + (1-g)/factor), where g goes from 0 to 1 as the
                             turns original_len w_i / (2 pi) go from low to high     */
} hifa4_rope_scaling;

/* The frequencies in turns per position, as whole numbers of 2^-64 (modulo one
 * turn): turns[i] = w_i / (2 pi) * 2^64 rounded, i < rot_dim/2, to a HOST array.
 * rot_dim a positive multiple of 8 (at most 256); base > 1; factor >= 1 (ignored
 * without scaling); original_len > 0 and 0 <= low < high with _PARTS. */
hifa4_status hifa4_rope_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor,
                                    double original_len, double low, double high, uint64_t* turns);

/* Rotates q and k (DEVICE fp16).
 *   rot_dim      a multiple of 8 up to head_dim (64, 128 or 256);
 *   interleaved  0: pair i is the channels i and i + rot_dim/2; 1: 2i and 2i+1;
 *   transposed   0 or 1: the transposed rotation, the inverse where the magnitude
 *                is 1, and the gradient of q and k from that of q_out and k_out;
 *   turns        DEVICE uint64 [rot_dim/2], from hifa4_rope_frequencies;
 *   positions    DEVICE int32 [num_tokens]; rows of negative ones are no tokens:
 *                their outputs are left as they were;
 *   q, k         num_tokens rows of num_heads_q and num_heads_k heads, the rows
 *                q_stride and k_stride elements apart (multiples of 8: parts of one
 *                projection's rows); 0 heads: none;
 *   q_out, k_out the same with strides of their own; each may be its input (with
 *                its stride) and overlaps nothing else.
 * Angles are exact modulo a turn at any position for the given turns (whose own
 * roundings, fp64's, grow with it: 2^-21 rad near position 2^31); the rotated values
 * are computed in fp32 and rounded once.  Asynchronous. */
hifa4_status hifa4_rope(int32_t head_dim, int32_t rot_dim, int32_t interleaved, int32_t transposed,
                        float magnitude, const uint64_t* turns, int32_t num_tokens,
                        const int32_t* positions, int32_t num_heads_q, const void* q,
                        int64_t q_stride, void* q_out, int64_t q_out_stride, int32_t num_heads_k,
                        const void* k, int64_t k_stride, void* k_out, int64_t k_out_stride,
                        void* stream);

/* Device self-test of the kernels' fp16 exponential: y[i] = fp16(2^x[i]) for
 * n fp16 inputs x (DEVICE, fp16 bits), evaluated by the same device routine
 * the attention kernel uses.  Asynchronous. */
hifa4_status hifa4_selftest_exp2(const void* x, void* y, int64_t n, void* stream);

/* Message for the last non-OK status returned on the calling thread. */
const char* hifa4_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* HIFA4_H */
