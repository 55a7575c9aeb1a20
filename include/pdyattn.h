/*
 * pdyattn -- packed variable-length softmax attention, forward and backward,
 * for AMD Instinct MI355X (gfx950).
 *
 * The operation is scaled dot-product attention as written in Eq. (2) of the
 * problem formulation (section 3):  A = Softmax(Q K^T / sqrt(d)) V, applied per
 * head to a packed batch of dynamic-length sequences laid out as in the
 * tensor-layout specification (Table 2, section 4.2: activations b x s/p x h,
 * here packed to [T, H, d] with segment offsets).  The backward computes the
 * gradient of that expression, which the training workloads of section 5.1
 * need.  Readings of points the paper leaves open:
 *   - d is the head dimension (h/n of Table 4); the scale is an argument.
 *   - segments never attend to each other; with causal = 1 key j is visible
 *     to query i iff j <= i within the segment.
 *   - grouped heads: query head h reads key/value head h / (Hq / Hkv).
 *   - lse is the natural-log log-sum-exp of the scaled logits, [Hq, T].
 *
 * Conventions shared by every entry point:
 *   - All tensor pointers are DEVICE pointers owned by the caller; the library
 *     never allocates or frees device memory.  Dense, row-major, last dim
 *     contiguous, 16-byte aligned.  bf16 tensors are raw IEEE bfloat16 bits.
 *   - cu_seqlens is an int32 device array of num_seqs + 1 offsets with
 *     cu[0] = 0, cu[i] <= cu[i+1], cu[num_seqs] = total_tokens.  Zero-length
 *     segments are allowed.  Its contents are trusted (reading them on the
 *     host would force a synchronisation); attn_validate_cu_seqlens checks it.
 *   - max_seqlen must be >= every segment length (an upper bound suffices);
 *     with num_seqs = 1 it must equal total_tokens (the one segment is
 *     [0, T)), else the call returns PDY_ERR_INVALID_ARG.
 *   - Work is enqueued on `stream` (a hipStream_t; NULL = default stream) and
 *     the call returns without synchronising.  Outputs are fully overwritten.
 *   - Argument errors are reported before anything is launched.  A non-OK
 *     status leaves a thread-local message in pdy_last_error().
 *   - Scratch memory comes from the caller's `workspace` (16-byte aligned,
 *     at least the size the matching *_workspace_size query returns).
 *   - Calls on different streams with disjoint outputs and workspaces may run
 *     concurrently, except attn_bwd_noalloc calls on the same GPU (they share
 *     its static scratch array); the library holds no other global state
 *     besides per-thread error text, the optional per-thread kernel timing
 *     records and a one-time setup of kernel attributes.
 *   - Results are bitwise reproducible run to run (no atomics feed outputs).
 *   - Launches too small to fill the GPU (fewer than 512 work items, e.g. a
 *     single 8K-token sequence over 4 heads) split each item's work into
 *     parts (split-K) whose fp32 partial results are combined in a second
 *     kernel (2 or 4 parts per item, or, for a causal single sequence whose
 *     parts fit one round on the GPU, at most 16, more for the heavier items),
 *     or among groups of a workgroup's waves; and short or few segments take
 *     smaller workgroups.  This shape of a launch (pdy_launch_shapes) follows
 *     from its sizes -- total_tokens, num_seqs, max_seqlen and the head counts
 *     and dimension, so from the whole batch -- the causal flag (the workspace
 *     queries cover both values), a chunk pair's offsets and how many run at a
 *     time, and the workspace: one
 *     smaller than the query asks for is taken where it holds fewer parts (chunk
 *     pairs) or the shape without groups, and refused else.
 *   - Results depend on the shape in rounding only (which keys share an exponent
 *     offset, the order of fp32 sums; the error against exact arithmetic is the
 *     same).  A segment's results do not depend on the contents of the other
 *     segments of its batch, but they are bitwise those of the same segment
 *     alone, or in another batch, only where the launches have one shape without
 *     parts.
 *   - A row that sees a NaN or +inf logit gets o = NaN and lse = -inf.
 */
#ifndef PDYATTN_H
#define PDYATTN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  PDY_OK = 0,
  PDY_ERR_INVALID_ARG = -1, /* null/misaligned pointer, bad size or flag          */
  PDY_ERR_UNSUPPORTED = -2, /* head_dim not in {64, 128}                            */
  PDY_ERR_WORKSPACE = -3,   /* workspace smaller than the query function asks for */
  PDY_ERR_HIP = -4          /* a HIP runtime call failed (message has the detail) */
} pdy_status;

/* Bytes of workspace attn_fwd needs for these sizes (>= 256; for a split-K
 * launch it includes the parts' fp32 O and LSE, under 129 MiB).
 * Returns 0 when the sizes are invalid. */
size_t attn_fwd_workspace_size(int32_t total_tokens, int32_t num_seqs, int32_t max_seqlen,
                               int32_t num_heads_q, int32_t num_heads_kv, int32_t head_dim);

/* Bytes of workspace attn_bwd needs (it holds D = rowsum(dO * O), fp32
 * [Hq, T], the tile schedules and, for split-K launches, the parts' fp32
 * partial gradients, under 384 MiB).  Returns 0 when the sizes are
 * invalid. */
size_t attn_bwd_workspace_size(int32_t total_tokens, int32_t num_seqs, int32_t max_seqlen,
                               int32_t num_heads_q, int32_t num_heads_kv, int32_t head_dim);

/* Forward of Eq. (2) (section 3) over a packed batch.
 *   q   bf16 [T, Hq,  d]        k, v  bf16 [T, Hkv, d]
 *   o   bf16 [T, Hq,  d] (out)  lse   fp32 [Hq, T]    (out, natural log)
 *   num_heads_q % num_heads_kv == 0;  head_dim in {64, 128};  causal in {0, 1};
 *   scale finite and > 0 (usually 1/sqrt(head_dim)).
 * T = 0 is a no-op.  o and lse must not alias the inputs. */
pdy_status attn_fwd(const void* q, const void* k, const void* v, const int32_t* cu_seqlens,
                    int32_t num_seqs, int32_t total_tokens, int32_t max_seqlen,
                    int32_t num_heads_q, int32_t num_heads_kv, int32_t head_dim,
                    int32_t causal, float scale,
                    void* o, float* lse,
                    void* workspace, size_t workspace_bytes, void* stream);

/* Backward of Eq. (2) (section 3): gradients of sum(dout * o).
 *   q, o, dout bf16 [T, Hq, d];  k, v bf16 [T, Hkv, d];  lse fp32 [Hq, T] as
 *   written by attn_fwd for the same inputs.
 *   dq fp32 [T, Hq, d] (out);  dk, dv fp32 [T, Hkv, d] (out; with grouped
 *   heads each sums its query heads).  Gradients are fp32 so that large
 *   accumulated values keep their precision.
 * Same size/flag rules as attn_fwd. */
pdy_status attn_bwd(const void* q, const void* k, const void* v, const void* o, const float* lse,
                    const void* dout, const int32_t* cu_seqlens,
                    int32_t num_seqs, int32_t total_tokens, int32_t max_seqlen,
                    int32_t num_heads_q, int32_t num_heads_kv, int32_t head_dim,
                    int32_t causal, float scale,
                    float* dq, float* dk, float* dv,
                    void* workspace, size_t workspace_bytes, void* stream);

/* ---- One long sequence split into chunks (context parallelism) ----
 * Sequence-sharded strategies (section 2.2: Megatron-style context
 * parallelism, its ZeRO-3 variant, the fine-grained two-level ring) give a
 * device the queries of positions q_offset .. q_offset+tq-1 and, one chunk
 * at a time, the keys/values of positions k_offset .. k_offset+tk-1 of the
 * same sequence.  Eq. (2) restricted to one key chunk gives a partial output
 * and log-sum-exp; attn_merge combines partials of the same rows into the
 * result over the union of the chunks.  With causal = 1 a key is visible to
 * a query iff its position is <= the query's; a row that sees no key of the
 * chunk gets o = 0 and lse = -inf (the neutral element of attn_merge).
 * Sizes: tq, tk >= 0, offsets >= 0; tensors [tq, Hq, d] (q, o, dout, dq),
 * [tk, Hkv, d] (k, v, dk, dv), lse fp32 [Hq, tq].  Other rules as above. */
size_t attn_fwd_chunk_workspace_size(int32_t tq, int32_t tk, int32_t num_heads_q,
                                     int32_t num_heads_kv, int32_t head_dim);
size_t attn_bwd_chunk_workspace_size(int32_t tq, int32_t tk, int32_t num_heads_q,
                                     int32_t num_heads_kv, int32_t head_dim);

/* Partial forward of a query chunk over one key/value chunk:
 * o bf16 [tq, Hq, d] and lse fp32 [Hq, tq] (out).  tq = 0 is a no-op;
 * tk = 0 gives o = 0, lse = -inf (k and v may then be NULL). */
pdy_status attn_fwd_chunk(const void* q, const void* k, const void* v, int32_t tq, int32_t tk,
                          int32_t q_offset, int32_t k_offset,
                          int32_t num_heads_q, int32_t num_heads_kv, int32_t head_dim,
                          int32_t causal, float scale,
                          void* o, float* lse,
                          void* workspace, size_t workspace_bytes, void* stream);

/* Contribution of one (query chunk, key chunk) pair to the gradient of
 * sum(dout * O): o and lse are the FINAL output and log-sum-exp of the query
 * rows (merged over every key chunk), dout their upstream gradient.
 * Writes dq fp32 [tq, Hq, d] (this pair's part; the chunk's dQ is the sum
 * over its key chunks) and dk, dv fp32 [tk, Hkv, d] (this pair's part; a key
 * chunk's gradient is the sum over query chunks); with accumulate = 1 the
 * part is added to what dq, dk and dv hold.  Rows with lse = -inf
 * contribute nothing.  tq = 0 writes zero dk, dv (accumulate = 0) or leaves
 * them (accumulate = 1). */
pdy_status attn_bwd_chunk(const void* q, const void* k, const void* v, const void* o,
                          const float* lse, const void* dout, int32_t tq, int32_t tk,
                          int32_t q_offset, int32_t k_offset,
                          int32_t num_heads_q, int32_t num_heads_kv, int32_t head_dim,
                          int32_t causal, float scale,
                          float* dq, float* dk, float* dv, int32_t accumulate,
                          void* workspace, size_t workspace_bytes, void* stream);

/* The same two calls for a caller that runs `launches` (>= 1) such pairs of about
 * these sizes at a time, on as many streams: the launch's shape then leaves the
 * chip to them together.  attn_fwd_chunk and attn_bwd_chunk are launches = 1.
 * (Each call has its own outputs and workspace, as any concurrent calls.) */
pdy_status attn_fwd_chunk_shared(const void* q, const void* k, const void* v, int32_t tq,
                                 int32_t tk, int32_t q_offset, int32_t k_offset,
                                 int32_t num_heads_q, int32_t num_heads_kv, int32_t head_dim,
                                 int32_t causal, float scale,
                                 void* o, float* lse,
                                 void* workspace, size_t workspace_bytes, void* stream,
                                 int32_t launches);
pdy_status attn_bwd_chunk_shared(const void* q, const void* k, const void* v, const void* o,
                                 const float* lse, const void* dout, int32_t tq, int32_t tk,
                                 int32_t q_offset, int32_t k_offset,
                                 int32_t num_heads_q, int32_t num_heads_kv, int32_t head_dim,
                                 int32_t causal, float scale,
                                 float* dq, float* dk, float* dv, int32_t accumulate,
                                 void* workspace, size_t workspace_bytes, void* stream,
                                 int32_t launches);

/* Combine two partial results of the same T query rows:
 *   lse = log(exp(lse_a) + exp(lse_b)),  o = sum_x exp(lse_x - lse) o_x
 * (bf16 [T, Hq, d] and fp32 [Hq, T]).  o/lse may alias o_a/lse_a or
 * o_b/lse_b (in place).  Needs no workspace. */
pdy_status attn_merge(const void* o_a, const float* lse_a, const void* o_b, const float* lse_b,
                      int32_t total_tokens, int32_t num_heads_q, int32_t head_dim,
                      void* o, float* lse, void* stream);

/* ---- Keys of another length, and keys shared by the batch ----
 * A batch of num_seqs sequences; sequence i has the queries cu_seqlens_q[i] ..
 * cu_seqlens_q[i+1]-1 and the keys cu_seqlens_k[i] .. cu_seqlens_k[i+1]-1 (int32
 * device arrays of num_seqs + 1).  Either may be empty.
 *   - seqlens_k (int32 device array of num_seqs, or NULL): only the first
 *     seqlens_k[i] of a sequence's keys are in use -- a cache with room left, or a
 *     padded batch (cu_seqlens_k then are multiples of the padded length).  Other
 *     keys are never read as numbers, whatever they hold.
 *   - Query rows from cu_seqlens_q[num_seqs] on and key rows from
 *     cu_seqlens_k[num_seqs] on belong to no sequence: their outputs and gradients
 *     are left as they were.
 *   - causal = 1 aligns the sequences' ends: with nq queries and nk keys in use,
 *     key j is visible to query i iff j <= i + nk - nq (the last query sees all).
 *   - attn_prefix_*: every row of the batch also sees the prefix_len keys k_prefix,
 *     v_prefix, bf16 [prefix_len, Hkv, d] (causal or not), which are read once for
 *     all rows where these are few a sequence.  prefix_len = 0 is attn_cross_*.
 *   - A row that sees no key gets o = 0, lse = -inf, and no gradient.
 *   - max_seqlen_q, max_seqlen_k: upper bounds of the sequences' queries and keys; with
 *     seqlens_k the latter may bound the keys in use alone.  Of a sequence with more,
 *     the rows beyond max_seqlen_q, and so the gradients of the keys that these see, and
 *     dk, dv beyond max_seqlen_k may stay unwritten or are wrong; other sequences have
 *     theirs.  Offsets are trusted as above, but clamped to the tensors: wrong ones give
 *     wrong results, no stray access.
 *   - Gradients of sum(dout * o), given o and lse as the forward wrote them; with
 *     grad_bf16 = 0 fp32, with 1 bf16 (rounded once, from 32-bit sums).  dk and dv of
 *     keys not in use are 0; dk_prefix and dv_prefix sum the rows of all sequences.
 *   - Probabilities (before the products with v and dout) and the logits' gradients
 *     (before those with k and q) are rounded to bf16, and the backward takes
 *     <dout, o> from the rounded o for rows with more than 64 keys; logits, sums and
 *     lse are 32 bits.
 *   - An infinity or NaN in a v in use, or in dout, may also reach rows (keys) of its
 *     sequence that the causal mask parts from it, as in attn_fwd and attn_bwd.
 * q, o bf16 [total_q, Hq, d]; k, v bf16 [total_k, Hkv, d] (NULL if total_k = 0); lse
 * fp32 [Hq, total_q].  Launch shapes and the parts of rows with few keys follow from
 * the sizes and the offsets' values: results of a sequence depend on its batch in
 * rounding only.  Hq * d is below 2^24, Hkv * d below 2^22.  Other rules as above. */
size_t attn_cross_fwd_workspace_size(int32_t total_q, int32_t total_k, int32_t num_seqs,
                                     int32_t max_seqlen_q, int32_t max_seqlen_k,
                                     int32_t num_heads_q, int32_t num_heads_kv, int32_t head_dim);
pdy_status attn_cross_fwd(const void* q, const void* k, const void* v, const int32_t* cu_seqlens_q,
                          const int32_t* cu_seqlens_k, const int32_t* seqlens_k, int32_t num_seqs,
                          int32_t total_q, int32_t total_k, int32_t max_seqlen_q,
                          int32_t max_seqlen_k, int32_t num_heads_q, int32_t num_heads_kv,
                          int32_t head_dim, int32_t causal, float scale, void* o, float* lse,
                          void* workspace, size_t workspace_bytes, void* stream);
size_t attn_prefix_fwd_workspace_size(int32_t prefix_len, int32_t total_q, int32_t total_k,
                                      int32_t num_seqs, int32_t max_seqlen_q, int32_t max_seqlen_k,
                                      int32_t num_heads_q, int32_t num_heads_kv, int32_t head_dim);
pdy_status attn_prefix_fwd(const void* q, const void* k, const void* v, const void* k_prefix,
                           const void* v_prefix, const int32_t* cu_seqlens_q,
                           const int32_t* cu_seqlens_k, const int32_t* seqlens_k,
                           int32_t prefix_len, int32_t num_seqs, int32_t total_q, int32_t total_k,
                           int32_t max_seqlen_q, int32_t max_seqlen_k, int32_t num_heads_q,
                           int32_t num_heads_kv, int32_t head_dim, int32_t causal, float scale,
                           void* o, float* lse, void* workspace, size_t workspace_bytes,
                           void* stream);
size_t attn_cross_bwd_workspace_size(int32_t total_q, int32_t total_k, int32_t num_seqs,
                                     int32_t max_seqlen_q, int32_t max_seqlen_k,
                                     int32_t num_heads_q, int32_t num_heads_kv, int32_t head_dim);
pdy_status attn_cross_bwd(const void* q, const void* k, const void* v, const void* o,
                          const float* lse, const void* dout, const int32_t* cu_seqlens_q,
                          const int32_t* cu_seqlens_k, const int32_t* seqlens_k, int32_t num_seqs,
                          int32_t total_q, int32_t total_k, int32_t max_seqlen_q,
                          int32_t max_seqlen_k, int32_t num_heads_q, int32_t num_heads_kv,
                          int32_t head_dim, int32_t causal, float scale, int32_t grad_bf16,
                          void* dq, void* dk, void* dv, void* workspace, size_t workspace_bytes,
                          void* stream);
size_t attn_prefix_bwd_workspace_size(int32_t prefix_len, int32_t total_q, int32_t total_k,
                                      int32_t num_seqs, int32_t max_seqlen_q, int32_t max_seqlen_k,
                                      int32_t num_heads_q, int32_t num_heads_kv, int32_t head_dim);
pdy_status attn_prefix_bwd(const void* q, const void* k, const void* v, const void* k_prefix,
                           const void* v_prefix, const void* o, const float* lse, const void* dout,
                           const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k,
                           const int32_t* seqlens_k, int32_t prefix_len, int32_t num_seqs,
                           int32_t total_q, int32_t total_k, int32_t max_seqlen_q,
                           int32_t max_seqlen_k, int32_t num_heads_q, int32_t num_heads_kv,
                           int32_t head_dim, int32_t causal, float scale, int32_t grad_bf16,
                           void* dq, void* dk, void* dv, void* dk_prefix, void* dv_prefix,
                           void* workspace, size_t workspace_bytes, void* stream);

/* ---- Rotary positions with several axes ----
 * Rotates the first 2 num_pairs elements of every head of q and k in pairs: pair p by
 * the angle positions[t][pair_axes[p]] * w_p (num_axes int32 positions a token, e.g.
 * time, height, width; negative ones too), and copies the rest.  A pair is elements p
 * and p + num_pairs, or with interleaved = 1 elements 2 p and 2 p + 1:
 *   (x, y) -> (x cos - y sin, x sin + y cos).
 * inverse = 1 takes the negative angle: it undoes the rotation, and turns the
 * gradients of rotated q and k into those of q and k.
 *   q, k (in) and q_out, k_out: [total_tokens, num_heads_q or num_heads_kv, head_dim],
 *   bf16, or fp32 with in_fp32 (out_fp32 = 1, or bf16 with 0); out may be in where the
 *   types are the same.  With a head count of 0 that tensor is NULL.
 *   positions: int32 device array [total_tokens, num_axes], num_axes 1 to 4.
 *   num_pairs: a multiple of 8 up to head_dim / 2.
 *   turns, pair_axes: HOST arrays of num_pairs, read during the call (a captured graph
 *   keeps their values); turns[p] = w_p / 2 pi as a 64-bit fraction of a turn, which
 *   attn_rotary_turns computes from the frequencies w_p (radians a position, finite),
 *   rounded to the nearest.
 * For every int32 position and frequency the angle is off by less than 2^-31 of a turn
 * from positions * w_p (w_p as the double that it is); products are 32 bits, rounded
 * once to a bf16 output.  Needs no workspace; total_tokens is below 2^26 - 4. */
pdy_status attn_rotary_turns(const double* freqs, int32_t num_pairs, uint64_t* turns);
pdy_status attn_rotary(const void* q, const void* k, const int32_t* positions,
                       int32_t total_tokens, int32_t num_axes, int32_t num_heads_q,
                       int32_t num_heads_kv, int32_t head_dim, int32_t num_pairs,
                       const uint64_t* turns, const int32_t* pair_axes, int32_t interleaved,
                       int32_t inverse, int32_t in_fp32, int32_t out_fp32, void* q_out,
                       void* k_out, void* stream);

/* ---- A paged key/value cache ----
 * A pool of num_pages pages of page_size keys (a multiple of 16):
 *   k_pages, v_pages [num_pages, Hkv, page_size, d], bf16, or with cache_e4m3 = 1 8-bit
 *   floats (e4m3, largest 448): a value is its byte's times k_scale (v_scale) of the head,
 *   fp32 device arrays [Hkv] (NULL with bf16), positive and finite;
 *   scores fp32 [num_pages, Hkv, page_size]: a running weight of every key, where kept.
 * page_table: int32 device array [num_seqs, max_pages]; key j of sequence i is key
 * j % page_size of page page_table[i][j / page_size].  seqlens_k: int32 device array
 * [num_seqs], the keys in use.  Entries behind the last page in use are not used, whatever
 * they hold.
 *   - Pages may be shared by sequences (a common beginning) in calls that only read them;
 *     what a call writes (new keys, scores -- those that attn_paged_fwd adds to, too: sums
 *     of sequences that share a page would be lost --, kept keys) is in pages of one
 *     sequence, each once in its table.
 *   - Tables and lengths are trusted, but clamped to the tensors: wrong ones give wrong
 *     results, no stray access (keys in no page of the pool are not written).
 *   - Slots that hold no key in use may hold anything, NaN among it.
 *   - num_pages * Hkv * page_size / 16 is below 2^31, max_pages * page_size below 2^30.
 * Other rules as above. */

/* New keys and values into their pages: token t of the nq = cu_seqlens[i+1] -
 * cu_seqlens[i] tokens of sequence i becomes its key seqlens_k[i] - nq + t (seqlens_k
 * counts the new ones; tokens that would lie in front of key 0 are dropped).
 *   k, v bf16 [total_tokens, Hkv, d]; tokens from cu_seqlens[num_seqs] on are no
 *   sequence's.  e4m3: the 32-bit quotient x / scale, up to 448, rounded to the nearest
 *   (ties to even).
 *   scores (or NULL): 0 for the new keys.
 * total_tokens is below 2^26 - 4.  Needs no workspace. */
pdy_status attn_paged_write(const void* k, const void* v, const int32_t* cu_seqlens,
                            const int32_t* page_table, const int32_t* seqlens_k,
                            const float* k_scale, const float* v_scale, int32_t num_seqs,
                            int32_t total_tokens, int32_t num_pages, int32_t page_size,
                            int32_t max_pages, int32_t num_heads_kv, int32_t head_dim,
                            int32_t cache_e4m3, void* k_pages, void* v_pages, float* scores,
                            void* stream);

/* attn_cross_fwd over a paged cache: the queries cu_seqlens_q[i] .. cu_seqlens_q[i+1]-1 of
 * sequence i over its first seqlens_k[i] keys (max_seqlen_k where these are more); the rules
 * of rows, masks and results are those of attn_cross_fwd.  Meant for one or few queries a
 * sequence (any number is right).
 *   scores (or NULL): adds to every key in use its weight, the sum over the sequence's
 *   rows and the heads of its group of exp(S - lse), with logits S and lse as above; rows
 *   with lse = -inf add nothing.
 * Probabilities (before the product with v) are rounded to bf16; logits, sums, weights and
 * lse are 32 bits.  The same call gives the same bits; launches of other sizes differ in
 * rounding.  With scores num_seqs is at most 65,535, and num_seqs * Hkv * (max_seqlen_k /
 * 512, rounded up) below 2^24.  with_scores: whether scores will be given.  The workspace
 * is for a call of just these sizes, the bound max_seqlen_k among them: at most about 70 MB,
 * and with scores up to 1 GiB of logits more (4 bytes a query head, query and key, where a
 * sequence has up to 16 queries times heads of a group; more logits than that are computed
 * twice). */
size_t attn_paged_fwd_workspace_size(int32_t total_q, int32_t num_seqs, int32_t max_seqlen_q,
                                     int32_t max_seqlen_k, int32_t num_heads_q,
                                     int32_t num_heads_kv, int32_t head_dim,
                                     int32_t with_scores);
pdy_status attn_paged_fwd(const void* q, const void* k_pages, const void* v_pages,
                          const int32_t* page_table, const int32_t* cu_seqlens_q,
                          const int32_t* seqlens_k, const float* k_scale, const float* v_scale,
                          int32_t num_seqs, int32_t total_q, int32_t num_pages, int32_t page_size,
                          int32_t max_pages, int32_t max_seqlen_q, int32_t max_seqlen_k,
                          int32_t num_heads_q, int32_t num_heads_kv, int32_t head_dim,
                          int32_t cache_e4m3, int32_t causal, float scale, void* o, float* lse,
                          float* scores, void* workspace, size_t workspace_bytes, void* stream);

/* Shortens every sequence of more than `budget` keys to so many, each kv head by its own
 * scores: the first `first` and the last `recent` keys stay, and of those between the ones of
 * the highest scores (equal ones: the earlier; a NaN is below every number).  What stays, of
 * the shorter sequences everything, is copied in its order, keys, values and scores, to the
 * pages of new_table, int32 device array [num_seqs, new_max_pages], which must be none that
 * the sequences use.  (Keys keep what they were rotated by.)
 *   kept int32 [num_seqs, Hkv, budget] (out): the old number of each key, -1 behind the
 *   last.  new_lens int32 [num_seqs] (out): min(seqlens_k, budget); may be seqlens_k (all
 *   of it, not a part).
 * first + recent <= budget <= new_max_pages * page_size (or max_seqlen_k is); num_seqs is at
 * most 65,535, num_seqs * Hkv below 2^22 and num_seqs * Hkv * budget below 2^31.  The
 * workspace, 256 bytes, is asked for and checked as other calls' is; nothing is held there. */
size_t attn_paged_evict_workspace_size(int32_t num_seqs, int32_t max_seqlen_k,
                                       int32_t num_heads_kv, int32_t budget);
pdy_status attn_paged_evict(void* k_pages, void* v_pages, float* scores, const int32_t* page_table,
                            const int32_t* seqlens_k, const int32_t* new_table, int32_t num_seqs,
                            int32_t num_pages, int32_t page_size, int32_t max_pages,
                            int32_t new_max_pages, int32_t max_seqlen_k, int32_t num_heads_kv,
                            int32_t head_dim, int32_t cache_e4m3, int32_t budget, int32_t recent,
                            int32_t first, int32_t* kept, int32_t* new_lens, void* workspace,
                            size_t workspace_bytes, void* stream);

/* Debug helper: copies cu_seqlens to the host (synchronising `stream`) and
 * checks cu[0] = 0, monotonicity and cu[num_seqs] = total_tokens.  On success
 * writes the longest segment length to *max_seqlen_out (may be NULL). */
pdy_status attn_validate_cu_seqlens(const int32_t* cu_seqlens, int32_t num_seqs,
                                    int32_t total_tokens, int32_t* max_seqlen_out,
                                    void* stream);

/* attn_bwd for callers that cannot allocate device memory (code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc): the
 * same computation, arguments and outputs as attn_bwd, without the
 * workspace.  Its scratch (the tile schedules, D and any split-K partial
 * gradients) is a static device array of 64 MiB per GPU, held from the
 * first call on that GPU until the process ends.  Sizes whose schedules and
 * D alone exceed 64 MiB (Hq * T beyond about 16.7 million (row, head)
 * pairs) return PDY_ERR_WORKSPACE before anything is launched.  A launch
 * small enough to split (see above) whose partial gradients would not fit
 * takes fewer parts, and one whose tile schedule would not fit another shape;
 * its results may then differ from attn_bwd's in rounding (well inside the
 * stated tolerance), otherwise they equal attn_bwd's bit for bit.  The call allocates nothing (no hipMalloc, no
 * library allocation); on its first use on a device it looks up that
 * device's address of the array.  The array keeps the last call's contents,
 * none of which a call reads before writing it.  Every call on one GPU uses
 * the same array: calls that overlap on one GPU (other streams, other
 * threads) race and must be serialised by the caller. */
pdy_status attn_bwd_noalloc(const void* q, const void* k, const void* v, const void* o,
                            const float* lse, const void* dout, const int32_t* cu_seqlens,
                            int32_t num_seqs, int32_t total_tokens, int32_t max_seqlen,
                            int32_t num_heads_q, int32_t num_heads_kv, int32_t head_dim,
                            int32_t causal, float scale, float* dq, float* dk, float* dv,
                            void* stream);

/* The launches that a call of these sizes takes, given a workspace of the
 * size the query above returns: for the forward, dQ and dK/dV kernels in turn
 * {waves per workgroup, groups of waves that split the inner loop over the same
 * rows (keys), parts per work item at most}, 9 values (host memory); zeros
 * where the kernel is not launched.  (A host computation: nothing is launched.) */
pdy_status pdy_launch_shapes(int32_t total_tokens, int32_t num_seqs, int32_t max_seqlen,
                             int32_t num_heads_q, int32_t num_heads_kv, int32_t head_dim,
                             int32_t causal, int32_t* shapes);
pdy_status pdy_chunk_launch_shapes(int32_t tq, int32_t tk, int32_t q_offset, int32_t k_offset,
                                   int32_t num_heads_q, int32_t num_heads_kv, int32_t head_dim,
                                   int32_t causal, int32_t launches, int32_t* shapes);

/* The same for attn_cross_* (prefix_len = 0) and attn_prefix_*: three values each for the
 * forward, dQ and dK/dV kernels (a launch is cut into that many parts per item at most,
 * as the offsets have it), then 1 where the shared keys are a list of their own beside
 * the sequences' (partial results of both), and 1 each where the forward and dQ keep
 * their first items whole: 12 values. */
pdy_status pdy_cross_launch_shapes(int32_t prefix_len, int32_t total_q, int32_t total_k,
                                   int32_t num_seqs, int32_t max_seqlen_q, int32_t max_seqlen_k,
                                   int32_t num_heads_q, int32_t num_heads_kv, int32_t head_dim,
                                   int32_t causal, int32_t* shapes);

/* The same for attn_paged_fwd: {waves per workgroup, packed rows (queries times heads of a
 * group) per tile, parts per tile's keys at most, 1 where the weights come from the logits
 * that the attention leaves, not from the keys again}: 4 values. */
pdy_status pdy_paged_launch_shapes(int32_t total_q, int32_t num_seqs, int32_t max_seqlen_q,
                                   int32_t max_seqlen_k, int32_t num_heads_q,
                                   int32_t num_heads_kv, int32_t head_dim, int32_t cache_e4m3,
                                   int32_t with_scores, int32_t* shapes);

/* Static text for a status code. */
const char* pdy_status_string(int32_t status);

/* Detail of the last non-OK status returned on this thread ("" if none). */
const char* pdy_last_error(void);

/* Kernel timing (measurement support for the per-length cost tables the
 * paper's hybrid cost models are fitted to, section 4.3).  Between
 * pdy_profile_start and pdy_profile_stop, every kernel this thread launches
 * is bracketed by two HIP events recorded on the launch's own stream.
 * pdy_profile_stop waits for those events and writes, for each kernel id
 * k < n, the number of launches and their summed duration in milliseconds
 * (arrays of n caller-owned host elements).  Kernel ids are
 * 0..pdy_kernel_count()-1, named by pdy_kernel_name. */
int32_t pdy_kernel_count(void);
const char* pdy_kernel_name(int32_t k);
pdy_status pdy_profile_start(void);
pdy_status pdy_profile_stop(int32_t* launches, double* total_ms, int32_t n);

#ifdef __cplusplus
}
#endif
#endif /* PDYATTN_H */
