/*
 * sift_serve.h - C ABI of libsift around the sparse prefill (sift.h): dense
 * attention of a plan's prompts with transformed scores, and the paged cache
 * that a prefill leaves: attention of new tokens over it, the accumulated
 * attention weights of its keys, and the eviction of those with the least.
 *
 * The conventions of sift.h hold (tensors, layouts, streams, errors, threads).
 */
#ifndef SIFT_SERVE_H_
#define SIFT_SERVE_H_

#include "sift.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Transform of the attention scores, of the calls that take one.  With z =
 * softmax_scale * (q . k), a score is s = cap * tanh(z / cap) (z itself where
 * cap is 0), less slopes[h] * |position of the query - position of the key|
 * where slopes are given.
 *   softmax_scale  <= 0 selects 1/sqrt(D); one that is not a float any more times
 *                  log2(e): SIFT_E_UNSUPPORTED
 *   cap            0 for none; negative, NaN or beyond 1e15: SIFT_E_UNSUPPORTED, and
 *                  so are caps too small or too large beside the scale: scale / cap
 *                  has to be a normal float and scale (scale / cap)^8 a finite one
 *                  (at the scale of D = 128 caps from 1e-6 on).  q . k beyond 1e19
 *                  has no defined score under a cap.
 *   slopes         device float [Hq], or NULL; positions are exact up to 2^24, and
 *                  |slope| * distance stays below 1e17
 * A NULL score is the default scale alone.
 */
typedef struct sift_score {
  float softmax_scale;
  float cap;
  const float* slopes;
} sift_score;

/* What a row of the dense attention sees of its prompt. */
typedef enum sift_mask {
  SIFT_MASK_CAUSAL = 0,   /* every token up to itself                          */
  SIFT_MASK_DOCUMENT = 1, /* a document's row: its own document up to itself;
                             a query's row: every token up to itself           */
  SIFT_MASK_PREFIX = 2    /* all of the prompt's documents, and every token up
                             to itself                                         */
} sift_mask;

/*
 * Dense attention of the plan's prompts with transformed scores, for the
 * layers of a model that are not sparse, or whose documents are prefilled
 * each by itself: softmax over the visible keys times V, no bit vectors.
 *   q, k, v, out   device tensors as everywhere else, all SIFT_BF16 or all
 *                  SIFT_F32, D 64 or 128 (any tile), 16-byte aligned
 *   mask           a sift_mask
 *   score          see sift_score; positions are the tokens' places in their
 *                  prompt
 *   lse            device float [tokens][Hq], or NULL: receives each row's
 *                  log sum exp of its scores (natural logarithm), as
 *                  sift_cache_accumulate takes it
 * Keys that a row does not see have no influence on it, whatever they hold.
 * The plan's lists are neither read nor changed.  bf16: the weights are
 * rounded to bf16 for their product with V, as in the sparse attention, the
 * sums are fp32.
 * out and lse overlap no input.
 * Errors: SIFT_E_NULL, SIFT_E_SHAPE, SIFT_E_UNSUPPORTED (mask, cap, dtypes,
 *   alignment, more than 2^17 kv heads), SIFT_E_PLAN (another device is current),
 *   SIFT_E_CAPACITY (2^24 workgroups of 128 rows of a head or more), SIFT_E_HIP.
 */
sift_status sift_plan_dense(sift_plan* plan, const sift_tensor* q, const sift_tensor* k,
                            const sift_tensor* v, int32_t mask, const sift_score* score,
                            sift_tensor* out, float* lse, void* stream);

/*
 * Rotary positions.  The first rot_dim dims of a head turn in pairs (x, y) by the
 * angle position * inv_freq[i], i < rot_dim / 2:
 *   x' = magnitude * (x cos - y sin),  y' = magnitude * (y cos + x sin)
 * the others stay.  The angle is formed and reduced to a turn in 64 bits, off by less than
 * 2^-51 of itself: 2e-7 of a turn at 2^31 radians (sift_rope forms it in fp32).
 *   inv_freq     device float [rot_dim / 2]: any table, so that any scaling of the
 *                frequencies for long contexts is one
 *   rot_dim      even, 2 .. D
 *   interleaved  0: pair i is dims i and rot_dim / 2 + i; else 2 i and 2 i + 1
 *   magnitude    finite, > 0
 */
typedef struct sift_rotary {
  const float* inv_freq;
  int32_t rot_dim;
  int32_t interleaved;
  float magnitude;
} sift_rotary;

/*
 * q and k turned by their tokens' positions, into q_out and k_out.
 *   q, q_out     [tokens][Hq][D];  k, k_out: [tokens][Hkv][D], or both NULL.  All
 *                SIFT_BF16 or all SIFT_F32, any D; an output is its input's buffer, or
 *                apart from all others.  16-byte aligned buffers of whole 16-byte
 *                chunks (rot_dim, and its half where pairs lie in halves, too) go
 *                fastest.
 *   positions    device int32 [tokens]
 *   back         not 0: by the negative angles.  That is the gradient of the call (its
 *                transpose), and where the magnitude is 1 its inverse: keys turned back
 *                and then by other positions have moved.
 * Rounded once.  Values that are not finite reach the other one of their pair.
 * Errors: SIFT_E_NULL, SIFT_E_SHAPE, SIFT_E_UNSUPPORTED (dtypes, magnitude, buffers that
 *   overlap), SIFT_E_CAPACITY (a token of 2^31 numbers or more), SIFT_E_HIP.
 */
sift_status sift_rotate(const sift_tensor* q, const sift_tensor* k, const int32_t* positions,
                        const sift_rotary* rotary, int32_t back, sift_tensor* q_out,
                        sift_tensor* k_out, void* stream);

/*
 * The paged cache of a batch of sequences, of one layer.
 *
 * Slots: sequence b owns max_pages pages of `page` slots.  Slot i is row
 *   i % page of pool page page_table[b][i / page] (the pools of
 *   sift_plan_run_paged, whose T is the page here); it holds a key where
 *   i < lens[b] and, where page_lens are given, i % page <
 *   page_lens[b][i / page] (a document's last page may end early).  Pages may
 *   be shared by sequences; the order of the slots means nothing but the
 *   positions: key_pos[b][kv head][i], or i itself where none are given.
 * Tables are device memory, read when the work runs, so that a captured graph
 *   serves growing caches.  Values outside their range are clamped: no access
 *   leaves the given buffers, and the result for such sequences is meaningless.
 */
typedef struct sift_cache_kv {
  const sift_tensor* k_pages;  /* [num_pages * page][Hkv][D]                     */
  const sift_tensor* v_pages;
  const int32_t* page_table;   /* [num_seqs][max_pages]                          */
  const int32_t* lens;         /* [num_seqs], 0 .. max_pages * page              */
  const int32_t* page_lens;    /* [num_seqs][max_pages], or NULL: full pages     */
  const int32_t* key_pos;      /* [num_seqs][Hkv][max_pages * page], or NULL     */
  /* Read with SIFT_E4M3 pools only (programs built without them pass none): a key is
   * its pool row times its page's and kv head's scale, any from 2^-100 to 2^120 (taken
   * as the nearer of these where it is below or above, by appends too, and NaN as 2^-100;
   * pages without keys: anything). */
  float* k_scales;             /* [num_pages][Hkv]                               */
  float* v_scales;
} sift_cache_kv;

/* The new tokens of the sequences, rows row_ptr[b] .. row_ptr[b+1]-1 (at most
 * max_rows) of q for sequence b. */
typedef struct sift_cache_rows {
  const int32_t* row_ptr;      /* device [num_seqs + 1], or NULL: as many of each */
  const int32_t* row_pos;      /* device [rows]: positions, or NULL: lens[b] and
                                  on, in order                                   */
} sift_cache_rows;

/* Opaque: the sizes of a batch's caches, and device scratch. */
typedef struct sift_cache sift_cache;

/*
 * Make a handle for caches of these sizes.  Allocates device memory on the
 * current device (scratch for partial results and for the eviction); the
 * calls below allocate nothing.  Calls on one handle must be ordered.
 *   num_seqs, num_q_heads, num_kv_heads >= 1, Hq % Hkv == 0
 *   head_dim   D: 64 or 128;  page: 16, 32, 64 or 128
 *   max_pages  pages of a sequence at most, >= 1
 *   max_rows   new tokens of a sequence in one call at most, >= 1
 * Errors: SIFT_E_NULL, SIFT_E_SHAPE, SIFT_E_UNSUPPORTED (D, page),
 *   SIFT_E_CAPACITY (slots or rows x heads beyond 2^31 - 256, more than 2^17 kv
 *   heads), SIFT_E_HIP.
 */
sift_status sift_cache_create(int32_t num_seqs, int32_t num_q_heads, int32_t num_kv_heads,
                              int32_t head_dim, int32_t page, int32_t max_pages,
                              int32_t max_rows, sift_cache** cache_out);

/* Free a handle and its scratch (waits first for the stream of its last
 * enqueued work).  NULL is accepted. */
sift_status sift_cache_destroy(sift_cache* cache);

/*
 * Attention of the new tokens over the cache and over each other: a single
 * token, a chain or a drafted tree for each sequence, in one call.
 *   q, out       [rows][Hq][D];  k_new, v_new: [rows][Hkv][D], the new tokens'
 *                own keys, which the cache does not hold yet.  All tensors and
 *                the pools SIFT_BF16 or all SIFT_F32, 16-byte aligned; with pools of
 *                SIFT_E4M3 all others SIFT_BF16.  But for fp32 the weights are rounded to
 *                bf16 for the product with V, and divided by the sum of the rounded ones.
 *   tree_mask    device uint64 [rows][mask_words], mask_words >=
 *                ceil(max_rows / 64): bit j % 64 of word j / 64 says whether the
 *                row sees new token j of its sequence (its ancestors and
 *                itself); every key of the cache is visible to every row.
 *                NULL: a chain, each row sees those up to itself.
 *   score        see sift_score
 *   lse          device float [rows][Hq], or NULL: the rows' log sum exp
 * bf16 handles of many rows and slots (max_pages, not the lengths, which only the
 *   device knows) go by larger units of work, slower for short caches: make a
 *   handle for the sizes that it meets.
 * A row that sees no key gets 0, and -infinity for its log sum; so does one
 * whose every visible score is -infinity.  Keys that a row does not see have no
 * influence on it.  Rows that row_ptr leaves out are not written.  Results
 * depend on nothing but the arguments (no atomics).
 * Errors: SIFT_E_NULL, SIFT_E_SHAPE, SIFT_E_UNSUPPORTED (dtypes, alignment,
 *   cap), SIFT_E_CAPACITY (mask_words; 2^24 rows x heads or more; 2^31 steps of 128
 *   keys of 32 rows of a kv head or more, were all sequences as long and as many new
 *   tokens as the handle and q allow), SIFT_E_PLAN (another device is current),
 *   SIFT_E_HIP.
 */
sift_status sift_cache_attention(sift_cache* cache, const sift_cache_kv* kv,
                                 const sift_cache_rows* new_rows, const sift_tensor* q,
                                 const sift_tensor* k_new, const sift_tensor* v_new,
                                 const uint64_t* tree_mask, int32_t mask_words,
                                 const sift_score* score, sift_tensor* out, float* lse,
                                 void* stream);

/*
 * New keys and values of every sequence into its pages, the keys turned by their
 * positions on the way.
 *   k, v         [rows][Hkv][D], 16-byte aligned, the pools' type; SIFT_BF16 where the
 *                pools are SIFT_E4M3.  They overlap no pool.
 *   new_rows     row_ptr: any number of rows of a sequence (max_rows is not meant);
 *                row_pos: the keys' positions
 *   rotary       how the keys turn, or NULL: as they are
 *   slots        device int32 [rows]: the slot of its sequence that a row goes to (none
 *                twice), or NULL: lens[b] and on, in order.  Not with SIFT_E4M3.
 *                row_pos NULL: a row's position is its slot.
 *   pos_out      device int32 [num_seqs][Hkv][max_pages * page], may be the key_pos, or
 *                NULL: receives the positions of the slots that are written
 *   lens_out     device int32 [num_seqs], may be the lens (a second, small launch), or
 *                NULL: the lens of the next calls.  Without slots only.
 * Rows past a sequence's last slot are left out, and rows of pages that are not in the
 * pools (page_table values out of range).  page_lens are neither read nor
 * changed.  The pages that rows enter must be the sequence's own.
 * SIFT_E4M3: a page's scale becomes the least power of two (2^-100 at least) such that
 *   448 times it holds max |x| of the page's new rows of the head (of dims that turn,
 *   sqrt(2) times that and the magnitude), and that is not below the scale under which
 *   the page held keys.  Where it grows the codes of the keys held are rounded again.  Values
 *   that are not finite are held as NaN and take no part in the scale.  The first row
 *   that enters a page begins it: whatever else it holds, and its scale, is forgotten.
 * Errors: SIFT_E_NULL, SIFT_E_SHAPE, SIFT_E_UNSUPPORTED (dtypes, alignment, magnitude;
 *   slots with lens_out or SIFT_E4M3; lens_out that overlaps the lens in part),
 *   SIFT_E_CAPACITY (2^31 rows x kv heads, or (sequence, page, kv head) triples that
 *   they could enter), SIFT_E_PLAN (another device is current), SIFT_E_HIP.
 */
sift_status sift_cache_append(sift_cache* cache, const sift_cache_kv* kv,
                              const sift_cache_rows* new_rows, const sift_tensor* k,
                              const sift_tensor* v, const sift_rotary* rotary,
                              const int32_t* slots, int32_t* pos_out, int32_t* lens_out,
                              void* stream);

/*
 * Accumulated attention weights of the cached keys, what an eviction goes by:
 *   out[b][kv][i] = decay * weights[b][kv][i]
 *                   + sum over the rows r of b and the query heads h of kv of
 *                     row_weight[r] * exp(s(r, h, i) - lse[r][h])
 * with the scores s of the attention call that left lse (same q, score and
 * tables; its new tokens' own keys are in lse, not here).
 *   lse          device float [rows][Hq]; a row of -infinity counts for nothing
 *   row_weight   device float [rows] >= 0, or NULL: 1.  0 leaves a row out (a
 *                drafted token that was not accepted), whatever it holds.
 *   weights      device float [num_seqs][Hkv][max_pages * page], or NULL: zeros
 *   out          the same shape, may be weights.  Slots before lens[b] that hold no
 *                key get 0, those from lens[b] on are not written.
 * Sums are fp32, in the order of the rows: the result is the same every time.
 * Errors: as sift_cache_attention; SIFT_E_UNSUPPORTED for a decay that is not
 *   finite.
 */
sift_status sift_cache_accumulate(sift_cache* cache, const sift_cache_kv* kv,
                                  const sift_cache_rows* new_rows, const sift_tensor* q,
                                  const float* lse, const float* row_weight,
                                  const sift_score* score, const float* weights, float decay,
                                  float* out, void* stream);

/*
 * Eviction: every (sequence, kv head) keeps n = min(its keys, budget) keys, its
 * protected ones first, then those of the largest weights; equal weights (-0 and
 * 0 among them) go to the lowest slot, NaN counts as less than every number.
 * Protected: positions before `sinks`, and from next_pos[b] - recent on
 * (next_pos: device int32 [num_seqs], the position of the next token, or NULL:
 * lens[b]).  The kept keys end up in slots 0 .. n - 1: those that lie there
 * stay, of the others the j-th in slot order moves to the j-th free slot, K and
 * V rows in place.
 *   budget       >= 1;  sinks, recent >= 0, sinks + recent <= budget
 *   weights      device float [num_seqs][Hkv][max_pages * page]
 *   weights_out, pos_out   the same shape (float, int32): the kept keys' weights
 *                and positions; past them 0 and -1.  pos_out is the key_pos of the
 *                next calls.
 *   lens_out     device int32 [num_seqs]: n, the lens of the next calls, which
 *                take no page_lens: the first slots are all used
 * weights, key_pos and lens are not changed; the outputs may not overlap them.
 * The pages of the first `budget` slots must be the sequence's own.
 * Errors: SIFT_E_NULL, SIFT_E_SHAPE (budget, sinks, recent), SIFT_E_UNSUPPORTED
 *   (overlap, alignment), SIFT_E_CAPACITY (2^22 (sequence, kv head) pairs or
 *   more, 2^33 slots of all of them or more), SIFT_E_PLAN, SIFT_E_HIP.
 */
sift_status sift_cache_evict(sift_cache* cache, const sift_cache_kv* kv, const float* weights,
                             const int32_t* next_pos, int32_t budget, int32_t sinks,
                             int32_t recent, float* weights_out, int32_t* pos_out,
                             int32_t* lens_out, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SIFT_SERVE_H_ */
