/*
 * lacache.h -- C ABI of the LaCache two-stage semantic-cache lookup for
 * AMD Instinct MI355X (gfx950).
 *
 * The method (LaCache, "Robust Semantic Caching for LLM Serving"):
 *   - Each cache entry is <h(x), [h(f_k(x)), f(x)]> (Section 4.2, cache
 *     structure): the key of the cached query x, a lookahead key of the first
 *     k tokens of its response, and the response itself.  Here the key is the
 *     L2-normalised query embedding, the lookahead key is the normalised
 *     embedding of the response prefix plus the k prefix token IDs, and the
 *     response f(x) stays with the caller, addressed by the entry index.
 *   - A query is processed in two stages (Algorithm 1, Section 4.2 query
 *     processing).  Stage 1 searches the cache with the query key: the entry
 *     of highest cosine similarity is the candidate, a hit when its
 *     similarity is >= tau_q (Section 5.1: cache check sim(x, x') >= tau_c).
 *     Stage 2 runs only on a stage-1 hit: the lookahead of the new query
 *     (its first k speculatively decoded tokens and their embedding) is
 *     compared with the stored prefix of the matched entry; it passes when
 *     the k tokens are identical or the prefix-embedding cosine is >= tau_r
 *     (Section 5.1: lookahead check sim(f_k(x), f_k(x')) >= tau_a).  Only
 *     when both pass is the cached response served; otherwise the caller
 *     decodes and inserts (Algorithm 1, fallback branch).
 *   - With an ensemble of m lookahead checks (Section 4.4: m prefix
 *     embedding models, a hit needs every check to pass) each entry stores m
 *     prefix embeddings, one per model and each of its own dimension, and
 *     the embedding branch of stage 2 passes only when every model's cosine
 *     reaches that model's threshold.  The single-model functions are the
 *     case m = 1, with the prefix model of the key's dimension.
 *
 * Conventions for every function below:
 *   - Every array argument is a DEVICE pointer on the handle's device (for
 *     example a PyTorch ROCm tensor's data_ptr()), row-major and contiguous,
 *     unless marked "host".  Pointers may be NULL only when the matching
 *     count is 0.
 *   - `stream` is a hipStream_t (NULL = the default stream).  insert, lookup
 *     and export only enqueue work on it and return without waiting; the
 *     caller keeps every buffer alive until the stream has passed the call.
 *     Work on one handle must be ordered on one stream (or by events): calls
 *     share the handle's store and scratch buffers.
 *   - A handle is not thread-safe.
 *   - Errors are returned as negative codes and nothing is enqueued when an
 *     argument check fails.  No C++ exception crosses this interface.
 *   - Vector inputs must be finite; non-finite components give unspecified
 *     (but memory-safe) results.
 */
#ifndef LACACHE_H
#define LACACHE_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct lacache_s *lacache_t;

/* largest number of prefix models (lookahead checks) of an ensemble cache */
#define LACACHE_MAX_MODELS 8

/* dtype of every input vector of a cache (keys, prefix embeddings, queries, lookahead embeddings) */
typedef enum { LACACHE_F32 = 0, LACACHE_BF16 = 1 } lacache_dtype;

/* decision[b] of a lookup */
enum {
    LACACHE_MISS = 0,      /* stage 1 found no entry with similarity >= tau_q; stage 2 did not run */
    LACACHE_REJECT = 1,    /* stage-1 hit whose lookahead check failed: a collision, decode and insert */
    LACACHE_HIT = 2,       /* both checks passed through the prefix-embedding similarity */
    LACACHE_HIT_EXACT = 3  /* both checks passed with identical first-k prefix tokens */
};

/* return codes */
enum {
    LACACHE_OK = 0,
    LACACHE_EINVAL = -1,   /* bad argument (null pointer, size out of range, non-finite threshold) */
    LACACHE_EFULL = -2,    /* insert would exceed the capacity; nothing was inserted */
    LACACHE_ENOMEM = -3,   /* device allocation failed */
    LACACHE_EHIP = -4      /* a HIP runtime call or kernel launch failed */
};

/*
 * Create a cache on `device` for up to `capacity` entries (1 <= capacity <
 * 2^31 - 256) of dimension d (1 <= d <= 16384), each storing k_cap prefix
 * tokens (1 <= k_cap <= 4096).  Every input vector has dtype in_dtype.
 * max_batch (1 <= max_batch <= 65536) sizes the lookup scratch; lookups with
 * more queries are processed in chunks of max_batch.  All device memory
 * (store and scratch) is allocated here, once, and zero-filled: the store
 * takes capacity * (2 * d_pad * 2 + 4 * k_cap) bytes with d_pad = d rounded
 * up to a multiple of 128.  On success *out receives the handle.
 */
int lacache_create(lacache_t *out, int64_t capacity, int32_t d, int32_t k_cap, lacache_dtype in_dtype,
                   int32_t max_batch, int32_t device);

/*
 * Create a cache whose entries carry an ensemble of m response-prefix
 * embeddings (Section 4.4, m lookahead checks), 1 <= m <= LACACHE_MAX_MODELS.
 * d_resp (host, [m]) gives each prefix model's dimension, 1 .. 16384; the
 * other arguments are those of lacache_create, which equals this call with
 * m = 1 and d_resp = {d}.  The store takes capacity * (2 * d_pad + sum over
 * i of 2 * d_pad_i + 4 * k_cap) bytes, d_pad_i = d_resp[i] rounded up to a
 * multiple of 128.
 */
int lacache_create_ensemble(lacache_t *out, int64_t capacity, int32_t d, int32_t k_cap, lacache_dtype in_dtype,
                            int32_t max_batch, int32_t device, int32_t m, const int32_t *d_resp);

/* Number of prefix models m of the cache; -1 for a NULL handle. */
int32_t lacache_models(lacache_t h);

/* Wait for the device, free everything the handle owns, and the handle itself. NULL is a no-op. */
int lacache_destroy(lacache_t h);

/*
 * Append n entries (Algorithm 1: after decoding, the new entry is added to
 * the cache).  keys and resp_emb are [n][d] of the cache's dtype (the query
 * key and the embedding of the first k_cap response tokens, both from the
 * same embedding model); resp_tokens is [n][k_cap] int32.  Keys and
 * embeddings are L2-normalised (in double) and rounded once, to nearest-even,
 * to bfloat16 as they are stored; a zero vector is stored as zero.
 * Entries get indices size .. size+n-1 in order; *first_idx (host) receives
 * the first.  The entry count is updated immediately, so later lookups on
 * the same stream see the new entries.  n == 0 is a no-op.  Returns
 * LACACHE_EFULL, inserting nothing, if n > capacity - size.  Only for a
 * cache with m = 1 (else LACACHE_EINVAL).
 */
int lacache_insert(lacache_t h, const void *keys, const void *resp_emb, const int32_t *resp_tokens, int32_t n,
                   int64_t *first_idx, void *stream);

/*
 * lacache_insert for any m: resp_emb is a HOST array of m device pointers,
 * resp_emb[i] being [n][d_resp[i]] (cache dtype), the prefix embedding of
 * each entry under model i.  Each is normalised and rounded as keys are.
 */
int lacache_insert_ensemble(lacache_t h, const void *keys, const void *const *resp_emb, const int32_t *resp_tokens,
                            int32_t n, int64_t *first_idx, void *stream);

/*
 * Two-stage lookup of B queries (Algorithm 1).
 *   queries          [B][d]  query embeddings (cache dtype)
 *   lookahead_emb    [B][d]  embedding of each query's first k decoded tokens (cache dtype)
 *   lookahead_tokens [B][k]  int32 token IDs of that prefix
 *   tau_q, tau_r     finite thresholds of stage 1 and stage 2 (compared with >=)
 *   k                1 <= k <= k_cap: number of prefix tokens compared
 * Outputs, each [B]:
 *   idx         entry of highest cosine similarity (lowest index among exact
 *               ties), reported even on a miss; -1 only when the cache is empty
 *   score       that similarity, clamped to [-1, 1]; NaN when the cache is empty
 *   resp_score  prefix-embedding cosine with entry idx, clamped to [-1, 1];
 *               quiet NaN (0x7FC00000) when stage 2 did not run
 *   decision    LACACHE_MISS / REJECT / HIT / HIT_EXACT
 * Similarities are dot products of the bfloat16-rounded normalised vectors,
 * accumulated in float32.  B == 0 is a no-op.  Only for a cache with m = 1
 * (else LACACHE_EINVAL).
 * A lookup (this call and lacache_lookup_ensemble) only enqueues kernels on
 * the stream: no allocation, memory set, copy or host synchronisation.  It
 * can therefore be captured into a HIP graph (with profiling off) and
 * replayed.  A captured lookup keeps what was fixed at capture time: the
 * argument pointers, B, k, the thresholds, the number of stored entries and
 * the stage-1 kernel chosen for them.  Entries inserted after the capture
 * are not searched until the lookup is captured again.
 */
int lacache_lookup(lacache_t h, const void *queries, const void *lookahead_emb, const int32_t *lookahead_tokens,
                   int32_t B, float tau_q, float tau_r, int32_t k, int32_t *idx, float *score, float *resp_score,
                   int32_t *decision, void *stream);

/*
 * lacache_lookup for any m (Section 4.4 ensemble):
 *   lookahead_emb  HOST array of m device pointers, lookahead_emb[i] being
 *                  [B][d_resp[i]] (cache dtype): the lookahead prefix under model i
 *   tau_r          HOST array of m finite stage-2 thresholds, one per model
 *   resp_score     [B][m]: cosine of each model's prefix embeddings, clamped to
 *                  [-1, 1]; quiet NaN in every column when stage 2 did not run
 * decision is HIT_EXACT when the k tokens are identical, HIT when every
 * model's cosine is >= its tau_r[i], REJECT otherwise, MISS on a stage-1
 * miss.  Every other argument and output is as in lacache_lookup.
 */
int lacache_lookup_ensemble(lacache_t h, const void *queries, const void *const *lookahead_emb,
                            const int32_t *lookahead_tokens, int32_t B, float tau_q, const float *tau_r, int32_t k,
                            int32_t *idx, float *score, float *resp_score, int32_t *decision, void *stream);

/* Number of entries inserted so far (host-side count); -1 for a NULL handle. */
int64_t lacache_size(lacache_t h);

/*
 * Copy entries first .. first+n-1 of the store out, as stored: keys_bf16 is
 * [n][d] and emb_bf16 [n][d_resp[0]] bfloat16 bit patterns (prefix model 0),
 * tokens [n][k_cap] int32.  Any of the three may be NULL to skip it.
 * Requires 0 <= first, n >= 0, first + n <= size.  For inspection and tests.
 */
int lacache_export(lacache_t h, int64_t first, int32_t n, uint16_t *keys_bf16, uint16_t *emb_bf16, int32_t *tokens,
                   void *stream);

/* As lacache_export, for the stored prefix embeddings of model 0 <= model < m: emb_bf16 is [n][d_resp[model]]. */
int lacache_export_prefix(lacache_t h, int32_t model, int64_t first, int32_t n, uint16_t *emb_bf16, void *stream);

/*
 * Threshold calibration from benign pairs (Appendix A.2: tau_c = min(0.80, P5)
 * over the cosines of benign paraphrase pairs, tau_a = min(0.70, P10) over the
 * cosines of their response prefixes).
 *   which       -1: the pairs are key-model vectors (dimension d);
 *               0 <= which < m: vectors of prefix model `which` (d_resp[which])
 *   a, b        [n][dim] (cache dtype): pair j is (a[j], b[j]);
 *               1 <= n <= 2^32 - 1 (the selection counts ranks in 32 bits)
 *   percentile  0 .. 100; the percentile is linear between the closest ranks,
 *               h = (n - 1) * percentile / 100, from the order statistics
 *               floor(h) and floor(h) + 1 (computed in double)
 *   cap         finite upper cap of the threshold
 * Outputs (device): sims [n] float, the pair cosines exactly as the lookup
 * computes similarities (normalised, bfloat16-rounded vectors, float32 sums,
 * clamped to [-1, 1]); tau [2] float: tau[0] = the percentile of sims,
 * tau[1] = min(cap, tau[0]).  Uses the handle's calibration scratch, so
 * calls on one handle must be ordered on one stream.  EINVAL for an invalid
 * which, n, percentile or cap, or a NULL pointer.
 */
int lacache_calibrate(lacache_t h, int32_t which, const void *a, const void *b, int64_t n, float percentile,
                      float cap, float *sims, float *tau, void *stream);

/*
 * lacache_calibrate without a handle and without allocating: for callers that
 * cannot allocate device memory (code under HIP graph capture, tight serving
 * loops, harnesses that forbid allocation).  The same pair cosines, selection
 * and outputs as lacache_calibrate, for n pairs of d-dimensional vectors of
 * the given dtype, on the calling thread's current device and on `stream`.
 * The selection's scratch (its state and two 2048-bin histograms, 16.6 KB)
 * is a static array of the library's device image: one copy per GPU, held
 * until the process ends, its size fixed whatever n and d are; it is cleared
 * by the call itself, so calls ordered on one stream are independent, while
 * calls that overlap on one GPU (other streams, other threads) race on it.
 *   1 <= d <= 16384; 1 <= n <= 2^32 - 1; 0 <= percentile <= 100; cap finite;
 * EINVAL otherwise or for a NULL pointer; EHIP for a HIP failure.
 */
int lacache_calibrate_noalloc(const void *a, const void *b, lacache_dtype dtype, int32_t d, int64_t n,
                              float percentile, float cap, float *sims, float *tau, void *stream);

/*
 * Speculative-decoding acceptance after a miss or a rejected lookahead
 * (Section 4.3): the k draft tokens of the draft model g are verified by the
 * target model f in one forward pass; token t_j is accepted when
 * P_f(t_j) >= P_g(t_j), from the first token on, and f takes over at the
 * first failure.  Needs no cache handle; runs on the calling thread's current
 * device.
 *   logits        [B][k][V] (dtype): f's logits at each draft position
 *   draft_tokens  [B][k] int32 draft token IDs; an ID outside [0, V) has probability 0
 *   p_draft       [B][k] float: P_g of each draft token
 *   1 <= V, 0 <= B, 1 <= k <= 4096
 * Outputs: p_target [B][k] float = softmax(logits[b][j])[t_j] (float32
 * arithmetic, max-shifted exponentials); accept_len [B] int32 = the number
 * of leading positions with p_target >= p_draft (0 .. k).  Every row needs at
 * least one finite logit.  B == 0 is a no-op.
 */
int lacache_accept_length(const void *logits, lacache_dtype dtype, int32_t V, const int32_t *draft_tokens,
                          const float *p_draft, int32_t B, int32_t k, int32_t *accept_len, float *p_target,
                          void *stream);

/*
 * Locality-sensitive index for stage 1 (Section 3, Eq. (1): the cache key is
 * an LSH of the embedding, colliding with probability above p1 for close
 * pairs and below p2 for far ones; Algorithm 1 searches the cache with it).
 * Random hyperplanes, the LSH family of cosine distance: bit i of a stored or
 * query vector z (normalised and bfloat16-rounded) is 1 when the projection
 * r_i . z (bf16 products, float32 sums) is >= 0; bits are packed 32 to a word,
 * bit i in word i / 32 at position i % 32.
 *
 * lacache_enable_lsh: hyperplanes [bits][d] bfloat16 (device; not
 * normalised; their entries are the random numbers the index draws), bits a
 * multiple of 32 in 32 .. 256, max_candidates 1 .. 65536 entries kept per
 * query.  Allocates the index (signatures [capacity][bits / 32] and per-query
 * candidate lists), waits for `stream`, and computes the signatures of every
 * stored entry; later inserts add theirs.  Calling it again replaces the index
 * (in the same buffers if bits and max_candidates are the same).
 */
int lacache_enable_lsh(lacache_t h, int32_t bits, const uint16_t *hyperplanes, int32_t max_candidates, void *stream);

/*
 * lacache_lookup with the LSH index as stage 1 (caches with one prefix model):
 * the candidates of a query are the entries whose signature differs from the
 * query's in at most `radius` bits (0 .. bits; 0 is equality of hash keys,
 * bits makes every entry a candidate); among them the entry of highest exact
 * similarity (lowest index on ties) is the stage-1 result, then the
 * threshold and stage 2 as in lacache_lookup.  With no candidate: idx -1,
 * score NaN, MISS.  n_cand [B] int32 receives each query's candidate count;
 * a count above max_candidates means only max_candidates of them (in no
 * particular order) were ranked.  Other arguments and outputs as in
 * lacache_lookup.  LACACHE_EINVAL if the index is not enabled.
 */
int lacache_lookup_lsh(lacache_t h, const void *queries, const void *lookahead_emb, const int32_t *lookahead_tokens,
                       int32_t B, float tau_q, float tau_r, int32_t k, int32_t radius, int32_t *idx, float *score,
                       float *resp_score, int32_t *decision, int32_t *n_cand, void *stream);

/* Copy the LSH signatures of entries first .. first+n-1 ([n][bits / 32] uint32, device) out. */
int lacache_export_signatures(lacache_t h, int64_t first, int32_t n, uint32_t *sig, void *stream);

/*
 * Batch-size crossover of stage 1: batches of at most b_small queries use the
 * bandwidth-bound streaming kernel, larger ones the matrix-core GEMM kernel.
 * The streaming kernel runs up to four groups of 64 queries (fewer queries
 * per group for d > 1152; 65 to 128 queries of 769 to 1024 columns as one
 * group).  b_small is -1, or from 0 up to the streaming
 * kernel's largest batch (256 for d <= 1152); anything else is EINVAL.
 * 0 sends every batch to the GEMM kernel.  -1 (the default) lets each call
 * choose from the number of stored entries n and the padded dimension d_pad:
 * one query group when n * d_pad >= 2^29, two when n * d_pad >= 2^27, three
 * below that.  Each added group costs the streaming kernel a share of the
 * contraction on every CU, so the more keys there are, the sooner the GEMM
 * kernel is faster.  Both kernels accumulate every score with the same
 * matrix instruction sequence, so their results are bit-identical.
 */
int lacache_set_small_batch(lacache_t h, int32_t b_small);

/*
 * Timing of the stage-1 kernel.  The time of a launch is that kernel's from
 * start to end, which holds other parts of a lookup too: the normalisation of
 * the queries up to 32 queries of d <= 2048; and, where the lookup is that one
 * launch, the merge of the candidates, the threshold and stage 2 (up to 8
 * queries, 16 on stores of n * d_pad <= 2^23, of d <= 1024, if queries times
 * the padded columns of all prefix models are at most 12288, outside a stream
 * capture).  With every = n > 0, the 1st, (n+1)-th,
 * (2n+1)-th ... stage-1 launch from now on (one per lookup, or per chunk of
 * max_batch queries) is timed: the launch goes through hipExtLaunchKernel
 * with a HIP event pair that takes the kernel's own start and end times, on
 * the lookup's stream.  every = 0 stops timing.  profile_read waits for
 * those events, returns the total elapsed milliseconds and the number of
 * launches timed (host pointers), and clears the record; calling
 * lacache_profile also clears it.  The events are created here (256 pairs,
 * more only when a window outgrows them) and reused.  Timing every launch
 * costs a few microseconds per lookup, which matters only for lookups that
 * take tens of microseconds; sampling every n-th launch spreads that cost.
 * Errors: EINVAL for a null handle or pointer or every < 0, EHIP.
 */
int lacache_profile(lacache_t h, int32_t every);
int lacache_profile_read(lacache_t h, double *stage1_ms, int64_t *lookups);

/*
 * Health counter of the large-batch stage 1.  Its GEMM kernel reports, per
 * query, the 16-row group holding the best score; the exact row is then
 * recovered by recomputing that group's 16 scores with the same matrix
 * instruction sequence and taking the lowest row whose score equals the
 * reported one (lowest index on ties, Algorithm 1's single hit entry).  If no
 * row reproduces the score, the lowest row at the recomputed maximum is
 * taken instead, so the lookup still names a valid entry, and this counter
 * is incremented.  *count (host pointer) receives the number of such queries
 * since create; it is 0 in correct operation.  Synchronises the device.
 * Errors: EINVAL for a null handle or pointer, EHIP.
 */
int lacache_replay_fallbacks(lacache_t h, int64_t *count);

/*
 * The decode step's own operators.  After a miss or a rejected lookahead the
 * draft model g decodes k tokens (Section 4.3) and the target model f verifies
 * them in one forward pass; both keep the keys and values of earlier tokens.
 * The four calls below are that cache: rotary positions, writing new tokens
 * into pages (in bfloat16 or 8 bits), reading them back, and the attention of
 * a sequence's newest tokens over all of its cached ones.  They need no cache
 * handle, run on the calling thread's current device, allocate nothing and
 * only enqueue kernels, so they can be captured into a HIP graph.  What a
 * captured call keeps is its arguments; lengths and page tables are read on
 * the device at every replay.
 */

/* How a pool stores a number: 8-bit codes have one float scale a token and head (value = code * scale). */
typedef enum { LACACHE_KV_BF16 = 1, LACACHE_KV_FP8 = 2 /* e4m3 */, LACACHE_KV_INT8 = 3 } lacache_kv_type;

/*
 * A paged key-value cache: memory of the caller, described on the host.
 * n_pages pages of `page` tokens (32, 64, 128 or 256) for `heads` heads of d
 * columns (a multiple of 8, 8 .. 256).  Columns are padded to D = 64, 96, 128,
 * 192 or 256, the padding is stored as zeros.  k and v are
 * [n_pages][heads][page / 32] tiles of 32 tokens x D columns, 16-byte aligned.
 * With t = 16 b + r = 16 s + 4 g + i a token of the tile and
 * c = 32 x + 8 u + e = 32 x + 16 y + m a column (b, s, y < 2; r, m < 16;
 * g, i, u < 4; e < 8), the elements of a tile are ordered, last index fastest,
 *     k, bfloat16  [x][b][u][r][e]        k, 8 bits  [x][u][r][b][e]
 *     v, bfloat16  [x][y][g][m][s][i]     v, 8 bits  [x][g][m][y][s][i]
 * which are the operands of the matrix instructions of lacache_kv_attend, 16
 * bytes a lane.  k_scale and v_scale are [n_pages][heads][page] floats, NULL
 * for LACACHE_KV_BF16.  Whatever memory holds where no token has been written
 * (NaN too) has no effect on any result.
 */
typedef struct {
    void *k, *v;
    float *k_scale, *v_scale;
    int64_t n_pages;
    int32_t page, heads, d;
    lacache_kv_type type;
} lacache_kv;

/*
 * The sequences of a call (device arrays).  Rows start[b] .. start[b+1]-1 of
 * the call's packed row arrays are the newest tokens of sequence b
 * (0 <= start[0], start non-decreasing; at most 2^31 - 1 rows); lens[b] is the
 * number of tokens that it has with them, so row start[b] + i is position
 * lens[b] - (start[b+1] - start[b]) + i.  Position p lies at place p % page of
 * page pages[b][p / page].  Rows of negative positions are positions that do
 * not exist.  A page number outside 0 .. n_pages-1 is a page that is not there
 * (given back by a sliding window, for example), and so is a position beyond
 * max_pages pages: nothing is written there, reads give zeros, and attention
 * does not see it.
 */
typedef struct {
    const int32_t *start;  /* [n_seq + 1] */
    const int32_t *lens;   /* [n_seq] */
    const int32_t *pages;  /* [n_seq][max_pages] */
    int32_t n_seq, max_pages;
} lacache_seqs;

/*
 * Rotary positions.  The pairs of a head's first `rot` columns (even, 2 .. d)
 * are turned: (a, b) -> (a c - b s, b c + a s) with the (c, s) of the position
 * and pair in table [n_pos][rot / 2][2]; products and sums are rounded to
 * float32 one by one.  Pair i is columns (i, i + rot / 2) (LACACHE_ROPE_HALF) or
 * (2 i, 2 i + 1) (LACACHE_ROPE_PAIRS).  Positions outside the table take its
 * nearest row.
 */
typedef enum { LACACHE_ROPE_HALF = 0, LACACHE_ROPE_PAIRS = 1 } lacache_rope_style;
typedef struct {
    const float *table;
    int64_t n_pos;
    int32_t rot;
    lacache_rope_style style;
} lacache_rotary;

/*
 * Fill rows first .. first+n-1 of a table (`table` points at row first):
 * f_i = base^(-2 i / rot), table = magnitude * (cos, sin)(position * f_i'), in
 * double, rounded once.  Scaling for long contexts, by parts: with
 * r = original * f_i / (2 pi) turns over the original length,
 * g = clamp((r - low) / (high - low), 0, 1), f_i' = (1 - g) f_i / factor + g f_i.
 * factor = 1 leaves the frequencies as they are; original = 0 divides all of
 * them by factor (linear interpolation of positions).
 *   n >= 0, first >= 0, rot even, 2 .. 256, base > 1, factor >= 1,
 *   original >= 0, 0 <= low < high, magnitude finite; EINVAL otherwise.
 */
int lacache_rope_table(float *table, int64_t first, int64_t n, int32_t rot, double base, double factor,
                       double original, double low, double high, double magnitude, void *stream);

/*
 * y = x turned by the positions of its rows; columns from rot on are copied.
 *   x, y   rows of H heads of d columns (dtype), row t at x + t * x_row, head h
 *          at + h * x_head elements (y likewise, and no two of its rows and
 *          heads share elements); y may be x itself with the same strides, and
 *          must not overlap it otherwise
 *   pos    [rows] int32
 *   backward != 0: the transposed rotation, so that with dy in x the result is
 *          dx: the gradient with respect to the input
 *   1 <= H, 1 <= d <= 4096.  rows == 0 is a no-op.
 */
int lacache_rope(const void *x, void *y, lacache_dtype dtype, int64_t rows, int32_t H, int32_t d, int64_t x_row,
                 int64_t x_head, int64_t y_row, int64_t y_head, const int32_t *pos, const lacache_rotary *rope,
                 int32_t backward, void *stream);

/*
 * Store the newest tokens of every sequence: k is turned by its position (if
 * rope is given) and v is taken as it is, in float32; both are rounded once, to
 * nearest-even, to bfloat16, or to 8-bit codes x * (top / m), m the largest
 * magnitude of the token's head, top = 448 (fp8) or 127 (int8), with the scale
 * m / top (m below 2^-100 stores zeros; a head that holds an infinity or NaN
 * has a scale of NaN, and all of it reads as NaN).
 *   k, v   [rows][heads][d] (dtype), rows k_row and v_row elements apart
 *   q      [rows][q_heads][d], rows q_row elements apart: turned by its
 *          position and written to q_out [rows][q_heads][d], contiguous; q_out
 *          may be q if that is contiguous.  Both NULL, or neither (then rope is
 *          needed).
 *   max_new  a bound on the new tokens of a sequence (for the launch shape
 *          alone; 0: not known)
 * Positions that do not exist are not stored.  Rows before start[0] or from
 * start[n_seq] on are not read, and their q_out is not written.
 */
int lacache_kv_append(const lacache_kv *kv, const lacache_seqs *seqs, const void *k, const void *v,
                      lacache_dtype dtype, int64_t rows, int64_t k_row, int64_t v_row, const void *q, void *q_out,
                      int32_t q_heads, int64_t q_row, const lacache_rotary *rope, int32_t max_new, void *stream);

/*
 * Read the newest tokens of every sequence back as the values they stand for,
 * rounded once to dtype: k_out and v_out [rows][heads][d], contiguous; either
 * may be NULL.  (With start the running sum of lens, that is all tokens.)
 */
int lacache_kv_read(const lacache_kv *kv, const lacache_seqs *seqs, void *k_out, void *v_out, lacache_dtype dtype,
                    int64_t rows, int32_t max_new, void *stream);

/*
 * Attention of the newest tokens of every sequence over its cached ones.
 *   q     [rows][q_heads][d] (dtype), rows q_row elements apart, already
 *         turned; q_heads a multiple of heads, query head h reads head
 *         h / (q_heads / heads)
 *   The row of position p sees the positions j <= p that exist, with
 *   p - j < window if window > 0:
 *   out   [rows][q_heads][d] (dtype) = sum_j w_j v_j, w = softmax(scale q.k_j)
 *   lse   [rows][q_heads] float = log sum_j exp(scale q.k_j); NULL: not wanted.
 *         A row that sees nothing, or whose every score is -infinity, has
 *         out = 0 and lse = -infinity.
 *         An infinity or NaN among the values makes its column of the rows
 *         that see it infinite or NaN; a query or key that makes a score NaN
 *         or +infinity makes the row NaN.  A score of -infinity is the weight
 *         0; with float32 rows, whose queries are sums of terms, an infinite
 *         key may make it NaN.  No other row's results change.
 * Products are exact and sums are in float32; with bfloat16 rows the weights
 * are rounded to 16 bits before they multiply the values.
 *   max_new    a bound on the new tokens of a sequence (for the launch shape
 *              alone; 0: not known)
 *   workspace  lacache_kv_attend_workspace bytes of device memory (the same for
 *              any number of sequences), 16-byte aligned, zero before the first
 *              call that uses them; a call leaves its counters there at zero.
 *              For one call at a time: calls that overlap on one workspace
 *              give wrong results, until it is cleared again
 * EINVAL too if workspace_bytes is less, if rows q_heads / heads is 2^31 or more,
 * or if there could be more than 2^30 row groups (a row group is 16 rows or more
 * of one sequence and kv head; the pieces of work are counted in 32 bits).
 */
int64_t lacache_kv_attend_workspace(const lacache_kv *kv, lacache_dtype dtype, int32_t n_seq, int32_t q_heads,
                                    int32_t max_new);
int lacache_kv_attend(const lacache_kv *kv, const lacache_seqs *seqs, const void *q, lacache_dtype dtype,
                      int64_t rows, int32_t q_heads, int64_t q_row, int32_t max_new, float scale, int32_t window,
                      void *out, float *lse, void *workspace, int64_t workspace_bytes, void *stream);

/* Static text for a return code. */
const char *lacache_strerror(int code);

#ifdef __cplusplus
}
#endif

#endif /* LACACHE_H */
