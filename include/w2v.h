/*
 * w2v.h — C ABI of the MI355X (gfx950) hierarchical-softmax word2vec library.
 *
 * The library trains skip-gram (and CBOW) word vectors against a hierarchical
 * softmax, as in Vuurens, Eickhoff and de Vries, "Efficient Parallel Learning
 * of Word2Vec" (Algorithm 1, Cached Skipgram HS), including the paper's
 * remedy for update collisions: the vectors of the top inner nodes of the
 * Huffman tree are cached per worker and their change is written back
 * periodically (§3.2). On the GPU the cache owner is a workgroup and the
 * cache lives in LDS.
 *
 * Conventions (all entry points):
 *   - Every pointer is a DEVICE pointer unless its name ends in _host.
 *   - The caller owns all memory; the library never allocates device memory.
 *     Scratch space comes in through (workspace, workspace_bytes); each call
 *     has a *_workspace_bytes() query.
 *   - Work is stream-ordered on hip_stream (a hipStream_t; NULL = the null
 *     stream). Calls that write *_host outputs synchronise that stream before
 *     returning; the others return without synchronising.
 *   - Return value: W2V_OK or a negative w2v_status. Arguments are checked
 *     before anything is launched; on W2V_E_ARG / W2V_E_RANGE /
 *     W2V_E_WORKSPACE no output has been touched. On W2V_E_DEVICE outputs are
 *     undefined. w2v_last_error() gives a message for the calling thread.
 *   - Calls on different streams with disjoint buffers may run concurrently;
 *     the only global state is the per-thread error message and a per-device
 *     cache of device properties and timing events.
 */
#ifndef W2V_H
#define W2V_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    W2V_OK = 0,
    W2V_E_ARG = -1,        /* a null pointer, a size out of range, an inconsistent setting */
    W2V_E_RANGE = -2,      /* data out of range: a token id outside [0, id_space), a code longer than 64 */
    W2V_E_WORKSPACE = -3,  /* workspace_bytes below what the *_workspace_bytes query returns */
    W2V_E_DEVICE = -4      /* a HIP runtime error (launch failure, fault surfaced at a synchronisation) */
} w2v_status;

/* Message for the calling thread's last non-OK return ("" if none). */
const char *w2v_last_error(void);

/* ------------------------------------------------------------------------
 * Vocabulary (the "mintf" setting of §4.1; Algorithm 1 iterates over word
 * ids of the text).
 *
 * Counts every id in tokens[0..n_tokens), keeps the ids whose count is at
 * least min_count and orders them by (count descending, id ascending); the
 * position in that order is the vocabulary index 0..V-1.
 *   tokens        int32[n_tokens], ids in [0, id_space)
 *   counts_by_id  int64[id_space]  out: occurrences of each id
 *   vocab_ids     int32[id_space]  out: id of vocabulary index r (r < V); -1 beyond V
 *   vocab_counts  int64[id_space]  out: count of vocabulary index r (r < V); 0 beyond V
 *   id_to_vocab   int32[id_space]  out: vocabulary index of each id, -1 if dropped
 *   tokens_out    int32[n_tokens]  out, may be NULL: tokens mapped to vocabulary
 *                                  indices (-1 = dropped); may not alias tokens
 *   V_host, train_words_host       out: V and the sum of kept counts
 * Errors: W2V_E_RANGE if a token lies outside [0, id_space) (outputs are then
 * written but invalid); W2V_E_ARG if id_space < 1, n_tokens < 0 or
 * min_count < 0. Synchronises the stream.
 * ---------------------------------------------------------------------- */
size_t w2v_build_vocab_workspace_bytes(int32_t id_space);
int w2v_build_vocab(const int32_t *tokens, int64_t n_tokens, int32_t id_space, int64_t min_count,
                    int64_t *counts_by_id, int32_t *vocab_ids, int64_t *vocab_counts, int32_t *id_to_vocab,
                    int32_t *tokens_out, int32_t *V_host, int64_t *train_words_host, void *workspace,
                    size_t workspace_bytes, void *hip_stream);

/* ------------------------------------------------------------------------
 * Huffman tree (§2: the output layer is a binary Huffman tree; a word is
 * predicted by the turns at the inner nodes on its path from the root).
 *
 * Built from vocab_counts[0..V) (descending) by the two-queue merge: leaves in
 * ascending count (vocabulary index V-1 first), inner nodes in creation order;
 * each merge takes the smaller front twice, a leaf winning a count tie; the
 * first child taken gets bit 0; merge a creates inner node a; the root is V-2.
 *   codelen    uint8[V]     out: depth of each word
 *   code       uint64[V]    out: bit j = turn at the j-th inner node from the root
 *   point_off  int32[V+1]   out: word v's inner nodes are points[point_off[v] ..
 *                           point_off[v+1]), root first
 *   points     int32[points_cap] out; NULL = size query (only codelen, code,
 *                           point_off and the host outputs are written)
 *   points_len_host, max_len_host  out: sum of code lengths, longest code
 * Errors: W2V_E_ARG if V < 2, vocab_counts is not in descending order, or
 * points_cap < sum of lengths (points given); W2V_E_RANGE if a code would be
 * longer than 64. Synchronises the stream.
 * ---------------------------------------------------------------------- */
size_t w2v_build_huffman_workspace_bytes(int32_t V);
int w2v_build_huffman(const int64_t *vocab_counts, int32_t V, uint8_t *codelen, uint64_t *code,
                      int32_t *point_off, int32_t *points, int64_t points_cap, int64_t *points_len_host,
                      int32_t *max_len_host, void *workspace, size_t workspace_bytes, void *hip_stream);

/* ------------------------------------------------------------------------
 * Model and training settings.
 *
 * syn0 ("vector[w]" of Algorithm 1) is float[V][row_stride], syn1
 * ("weight[n]", the inner-node vectors) is float[V-1][row_stride]; only the
 * first dim floats of a row are used. row_stride >= dim, a multiple of 4;
 * both arrays 16-byte aligned. Training may write zeros into a row's padding
 * columns (dim .. row_stride-1); their contents are otherwise ignored.
 * ---------------------------------------------------------------------- */
typedef struct {
    float *syn0;
    float *syn1;
    int32_t V, dim, row_stride;
    int32_t reserved0;
    const int64_t *vocab_counts;  /* int64[V] from w2v_build_vocab (keep probabilities) */
    int64_t train_words;          /* sum of vocab_counts (N_t) */
    const uint8_t *codelen;       /* from w2v_build_huffman */
    const uint64_t *code;
    const int32_t *point_off;
    const int32_t *points;
} w2v_model;

typedef struct {
    int32_t arch;            /* 0 = skip-gram (Algorithm 1), 1 = CBOW (mean of the window as input),
                                2 = skip-gram with the reversed orientation: for each window word w in order
                                the path of w is walked with the centre's vector as input, which gains that
                                pair's hidden-layer gradient before the next pair (asynchronous mode only) */
    int32_t mode;            /* 0 = asynchronous (lock-free, top-k cache in LDS), 1 = synchronous batches
                                (skip-gram, arch 0, only) */
    int32_t window;          /* W ("windowsize", §4.1), 1..10; effective half-width uniform on 1..W */
    int32_t doc_len;         /* documents of doc_len raw tokens (1..65535); windows never cross them */
    double sample;           /* subsampling threshold t ("downsample", §4.1); 0 = keep all */
    float alpha0;            /* initial learning rate */
    int32_t epoch, n_epochs; /* this epoch and the total, for the learning-rate schedule */
    int32_t reserved1;
    int64_t corpus_tokens;   /* raw tokens of one epoch (the whole corpus, for the schedule) */
    int64_t first_raw_index; /* global raw index of tokens[0]; a multiple of doc_len */
    uint64_t seed;           /* Philox4x32-10 key for subsampling and window draws */
    int32_t cache_k;         /* inner nodes cached per workgroup ("isFrequent"): the k created last */
    int32_t flush_every;     /* write the cache back after this many centre words per workgroup (>= 1) */
    int32_t sync_batch;      /* synchronous mode: kept centres per batch (>= 1) */
    int32_t workers;         /* wavefronts that take documents; 0 = fill the GPU; 1 = one sequential worker */
    int32_t write_policy;    /* bit 0: uncached inner-node rows are stored (lock-free, concurrent updates may be
                                overwritten, as in Hogwild) instead of atomically adding their change;
                                bit 1: the same for the word vectors syn0 (a word repeated within a window
                                stores at its first position and adds the change of the others);
                                bit 2: the same for the cached rows in the workgroup's LDS copy;
                                bit 3 (needs bit 1): word rows kept across centres -- a wavefront
                                holds the rows of the kept words within `window` positions of its centre in
                                registers while it walks a document's centres in order, loading a row when it
                                enters that span and storing it when it leaves or becomes the centre (one read
                                and write per word and span instead of one per pair). Applies to rows of 129 to
                                512 floats with window <= 5: CBOW always, skip-gram on the store-only walk
                                (bit 0; bit 2 when cache_k > 0; hot_k 0; cache_mode 0) and with window <= 2
                                above 320 floats; elsewhere the bit is ignored; w2v_train_word_span reports
                                which */
    int32_t flush_policy;    /* cache write-back: 0 = add the change (cached - original), the write-back of
                                §3.2 as printed (stable at a few hundred wavefronts; at full occupancy the
                                top rows' summed stale changes diverge); 1 = add the change divided by the
                                number of workgroups, so that their progress on the cached rows is averaged
                                (local SGD on those rows) -- a departure from §3.2, and the default */
    int32_t hot_k;           /* with write_policy bit 0: the hot_k inner nodes created just before the cached
                                ones (on most paths, so the most contended rows) still take atomic adds of
                                their change; >= 0 */
    int32_t negative;        /* negative sampling (w2v_train_ns_epoch, w2v_ns_objective): negatives per centre,
                                shared by its window words; 1..11 (1..7 above 320 columns); ignored elsewhere */
    int32_t cache_mode;      /* asynchronous mode's cache: 0 = each workgroup holds a copy of the cached rows and
                                their values at the last write-back, whose difference it writes back (§3.2);
                                1 = delta-only: it holds just its change since the last write-back, reads a
                                cached row as the HBM row plus that change and adds its updates to the change
                                with LDS atomics (write_policy bit 2 does not apply); half the LDS per row */
    int32_t span_refresh;    /* with write_policy bit 3 in effect: the words of vocabulary index below this
                                (the most frequent) are written back, if changed, and read again after every
                                centre while they stay in the span, so that other wavefronts' updates to them
                                are lost for one centre at most, as without bit 3; 0 = off; >= 0 */
    int32_t span_stash;      /* with write_policy bit 3 in effect: 1 = the row of the word that
                                becomes the next centre waits in a per-wavefront LDS row while that word is the
                                centre, and re-enters the span from there instead of from memory (one row read
                                less per centre when the row fits beside the cache), so other wavefronts'
                                updates to it during that centre are lost when it is stored again (for the
                                frequent words, with many wavefronts, this lowers the held-out log-likelihood
                                and widens its run-to-run spread: see stash_from); 0 = off (the default) or 1 */
    int32_t stash_from;      /* with span_stash 1: only words of vocabulary index >= stash_from (the less
                                frequent ones, whose rows few other wavefronts update meanwhile) re-enter from
                                the stash; the more frequent ones are read again from memory (10000 at V = 1M
                                keeps the log-likelihood of the run without the stash); >= 0 */
} w2v_params;

/* stats int64[5]: raw tokens, in-vocabulary tokens, kept centre words, (centre, context) pairs,
   node updates (pair-node updates for skip-gram, centre-node updates for CBOW). */
#define W2V_N_STATS 5

/* ------------------------------------------------------------------------
 * One training pass over tokens[0..n_tokens) (vocabulary indices, -1 =
 * dropped), updating m->syn0 and m->syn1 in place.
 *
 * Per kept centre word v (subsampling: keep with probability
 * min(1, sqrt(q) + q), q = t N_t / count(v), drawn from Philox4x32-10 keyed
 * by (seed; raw index, epoch)), with window words w_1..w_P (the kept words of
 * the same document within the effective half-width), the path of v is
 * walked once; at each inner node n with turn t and every window word in
 * order: f = sigmoid(syn0[w].syn1[n]), g = (1 - t - f) alpha, the
 * hidden-layer gradient of w gains g syn1[n] and syn1[n] gains g syn0[w];
 * afterwards each syn0[w] gains its hidden-layer gradient (Algorithm 1 with
 * the window and node loops swapped, which is the same computation whenever
 * a window holds no repeated word). alpha decays linearly with the raw stream
 * position in steps of 10,000 tokens down to 1e-4 alpha0.
 *
 * mode 0: segments of up to 128 kept centres of a document are claimed by
 * wavefronts from a queue (in stream order); the top cache_k
 * inner-node vectors live in each workgroup's LDS and are written back as a
 * change (cached - original) every flush_every centres (§3.2); other rows are
 * updated in HBM, by atomic adds of their change or, as write_policy selects,
 * by stores of the new row. Lock-free: results vary with scheduling, as in
 * the paper's Hogwild setting, except with workers=1.
 * mode 1: every gradient of a batch of sync_batch consecutive kept centres
 * uses the model at the start of the batch; the sums (exact int64 fixed
 * point, 40 fraction bits) are applied at its end. Deterministic. A row's
 * change within one batch must stay below 2^23 in magnitude (the fixed
 * point's range); a batch that large has diverged (e.g. batches of hundreds
 * of centres over a vocabulary of a few dozen words). Synchronises the
 * stream once (to read the number of kept centres).
 * stats: int64[W2V_N_STATS] device buffer, overwritten (may be NULL).
 * Errors: W2V_E_ARG for a bad model/params (V < 2, dim not in 1..1024,
 * window not in 1..10, cache_mode not 0 or 1, LDS budget exceeded: 2 cache_k
 * rows (1 with the delta-only cache) of 4-byte floats,
 * a row being dim rounded up to 64, 128, 256, 320 or 512 for dim <= 512 and
 * dim above, plus, for dim <= 512, 2 KiB of centre records per wavefront of
 * a workgroup (16 wavefronts for dim <= 64, 12 for dim <= 320, 8 above), ...).
 * ---------------------------------------------------------------------- */
size_t w2v_train_workspace_bytes(const w2v_model *m, int64_t n_tokens, const w2v_params *p);
int w2v_train_hs_epoch(const w2v_model *m, const int32_t *tokens, int64_t n_tokens, const w2v_params *p,
                       int64_t *stats, void *workspace, size_t workspace_bytes, void *hip_stream);

/* Half-width of the word-row span that w2v_train_hs_epoch keeps in registers
   for these arguments (write_policy bit 3): the rows of the kept words within
   that many positions of the centre stay in registers across centres; 0 when
   every centre reads and writes its window rows itself. Host-side, no launch;
   returns -1 for a NULL pointer or an invalid model or parameter block
   (w2v_last_error says which). */
int32_t w2v_train_word_span(const w2v_model *m, const w2v_params *p);

/* Duration in milliseconds of the main training kernel of the last
   w2v_train_hs_epoch call on the calling thread's current device (HIP events
   recorded on that call's stream). Waits for that kernel to finish. */
int w2v_last_train_kernel_ms(float *ms_host);

/* Launch shape of the main training kernel of the last asynchronous
   w2v_train_hs_epoch call on the calling thread's current device: workgroups
   (cache owners) and wavefronts that took documents. Host-side, no wait. */
int w2v_last_train_launch(int32_t *workgroups_host, int32_t *wavefronts_host);

/* Resources of that same launch (the last asynchronous hierarchical-softmax
   or negative-sampling training kernel on the calling thread's current
   device): LDS bytes per workgroup (static centre records plus the dynamic
   cache rows), vector registers per lane as the HIP runtime reports them,
   and resident wavefronts per SIMD at that LDS size (occupancy). All three
   are 0 before the first launch. Host-side, no wait. Errors: W2V_E_ARG for a
   NULL pointer. */
int w2v_last_train_resources(int32_t *lds_bytes_host, int32_t *vgprs_host, int32_t *waves_per_simd_host);

/* ------------------------------------------------------------------------
 * Hierarchical-softmax log-likelihood (evaluation, §2's objective): over the
 * (centre, context) pairs that the sampler draws from tokens with p's seed,
 * epoch, window and sample settings, sum_ll = sum of log P(v | syn0[w]) with
 * P(v|x) = prod_j sigmoid((1 - 2 t_j) x . syn1[n_j]) over v's path, and
 * n_pairs = the number of pairs (p->arch 0 or 2).
 * p->arch 1 (CBOW): the same softmax with CBOW's input, one term per sampled
 * centre v that has at least one window word: sum_ll = sum of log P(v | h),
 * h = the mean of the window words' syn0 rows; n_pairs = the number of such
 * centres. n_nodes (may be NULL): the path nodes the terms visit.
 * Skip-gram: dot products in fp32; CBOW: h and its dot products in fp64;
 * logarithms and sums in fp64, summed in a fixed order (deterministic).
 * Read-only on the model. Synchronises the stream. Errors: W2V_E_ARG for a
 * bad model, params (arch outside 0..2) or NULL required pointer,
 * W2V_E_WORKSPACE for a short workspace, W2V_E_DEVICE for a HIP failure.
 * ---------------------------------------------------------------------- */
size_t w2v_hs_loglik_workspace_bytes(const w2v_model *m, int64_t n_tokens, const w2v_params *p);
int w2v_hs_loglik(const w2v_model *m, const int32_t *tokens, int64_t n_tokens, const w2v_params *p,
                  double *sum_ll_host, int64_t *n_pairs_host, int64_t *n_nodes_host, void *workspace,
                  size_t workspace_bytes, void *hip_stream);

/* ------------------------------------------------------------------------
 * w2v_hs_loglik on the library's own scratch memory, for callers that cannot
 * allocate device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc). Same arguments, results and errors as
 * w2v_hs_loglik without the workspace: the workspace is a static device
 * array of w2v_noalloc_scratch_bytes() bytes (64 MiB) that every GPU the
 * library runs on holds until the process ends. The call itself allocates
 * nothing; its first call on a device looks up that device's copy of the
 * array. Evaluations whose w2v_hs_loglik_workspace_bytes exceed the scratch
 * return W2V_E_RANGE before anything is launched (about 11 bytes per token
 * with 1,000-token documents, plus 8 bytes per vocabulary word: e.g. V = 1M
 * with up to about 5.3M tokens). Every call on a device shares that device's
 * scratch, which keeps the last call's contents: calls that overlap on one
 * device (other streams or threads) race on it and must not be issued
 * concurrently. Synchronises the stream.
 * ---------------------------------------------------------------------- */
size_t w2v_noalloc_scratch_bytes(void);
int w2v_hs_loglik_noalloc(const w2v_model *m, const int32_t *tokens, int64_t n_tokens, const w2v_params *p,
                          double *sum_ll_host, int64_t *n_pairs_host, int64_t *n_nodes_host, void *hip_stream);

/* ------------------------------------------------------------------------
 * Negative sampling: the alternative objective to the hierarchical softmax
 * that §2 names, trained in the mini-batch form of Ji et al. that the opening
 * of §3.2 describes (every window word of a centre trains against the same
 * targets, all gradients of the centre taken before any of its updates).
 * For these calls m->syn1 holds the output vectors of the words,
 * float[V][row_stride]; the Huffman arrays of m are not used (may be NULL).
 *
 * w2v_build_noise_table: the noise distribution, unigram counts raised to
 * 3/4, with the weight of count c taken in integers as isqrt(c * isqrt(c)),
 * laid out in table int32[2^log2_size]: entry i holds the vocabulary index
 * v with Q[v] <= floor(i Q / 2^log2_size) < Q[v+1] (Q[v] = weight of the
 * indices below v, Q = total). log2_size in 1..30; total_weight_host gets Q.
 * Errors: W2V_E_ARG for bad sizes or NULL pointers; W2V_E_RANGE if Q is not
 * in [1, 2^(63 - log2_size)). Synchronises the stream.
 * ---------------------------------------------------------------------- */
size_t w2v_noise_table_workspace_bytes(int32_t V);
int w2v_build_noise_table(const int64_t *vocab_counts, int32_t V, int32_t log2_size, int32_t *table,
                          int64_t *total_weight_host, void *workspace, size_t workspace_bytes, void *hip_stream);

/* ------------------------------------------------------------------------
 * One pass of skip-gram with shared negatives over tokens (vocabulary
 * indices, -1 = dropped): the same subsampling, documents, window draws and
 * learning-rate schedule as w2v_train_hs_epoch. Per kept centre v with
 * window words w_1..w_P, its targets are v (label 1) and p->negative
 * negatives (label 0): negative 4h+i is table[r_i >> (32 - log2_size)], r =
 * Philox4x32-10(counter (raw index lo, raw index hi, epoch, 1 + h), key =
 * seed); one equal to v is dropped. With S_qk = syn0[w_q] . syn1[t_k] and
 * g_qk = alpha (label_k - sigmoid(S_qk)), syn0[w_q] gains sum_k g_qk
 * syn1[t_k] and syn1[t_k] gains sum_q g_qk syn0[w_q], all from the values
 * before the centre. Write-back (p->write_policy): bit 0 set, a target row is
 * stored as its value before the centre plus its change (lock-free, as in
 * Hogwild: concurrent changes can be overwritten); bit 1 set, a word row is
 * re-read and stored with its change; otherwise, and for a word or negative
 * repeated within the centre, the change is added atomically. Centres run
 * concurrently, so results vary with scheduling except with workers = 1. stats int64[W2V_N_STATS]: raw tokens, in-vocabulary tokens,
 * kept centres, pairs, pair-target updates. Asynchronous (mode 0) skip-gram
 * only; dim <= 512. Errors as w2v_train_hs_epoch, and W2V_E_ARG for a NULL
 * table, log2_size outside 1..30 or negative out of range.
 * ---------------------------------------------------------------------- */
size_t w2v_train_ns_workspace_bytes(const w2v_model *m, int64_t n_tokens, const w2v_params *p);
int w2v_train_ns_epoch(const w2v_model *m, const int32_t *noise_table, int32_t log2_size, const int32_t *tokens,
                       int64_t n_tokens, const w2v_params *p, int64_t *stats, void *workspace, size_t workspace_bytes,
                       void *hip_stream);

/* Negative-sampling objective (evaluation) over the sampler's pairs drawn
   with p's seed and epoch, each pair with its centre's negatives: sum_host =
   sum over pairs (v, w) of log sigmoid(syn0[w] . syn1[v]) + sum over kept
   negatives n of log sigmoid(-syn0[w] . syn1[n]). Dot products in fp32, logs
   and sums in fp64, in a fixed order (deterministic). n_terms_host (may be
   NULL) = number of log-sigmoid terms. Read-only. Synchronises the stream. */
size_t w2v_ns_objective_workspace_bytes(const w2v_model *m, int64_t n_tokens, const w2v_params *p);
int w2v_ns_objective(const w2v_model *m, const int32_t *noise_table, int32_t log2_size, const int32_t *tokens,
                     int64_t n_tokens, const w2v_params *p, double *sum_host, int64_t *n_pairs_host,
                     int64_t *n_terms_host, void *workspace, size_t workspace_bytes, void *hip_stream);

/* ------------------------------------------------------------------------
 * Operators of a mini-batch step on hidden vectors: layer norm, the
 * hierarchical softmax as a loss with gradients, AdamW. They write no host
 * output and do not synchronise, so they can be captured into a HIP graph
 * (w2v_adamw_build_plan excepted); overlapping calls need workspaces of their
 * own. Rows are dim (cols) neighbouring elements, `stride` elements apart
 * (stride >= dim where there is more than one row); columns between the rows
 * are neither read nor written (but see dsyn1). Any element-aligned address is allowed.
 * bf16 and fp16 elements are converted to fp32 exactly, all arithmetic and
 * sums are fp32 and results are rounded once, to nearest. Sums over rows have
 * a fixed order: equal inputs give equal bits.
 * ---------------------------------------------------------------------- */
typedef enum { W2V_F32 = 0, W2V_BF16 = 1, W2V_F16 = 2 } w2v_type;

/* Layer norm: mean = sum x / dim, rstd = 1 / sqrt(sum (x - mean)^2 / dim + eps),
   y = (x - mean) rstd weight + bias.
     x, y        rows x dim elements of type; y may be x (the same rows, with
                 the same stride), and may not overlap it otherwise
     weight, bias  dim elements of w_type (W2V_F32 or type), each may be NULL (1, 0)
     mean, rstd  float[rows] out, each may be NULL
   With eps 0 a row of equal values has no finite rstd, and its y is NaN.
   Errors: W2V_E_ARG for rows < 0, dim not in 1..16384, a short stride, eps
   that is negative or not finite, an unknown type or a NULL required pointer. */
int w2v_layer_norm(const void *x, int32_t type, int64_t rows, int32_t dim, int64_t x_stride, const void *weight,
                   const void *bias, int32_t w_type, float eps, void *y, int64_t y_stride, float *mean, float *rstd,
                   void *hip_stream);

/* Its gradients, from the upstream gradient dy and the forward pass's x, mean
   and rstd: with h = (x - mean) rstd and a = dy weight,
   dx = rstd (a - sum a / dim - h sum (a h) / dim) (elements of type; may be dy
   or x), dweight = sum over rows of dy h and dbias = sum over rows of dy
   (float[dim], each may be NULL; zeros for rows = 0). */
size_t w2v_layer_norm_backward_workspace_bytes(int64_t rows, int32_t dim);
int w2v_layer_norm_backward(const void *dy, int64_t dy_stride, const void *x, int32_t type, int64_t rows, int32_t dim,
                            int64_t x_stride, const void *weight, int32_t w_type, const float *mean,
                            const float *rstd, void *dx, int64_t dx_stride, float *dweight, float *dbias,
                            void *workspace, size_t workspace_bytes, void *hip_stream);

/* The hierarchical softmax of rows hidden vectors x (rows x m->dim elements of
   type) with target words targets int32[rows], as a loss with its gradients:
     loss    float[rows] out, may be NULL: -log P(targets[i] | x_i), with
             P(v|x) = prod_j sigmoid((1 - 2 t_j) x . syn1[n_j]) over v's path
     dx      rows x dim elements of type out, may be NULL
     dsyn1   float[V-1][dsyn1_stride] out, may be NULL: every row's first dim
             columns are written; where dsyn1_stride is m->row_stride and less
             than dim + 32, zeros are written into the rows' padding columns,
             too (as in training)
   The gradients are those of sum_i weights[i] loss[i] (weights float[rows], or
   NULL: ones). A negative target means none: loss 0, a dx of zeros, x not
   read into any sum. A target outside the vocabulary, or one whose code is
   longer than max_code_len (w2v_build_huffman's max_len_host, 1..64), has the
   loss NaN and no gradient. Of m: V, dim, row_stride, syn1 and the Huffman
   arrays; the others are not used. dx may not overlap x, nor dsyn1 m->syn1. Errors:
   W2V_E_ARG, W2V_E_WORKSPACE (the workspace is needed with dsyn1 only). */
size_t w2v_hs_loss_workspace_bytes(const w2v_model *m, int32_t max_code_len, int64_t rows);
int w2v_hs_loss(const w2v_model *m, int32_t max_code_len, const void *x, int32_t type, int64_t rows, int64_t x_stride,
                const int32_t *targets, const float *weights, float *loss, void *dx, int64_t dx_stride, float *dsyn1,
                int64_t dsyn1_stride, void *workspace, size_t workspace_bytes, void *hip_stream);

/* AdamW with decoupled weight decay, over many tensors in one launch. At step
   t (1, 2, ...), for every element, in fp32:
     g = grad grad_scale;  m = beta1 m + (1 - beta1) g;  v = beta2 v + (1 - beta2) g^2
     p = p (1 - lr weight_decay) - lr / (1 - beta1^t) m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
   The moments of all tensors lie in two arrays of n_moments elements, tensor
   i's (in row order, without gaps) from moment_offset on, a multiple of 256.
   bits = 32: float arrays. bits = 8: uint8 arrays with a scale for each 256
   elements, m_scale and v_scale float[n_moments / 256]: m = e4m3 code x scale,
   sqrt(v) = u x scale with u(c) = c 2^-18 for c < 16, else
   (1 + (c % 16) / 16) 2^(c / 16 - 15). m is rounded to nearest, sqrt(v) up or
   down in proportion by a hash of (seed, t, place of the moment), a positive
   one never to 0. A block with a moment that is not finite stays not finite.
   All zeros is the state before the first step in either form. With eps 0 a
   parameter whose gradients were all zero becomes NaN. */
typedef struct {
    void *param;              /* rows x cols elements of param_type */
    const void *grad;         /* rows x cols elements of grad_type */
    int64_t rows, cols;
    int64_t param_stride, grad_stride;
    int64_t moment_offset;
    int32_t param_type, grad_type;
    float weight_decay;
    int32_t reserved0;
} w2v_adamw_tensor;

typedef struct {
    double lr, beta1, beta2, eps;
    int64_t step;               /* t, >= 1 */
    const float *lr_device;     /* NULL, or the learning rate in device memory (instead of lr) */
    const int64_t *step_device; /* NULL, or t in device memory (instead of step): for steps replayed from a graph */
    float grad_scale;
    uint32_t seed;
} w2v_adamw_params;

/* The plan of a list of tensors: which parts of which tensor a step's
   workgroups update, laid out once in plan, device memory of
   w2v_adamw_plan_bytes bytes that the caller keeps (0: an invalid list).
   n_chunks_host is handed to every step. Synchronises the stream. A plan
   belongs to one step at a time. Errors: W2V_E_ARG for sizes, strides, types
   or NULL pointers out of range, moments that overlap or reach past n_moments
   (a tensor's last block counts whole), or packed parameters that overlap.
   Gradients may share memory with each other, not with a parameter. */
size_t w2v_adamw_plan_bytes(const w2v_adamw_tensor *tensors_host, int32_t n_tensors);
int w2v_adamw_build_plan(const w2v_adamw_tensor *tensors_host, int32_t n_tensors, int64_t n_moments, void *plan,
                         size_t plan_bytes, int64_t *n_chunks_host, void *hip_stream);
int w2v_adamw_step(void *plan, int64_t n_chunks, int32_t bits, void *m, void *v, float *m_scale, float *v_scale,
                   const w2v_adamw_params *p, void *hip_stream);

/* The values that 8-bit moments stand for: m_out, v_out float[n_moments]. */
int w2v_adamw_moments(const void *m, const void *v, const float *m_scale, const float *v_scale, int64_t n_moments,
                      float *m_out, float *v_out, void *hip_stream);

/* ------------------------------------------------------------------------
 * A gated feed-forward block of rows x (rows x dim elements of type), with the
 * weights w_gate, w_up (hidden x dim) and w_down (dim x hidden) of the same
 * type:
 *     g = x w_gate',  u = x w_up',  h = act(g) u,  y = h w_down'
 * act: W2V_SILU, g sigmoid(g), or W2V_GELU, g Phi(g) with the normal
 * distribution's Phi. Strides count elements; dim and hidden are 1..2^20.
 * gate and up (rows x hidden elements of type, may be NULL) receive g and u,
 * which the backward pass takes. y may be x with the same stride; outputs may
 * not overlap any other array. Sums are fp32. With type fp32 the products keep
 * 24 bits of each factor. With 16-bit types h is rounded to type before the
 * second product (one beyond the type's range becomes an infinity), but for few
 * rows it stays fp32: for one, for up to 64 where rows * dim * hidden is at most
 * 2^26, for up to 16 where a weight's rows are not whole aligned 16 bytes or
 * w_gate's and w_up's strides differ. An infinity among the factors of a fp32
 * product may make it NaN. Errors: W2V_E_ARG, W2V_E_WORKSPACE, W2V_E_RANGE
 * (more rows than a launch takes).
 *
 * w2v_gated_ffn_backward: the gradients for an upstream gradient dy (rows x
 * dim), from x, the weights and g and u as the forward pass left them:
 *     dh = dy w_down,  du = dh act(g),  dg = dh u act'(g)
 *     dx = dg w_gate + du w_up,  dw_gate = dg' x,  dw_up = du' x,
 *     dw_down = dy' h
 * Each may be NULL: not wanted. All are of type; the weights' are written, not
 * added to (zeros for rows = 0). dx may be dy or x with the same stride; other
 * outputs may not overlap any array. With 16-bit types dg, du and h are
 * rounded to type between the products.
 *
 * Calls that overlap in time need a workspace each. One of less than the bytes
 * that are named is refused where these arrays need more of it.
 * ---------------------------------------------------------------------- */
enum { W2V_SILU = 0, W2V_GELU = 1 };

typedef struct {
    const void *p;
    int64_t stride;   /* elements from a row to the next */
} w2v_rows;

size_t w2v_gated_ffn_workspace_bytes(int64_t rows, int32_t dim, int32_t hidden, int32_t type);
int w2v_gated_ffn(w2v_rows x, w2v_rows w_gate, w2v_rows w_up, w2v_rows w_down, int64_t rows, int32_t dim, int32_t hidden,
                  int32_t type, int32_t act, w2v_rows y, w2v_rows gate, w2v_rows up, void *workspace,
                  size_t workspace_bytes, void *hip_stream);
size_t w2v_gated_ffn_backward_workspace_bytes(int64_t rows, int32_t dim, int32_t hidden, int32_t type);
int w2v_gated_ffn_backward(w2v_rows dy, w2v_rows x, w2v_rows w_gate, w2v_rows w_up, w2v_rows w_down, w2v_rows gate,
                           w2v_rows up, int64_t rows, int32_t dim, int32_t hidden, int32_t type, int32_t act, w2v_rows dx,
                           w2v_rows dw_gate, w2v_rows dw_up, w2v_rows dw_down, void *workspace, size_t workspace_bytes,
                           void *hip_stream);

/* ------------------------------------------------------------------------
 * Nearly orthogonal matrices by Newton-Schulz products: X = g / (|g| + eps)
 * with the Frobenius norm, then `steps` (1..20) times X = (a I + b A + c A A) X
 * with A = X X' and a, b, c = 3.4445, -4.7750, 2.0315. Five steps bring
 * singular values of 0.002 of the norm or more between 0.68 and 1.21. A step
 * multiplies smaller ones by up to 3.4445 (0.0001 becomes 0.05, 0 stays 0), and
 * so what rounding leaves in directions that g lacks: 1e-4 of the result of a
 * matrix of rank 1 in five steps, all of it in twenty. g and out: batch (up to
 * 2^31 - 1) matrices of rows x cols elements of type (sides up to 2^20), a row
 * `stride` and a matrix `step` elements behind the one before, out's a whole
 * matrix or more; out may be g with the same strides. The products keep 22 bits
 * of each factor and sum in fp32; with type bf16 what is added to X in a step
 * keeps 11, and X itself 22: an error of some 1e-3 of the result in norm in
 * five steps, 3.6e-3 where all of its roundings have one sign (a unit matrix),
 * beside the 1.7e-3 of bf16's rounding. A matrix with an element that is not
 * finite becomes NaN, the others do not; one of zeros stays zero (NaN with eps
 * 0). Errors: W2V_E_ARG, W2V_E_WORKSPACE, W2V_E_RANGE. */
size_t w2v_orthogonalize_workspace_bytes(int64_t batch, int32_t rows, int32_t cols, int32_t type);
int w2v_orthogonalize(const void *g, int64_t g_stride, int64_t g_step, int64_t batch, int32_t rows, int32_t cols,
                      int32_t type, int32_t steps, double eps, void *out, int64_t out_stride, int64_t out_step,
                      void *workspace, size_t workspace_bytes, void *hip_stream);

/* Muon over many matrices: with G = grad grad_scale and a momentum M (fp32),
 *     M = momentum M + G;  U = G + momentum M if nesterov, else M
 *     param = param (1 - lr weight_decay) - lr scale orthogonalize(U)
 * where bf16 parameters take orthogonalize's products for bf16. The momenta lie
 * in one float array m, matrix i's (in row order, without gaps) from
 * moment_offset on, a multiple of 256; zeros before the first step. The plan,
 * device memory of w2v_muon_plan_bytes bytes that the caller keeps, is made
 * once from a list (synchronises the stream), and a step is given the same list
 * again. Matrices of the same sizes and types go through the products together.
 * A plan, and a workspace, belong to one step at a time. Errors: W2V_E_ARG for
 * sizes, strides, types or NULL pointers out of range, momenta that overlap or
 * reach past n_moments (a matrix's last 256 count whole), or packed parameters
 * that overlap; W2V_E_WORKSPACE; W2V_E_RANGE. */
typedef struct {
    void *param;              /* rows x cols elements of param_type */
    const void *grad;         /* rows x cols elements of grad_type */
    int64_t rows, cols;       /* 0..2^20 */
    int64_t param_stride, grad_stride;
    int64_t moment_offset;
    int32_t param_type, grad_type;
    float weight_decay, scale;
} w2v_muon_matrix;

typedef struct {
    double lr, momentum, eps;
    const float *lr_device;   /* NULL, or the learning rate in device memory (instead of lr) */
    float grad_scale;
    int32_t nesterov, steps;  /* steps 1..20 */
    int32_t reserved0;
} w2v_muon_params;

size_t w2v_muon_plan_bytes(const w2v_muon_matrix *matrices_host, int32_t n);
size_t w2v_muon_workspace_bytes(const w2v_muon_matrix *matrices_host, int32_t n);
int w2v_muon_build_plan(const w2v_muon_matrix *matrices_host, int32_t n, int64_t n_moments, void *plan, size_t plan_bytes,
                        void *hip_stream);
int w2v_muon_step(const w2v_muon_matrix *matrices_host, int32_t n, const void *plan, float *m, const w2v_muon_params *p,
                  void *workspace, size_t workspace_bytes, void *hip_stream);

/* ------------------------------------------------------------------------
 * Training in mini-batches with the operators above: CBOW whose hidden vector
 * is the mean of the window's vectors, through a layer norm if gain and bias
 * are given, scored against the centre word by the hierarchical softmax.
 * Sampling, windows and the learning-rate schedule are w2v_train_hs_epoch's
 * (p->arch 1); of p's other settings only sync_batch is used. Every
 * sync_batch (1..2^20) consecutive kept centres make a batch; all gradients
 * of its mean loss (the sum over the centres that have a window, divided by
 * the batch's centres) are taken against the model at its start; then AdamW,
 * with the learning rate of its first centre, updates syn0 and syn1 (decay
 * weight_decay) and gain and bias (no decay): every row, whether or not the
 * batch reached it. Deterministic. A centre without a window has no part in
 * any gradient. With norm_eps 0 a window whose mean has equal columns has no
 * finite deviation and makes the model NaN.
 *   m, v, m_scale, v_scale  moments as in w2v_adamw_step, of
 *                    w2v_batch_n_moments elements: syn0 (V x dim), syn1
 *                    (V-1 x dim), gain, bias, each from the next multiple of
 *                    256 on
 *   step0            steps taken before this call
 * stats int64[W2V_N_STATS] may be NULL. steps_host: batches of this call, after
 * an error those whose update was launched before it.
 * sum_ll_host, n_terms_host (may be NULL): sum of log P(centre | hidden) over
 * the centres with a window, each scored before its batch's update, and their
 * number. Synchronises the stream. Errors: as w2v_train_hs_epoch, and
 * W2V_E_ARG for an arch other than 1, settings out of range or a NULL moment.
 *
 * w2v_batch_loglik: the same score without any update (the held-out
 * objective; of bp gain, bias, norm_eps and max_code_len are used).
 * ---------------------------------------------------------------------- */
typedef struct {
    float *gain, *bias;       /* float[dim] of the layer norm, both or neither */
    void *m, *v;
    float *m_scale, *v_scale; /* bits 8 only */
    double beta1, beta2, eps;
    int64_t step0;
    float norm_eps, weight_decay;
    int32_t bits;             /* of the moments: 32 or 8 */
    int32_t max_code_len;     /* from w2v_build_huffman, 1..64 */
    uint32_t seed;            /* of the 8-bit moments' rounding */
    int32_t reserved0;
} w2v_batch_params;

int64_t w2v_batch_n_moments(const w2v_model *m, const w2v_batch_params *bp);
size_t w2v_train_batch_workspace_bytes(const w2v_model *m, int64_t n_tokens, const w2v_params *p,
                                       const w2v_batch_params *bp);
int w2v_train_batch_epoch(const w2v_model *m, const int32_t *tokens, int64_t n_tokens, const w2v_params *p,
                          const w2v_batch_params *bp, int64_t *stats, int64_t *steps_host, double *sum_ll_host,
                          int64_t *n_terms_host, void *workspace, size_t workspace_bytes, void *hip_stream);
size_t w2v_batch_loglik_workspace_bytes(const w2v_model *m, int64_t n_tokens, const w2v_params *p,
                                        const w2v_batch_params *bp);
int w2v_batch_loglik(const w2v_model *m, const int32_t *tokens, int64_t n_tokens, const w2v_params *p,
                     const w2v_batch_params *bp, double *sum_ll_host, int64_t *n_terms_host, void *workspace,
                     size_t workspace_bytes, void *hip_stream);

/* ------------------------------------------------------------------------
 * Test hooks (not part of the training contract).
 *
 * w2v_sample_pairs: the (centre, context) pairs of the sampler in stream
 * order (documents, then centres, then window positions ascending), as global
 * raw indices; the first pair_cap are written (centre_raw/context_raw may be
 * NULL); keep_mask uint8[n_tokens] (may be NULL) marks kept centres;
 * checksum_host = sum over all pairs of fmix64(centre * 0x9E3779B97F4A7C15 +
 * context) mod 2^64 (MurmurHash3 finaliser). Synchronises the stream.
 *
 * w2v_keep_thresholds: thr[v] = 2^32 if the keep probability is >= 1, else
 * floor(p_keep 2^32); a token is kept iff its first Philox word < thr.
 *
 * w2v_sample_negatives: the p->negative negatives of every kept centre in
 * stream order (-1 where dropped), the first negatives_cap centres written to
 * negatives int32[cap][negative] (may be NULL); checksum_host = sum over kept
 * centres and k of fmix64(raw * 0x9E3779B97F4A7C15 + k * 2^32 + (negative + 1))
 * mod 2^64. Synchronises the stream.
 * ---------------------------------------------------------------------- */
size_t w2v_sample_pairs_workspace_bytes(int32_t V, int64_t n_tokens, const w2v_params *p);
int w2v_sample_pairs(const int32_t *tokens, int64_t n_tokens, int32_t V, const int64_t *vocab_counts,
                     int64_t train_words, const w2v_params *p, int64_t *centre_raw, int64_t *context_raw,
                     int64_t pair_cap, uint8_t *keep_mask, int64_t *n_pairs_host, int64_t *n_kept_host,
                     uint64_t *checksum_host, void *workspace, size_t workspace_bytes, void *hip_stream);
int w2v_keep_thresholds(const int64_t *vocab_counts, int32_t V, double sample, int64_t train_words, uint64_t *thr,
                        void *hip_stream);
size_t w2v_sample_negatives_workspace_bytes(int32_t V, int64_t n_tokens, const w2v_params *p);
int w2v_sample_negatives(const int32_t *tokens, int64_t n_tokens, int32_t V, const int64_t *vocab_counts,
                         int64_t train_words, const w2v_params *p, const int32_t *noise_table, int32_t log2_size,
                         int32_t *negatives, int64_t negatives_cap, int64_t *n_kept_host, uint64_t *checksum_host,
                         void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* W2V_H */
