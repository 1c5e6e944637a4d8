/*
 * libw2v: HogBatch skip-gram negative-sampling SGD on MI355X (gfx950).
 *
 * Implements the shared-memory hot path of Ji, Satish, Li and Dubey,
 * "Parallelizing Word2Vec in Multi-Core and Many-Core Architectures"
 * (arXiv 1611.06172): for every target word, one minibatch of N input
 * (context) words and K negatives shared by those N words (Sec. 1.1, negative
 * sample sharing), whose dot products form an N x (K+1) block computed as one
 * small matrix product; the sigmoid error of Alg. 1 and both gradient
 * products follow, and the model updates are written back Hogwild-style (no
 * locks, conflicts between concurrent minibatches tolerated; Sec. 1.1,
 * "HogBatch").
 *
 * Conventions for every entry point:
 *   - M_in and M_out are V x D fp32 matrices, row-major, row stride ld >= D
 *     (floats). Word w is row w (Alg. 1: M_in holds input-word vectors, M_out
 *     output-word vectors). Columns D..ld-1 are never read or written.
 *   - "device" pointers are GPU global memory of the current HIP device;
 *     "host" pointers are ordinary CPU memory. The caller owns every buffer;
 *     the library keeps no pointer after a call returns and allocates no
 *     device memory.
 *   - GPU entry points are asynchronous on `stream` (a hipStream_t; NULL is
 *     the null stream). Results are visible once the caller synchronises it.
 *   - Return value: W2V_OK (0) or a negative W2V_E* code; w2v_last_error()
 *     then describes the failure. Arguments are validated on the host before
 *     any HIP call; a call that fails validation launches nothing.
 *   - Ids read from device memory (corpus, tables, batches) are always checked
 *     on the device: a minibatch that would touch a row outside [0, V) is
 *     skipped (no memory outside the given buffers is ever accessed), counted
 *     in the optional stats output, and recorded in the device's error word.
 *     The first GPU call on that device that starts after the skipping kernel
 *     has finished returns W2V_EDEVICE_FLAG, clears the word and launches
 *     nothing; w2v_device_status waits for a stream and reports the same.
 *     In the corpus, -1 marks a word removed from the vocabulary
 *     (w2v_build_vocab) and is no error: the position is dropped before
 *     windows form.
 *
 * Readings of points the paper leaves open (sentence cut, window shrink,
 * subsampling rule, negative distribution, learning-rate decay, random
 * numbers) are stated beside each entry point.
 */
#ifndef W2V_H
#define W2V_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define W2V_OK 0
#define W2V_EINVAL (-1)      /* an argument is out of range or NULL */
#define W2V_EHIP (-2)        /* the HIP runtime reported an error */
#define W2V_ENOMEM (-3)      /* a host allocation failed */
#define W2V_EUNSUPPORTED (-4)/* valid arguments outside the compiled shapes */
#define W2V_EDEVICE_FLAG (-5)/* an earlier call skipped work for an id outside
                                [0, V), or rows of scores for an id, a label or
                                a setting out of range, or rows for a word or a
                                parent out of range; nothing was launched by
                                this call */
#define W2V_ENONFINITE (-6)  /* a loss bucket holds NaN or Inf (w2v_check_loss) */

/* Shape limits of the compiled kernels. The HogBatch kernels keep all N
 * input rows of a minibatch in registers, so they compile D <= 640 for up to
 * 10 input words (window <= 5), D <= 320 for up to 16 (window <= 8) and
 * D <= 128 for up to 32 (window <= 16); other valid combinations return
 * W2V_EUNSUPPORTED. Algorithm 1 compiles D <= 640 at every window. */
#define W2V_MAX_DIM 640          /* D */
#define W2V_MAX_WINDOW 16        /* window: up to 2*window input words */
#define W2V_MAX_NEGATIVE 64      /* K */
#define W2V_MAX_SENTENCE 1024    /* sentence_len */
#define W2V_MAX_BATCH_INPUTS 32  /* N of w2v_step_batch */

/* Partial rows per split row of w2v_train_epoch (one per XCD of MI355X). */
#define W2V_SPLIT_PARTS 8

/* Bytes of the library's static device scratch array, the partial rows of
 * w2v_train_epoch_noalloc (one copy per device, held until the process
 * ends): 2 * split_rows * W2V_SPLIT_PARTS * ld * 4 bytes must fit, e.g.
 * 204 split rows at ld = 320. */
#define W2V_NOALLOC_SCRATCH_BYTES 4194304

/* The `algorithm` argument of w2v_train_epoch. */
#define W2V_ALGORITHM_HOGBATCH 0  /* Sec. 1.1: minibatch, shared negatives */
#define W2V_ALGORITHM_PAIRWISE 1  /* Alg. 1: per-pair SGD, private negatives */
#define W2V_ALGORITHM_HOGBATCH_IMMEDIATE 2 /* Sec. 1.1, no pending input rows */

/* Version of this ABI (major * 100 + minor). */
int w2v_version(void);

/* Message of the last failed call on this thread ("" if none). The pointer
 * stays valid until the next call on the same thread. */
const char* w2v_last_error(void);

/* Sets up the library's per-device state on the current HIP device: the
 * device's error word (pinned host memory mapped into the device, 256 bytes,
 * held until the process ends) and the device address of the library's
 * static scratch array. Every GPU entry point does this itself on its first
 * call on a device, except w2v_train_epoch_noalloc, which allocates nothing
 * and so needs w2v_init to have run on the device first. Safe to call
 * repeatedly and from several threads. */
int w2v_init(void);

/* Waits for `stream` (a hipStream_t; NULL is the null stream), then returns
 * W2V_EDEVICE_FLAG (and clears the error word) if a kernel of this library on
 * the current device skipped a minibatch for an id outside [0, V), or a row of
 * scores for an id, a label or a setting out of range, since the word was last
 * reported, else W2V_OK. */
int w2v_device_status(void* stream);

/* Failure detection for training (not in the paper, which reports no loss):
 * waits for `stream`, reads the n_buckets (sum, count) pairs of
 * loss_buckets (device double[n_buckets][2], as w2v_train_epoch fills them)
 * and returns W2V_ENONFINITE, naming the first such bucket, if a sum or a
 * count is NaN or Inf; W2V_OK otherwise. A NaN or Inf that reaches a row of
 * M_in or M_out makes the loss of every later minibatch reading the row
 * non-finite, so its bucket flags it. Launches nothing; copies 16 n_buckets
 * bytes to the host. W2V_EINVAL for n_buckets < 0 or a NULL pointer with
 * n_buckets > 0. */
int w2v_check_loss(const double* loss_buckets, int32_t n_buckets, void* stream);

/*
 * Sampling tables from unigram counts (host only; no HIP call).
 * Paper: Sec. 2 trains with 5 negative samples and sample = 1e-4; Alg. 1
 * draws each negative "from V". Readings:
 *   neg_table (host out, int32[table_size], may be NULL): word w owns slots
 *     [bound(w-1), bound(w)), bound(-1) = 0, bound(V-1) = table_size and
 *     bound(w) = floor(S_w / S_{V-1} * table_size) with
 *     S_w = sum_{v <= w} counts[v]^neg_power, summed left to right in fp64
 *     (neg_power = 0.75 gives the unigram^0.75 distribution).
 *   keep_thresh (host out, uint32[V], may be NULL): with f = counts[w] /
 *     sum(counts) and p = sqrt(t/f) + t/f, a position holding w is kept iff
 *     its 32-bit draw r <= keep_thresh[w]; keep_thresh[w] = 0xFFFFFFFF when
 *     t == 0, counts[w] == 0 or p >= 1, else max(floor(p * 2^32) - 1, 0).
 * counts: host int64[V], all >= 0 with a positive sum. table_size in
 * [1, 2^32). sample_t >= 0.
 */
int w2v_build_tables(const int64_t* counts, int32_t V, double neg_power,
                     double sample_t, int32_t* neg_table, int64_t table_size,
                     uint32_t* keep_thresh);

/*
 * Update-path choice for w2v_train_epoch (host only; no HIP call): the
 * number H of leading ids that should receive atomic updates. With the
 * sampling of w2v_build_tables, one minibatch writes the M_out row of word w
 * with probability about p_out(w) = rho_w + K q_w (rho: share of w among
 * kept words, q: its negative-sampling share) and the M_in row with
 * probability about p_in(w) = (window + 1) rho_w. With `inflight` minibatches
 * in flight, (inflight - 1) max(p_in, p_out) is the expected number of other
 * minibatches writing the row while one holds it. H is one more than the
 * largest id whose expected count reaches `tol` (0 if none), so every row at
 * or above H is rarely written concurrently. counts as for w2v_build_tables;
 * ids are expected to be ranked by frequency. Returns H >= 0, or a negative
 * W2V_E* code.
 */
int32_t w2v_hot_rows(const int64_t* counts, int32_t V, double neg_power,
                     double sample_t, int32_t window, int32_t K,
                     int64_t inflight, double tol);

/* Number of sentences w2v_train_epoch processes concurrently when called with
 * max_inflight = 0 on the current device (one wavefront each), or a negative
 * W2V_E* code: the wavefronts the device holds at once for this shape,
 * capped at max(1, floor(V / (4 group (2 window + K + 1)))). The cap keeps
 * the rows that the concurrent minibatches hold (up to 2 window input rows
 * and K + 1 output rows each, group times that for a group) under a quarter
 * of the vocabulary, so that a small vocabulary is not trained mostly from
 * stale rows; Hogwild staleness is what separates the concurrent epoch from
 * the sequential one (Sec. 1.1). At V = 10^6, window 5, K = 5 the cap
 * (15,625) is above what the GPU holds. A second cap, 131072 / (K + 1)
 * (2016 at K = 64), bounds how many concurrent sentences update the rows of
 * the words most often drawn as negatives, each from the row as it was
 * before the others' updates: at K = 64, D = 100 and alpha 0.025 the epoch
 * over a Zipf(1.07) vocabulary of 10^6 words learned with up to 2048
 * sentences in flight and diverged (NaN) with 2560. */
int64_t w2v_default_inflight(int32_t V, int32_t D, int32_t window, int32_t K,
                             int32_t group);

/* LDS slots per wavefront in which w2v_train_epoch (W2V_ALGORITHM_HOGBATCH,
 * group 1) collects pending input-row updates for this shape on the current
 * device (0: none), or a negative W2V_E* code. */
int32_t w2v_pending_slots(int32_t D, int32_t window, int32_t K);

/*
 * One Hogwild epoch (or a sentence-aligned part of one) of HogBatch SGD,
 * updating M_in and M_out in place on the GPU.
 *
 * Minibatch formation (readings; every random decision is a pure function of
 * (seed, raw position p, epoch) through Philox4x64-10, Salmon et al. SC'11,
 * with counter (p, epoch, j, 0) and key (seed, 0); block j's four 64-bit
 * outputs give 32-bit words 8j..8j+7, low half first):
 *   - the corpus is cut into sentences of sentence_len raw tokens (the last
 *     may be shorter); windows never cross a sentence;
 *   - position p is kept iff keep_thresh == NULL or word 0 <= keep_thresh[x_p];
 *   - each kept word (retained index q in its sentence) is a target; with
 *     b = floor(word1 * window / 2^32) and h = window - b its input words are
 *     the kept words at retained indices q-h..q+h except q; a target with no
 *     input word forms no minibatch;
 *   - negative k (k < K) is neg_table[floor(word(2+k) * table_size / 2^32)];
 *     a negative equal to the target is masked (contributes nothing);
 *   - alpha = fp32(alpha0 * max(min_alpha_frac, 1 - (epoch*T + p) /
 *     (n_epochs*T))), evaluated in IEEE fp64.
 * Minibatch step (Sec. 1.1, Alg. 1 error and update directions): with A the
 * input-word rows of M_in and O = [target row; negative rows] of M_out,
 *   X = A O^T, E = alpha * (l - sigma(X)), l = (1, 0, ..., 0),
 *   M_in[input words] += E O, M_out[target, negatives] += E^T A,
 * all from the rows as read at the start of the minibatch (repeated words
 * of one minibatch are merged, so each row is read and written once per
 * minibatch). Minibatches of one sentence run in order on one wavefront; up
 * to max_inflight sentences run concurrently and their updates interleave
 * without locks (Hogwild). max_inflight = 1 processes every minibatch in
 * sequence; 0 picks min(w2v_default_inflight(V, D, window, K, group),
 * ceil(S / 8)) for the S sentences of the range, so that they run in at
 * least 8 rounds (with every sentence of a short range in flight at once,
 * each would start from the initial model).
 * Pending input rows (W2V_ALGORITHM_HOGBATCH with group 1): consecutive
 * targets share most input words, so a wavefront adds the updates of a cold
 * input row (id >= max(hot_rows, split_rows)) to one of
 * w2v_pending_slots() LDS slots instead of M_in, reads the row as (M_in row
 * + pending updates) while its word is in the window, and adds the slot to
 * M_in atomically when it releases the word: when the slot is needed for
 * another word, when 2 * window targets have passed without the word and the
 * next one does not hold it either, and at the end of the sentence. Every
 * update reaches M_in before the call returns.
 * With one sentence in flight this changes only the order of the fp32
 * additions; with several, another sentence sees these updates late (as
 * late as the word stays in this sentence's window) and never loses them.
 * Rows below max(hot_rows, split_rows), which other sentences write
 * constantly, take their updates at once: deferring those lets the
 * concurrent sentences' stale steps pile up on them.
 * W2V_ALGORITHM_HOGBATCH_IMMEDIATE applies every update at the end of its
 * minibatch.
 * algorithm = W2V_ALGORITHM_PAIRWISE runs Alg. 1 instead (the original
 * per-pair Hogwild SGD, the paper's baseline) over the same targets, input
 * words and learning rates: each input word i in window order runs K+1
 * logistic regressions against the target and K negatives of its own
 * (draws 2 + iK + k of the target's stream; a draw equal to the target is
 * skipped); each pair reads the M_out row as moved by the pairs before it,
 * that row moves right after its pair, and the M_in row of i moves once,
 * after its K+1 pairs. A target with any negative outside [0, V) is skipped
 * and counted in stats[3]. split_rows must be 0 with this algorithm.
 * group (HogBatch algorithms; 1 is the paper's method): G in {2, 4, 8} shares the
 * K negatives among G consecutive targets instead of one target's input
 * words (the sharing of Sec. 1.1 widened). The retained targets of a
 * sentence are cut at multiples of G; the members of a group (its targets
 * with input words) take the negatives drawn at the group's first retained
 * position (draws 2..K+1 of its stream); a negative equal to a member's own
 * target is masked for that member; all members' steps read the rows as
 * they were before the group and their updates to a row are summed; a
 * group's loss goes to the bucket of its first member. Needs 2 window G <=
 * 64, 2 window + G <= 32 and G + K <= 32; G + K output columns are compiled
 * up to 16 for D <= 384 and 10 for D <= 640, up to 32 for D <= 128.
 * Update path: a row with id < hot_rows receives fp32 atomic adds (no update
 * is lost under concurrency); a row with id >= hot_rows is written back as
 * (value read + update) by a store written through to device scope, so a
 * concurrent update of the same row by another sentence may be
 * overwritten, as in Hogwild. With ids
 * ranked by frequency (id 0 the most frequent word) hot_rows selects the
 * frequent words, whose rows see concurrent updates; hot_rows >= V makes
 * every update atomic.
 * Split rows: atomics are performed at the memory side and those to one
 * address queue behind each other, so the few rows that nearly every
 * concurrent sentence writes (the head of the Zipf law) would stall the
 * whole memory system. A row with id < split_rows (regardless of hot_rows)
 * is therefore spread over W2V_SPLIT_PARTS partial rows in `workspace`:
 * each sentence adds its updates atomically to the partial row of its
 * wavefront's group, every read of the row returns the matrix row plus all
 * of its partial rows (so no update is hidden from any reader, as with a
 * single atomic row), and after the epoch the partial rows are added into
 * M_in/M_out and cleared. split_rows = 0 disables this; workspace may then
 * be NULL.
 *
 * corpus: device int32[T]. [pos_begin, pos_end) must start on a sentence
 * boundary and end on one or at T. M_in, M_out: device, see conventions.
 * neg_table: device int32[table_size]. keep_thresh: device uint32[V] or NULL.
 * loss_buckets: device double[2 * n_buckets] or NULL; for a minibatch of
 * target position p, bucket b = floor(p * n_buckets / T) receives
 * [2b] += sum_i [-log sigma(X_i0) - sum_{k unmasked} log sigma(-X_ik)] and
 * [2b+1] += N. workspace: device memory of at least
 * w2v_train_epoch_workspace_bytes(split_rows, ld) bytes, 256-byte aligned,
 * caller-owned, its
 * contents need not be initialised (the call clears what it uses), and it
 * must not be shared by calls that overlap in time. stats: device int64[5]
 * or NULL, accumulated into:
 * [0] minibatches applied, [1] sum of N over them, [2] raw positions
 * visited, [3] minibatches skipped for an id outside [0, V) (for the corpus:
 * positions holding such an id, -1 excepted), [4] rows read and written
 * back: per minibatch its distinct input and output rows, per group of
 * targets (group > 1) the distinct rows of the group, per input word of
 * Alg. 1 its row and K + 1 output rows.
 * Limits: 1 <= D <= W2V_MAX_DIM, 1 <= window <= W2V_MAX_WINDOW,
 * 0 <= K <= W2V_MAX_NEGATIVE, 1 <= sentence_len <= W2V_MAX_SENTENCE.
 */
int w2v_train_epoch(const int32_t* corpus, int64_t T, int64_t pos_begin,
                    int64_t pos_end, int32_t sentence_len, float* M_in,
                    float* M_out, int32_t V, int32_t D, int32_t ld,
                    int32_t window, int32_t K, const int32_t* neg_table,
                    int64_t table_size, const uint32_t* keep_thresh,
                    float alpha0, float min_alpha_frac, int32_t epoch,
                    int32_t n_epochs, uint64_t seed, double* loss_buckets,
                    int32_t n_buckets, int64_t* stats, int32_t max_inflight,
                    int32_t hot_rows, int32_t split_rows, void* workspace,
                    size_t workspace_bytes, int32_t algorithm, int32_t group,
                    void* stream);

/*
 * w2v_train_epoch for callers that cannot allocate (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): the same
 * arguments, readings, limits and results, minus the workspace. The split
 * rows' partial rows live in the library's static device scratch array
 * (W2V_NOALLOC_SCRATCH_BYTES per device), so split_rows must satisfy
 * 2 * split_rows * W2V_SPLIT_PARTS * ld * 4 <= W2V_NOALLOC_SCRATCH_BYTES,
 * else W2V_EINVAL (nothing launched). The call allocates no device or
 * pinned memory and calls no hipMalloc or hipFree; w2v_init must have run
 * on the current device (else W2V_EINVAL). It clears the partial rows it
 * uses before the epoch (with a kernel, no memset) and after it. All calls
 * on one device share the one scratch array: calls that overlap in time on
 * the same device (other streams, other threads) race on it and must not
 * be issued. (A shape's launch configuration is computed on its first call
 * and cached in host memory.)
 */
int w2v_train_epoch_noalloc(const int32_t* corpus, int64_t T, int64_t pos_begin,
                            int64_t pos_end, int32_t sentence_len, float* M_in,
                            float* M_out, int32_t V, int32_t D, int32_t ld,
                            int32_t window, int32_t K, const int32_t* neg_table,
                            int64_t table_size, const uint32_t* keep_thresh,
                            float alpha0, float min_alpha_frac, int32_t epoch,
                            int32_t n_epochs, uint64_t seed, double* loss_buckets,
                            int32_t n_buckets, int64_t* stats, int32_t max_inflight,
                            int32_t hot_rows, int32_t split_rows, int32_t algorithm,
                            int32_t group, void* stream);

/* Workspace bytes w2v_train_epoch needs for split_rows rows of stride ld:
 * 2 * split_rows * W2V_SPLIT_PARTS * ld * 4 (0 when split_rows is 0). */
size_t w2v_train_epoch_workspace_bytes(int32_t split_rows, int32_t ld);

/*
 * Vocabulary of a raw id stream (GPU; the step before w2v_build_tables: the
 * paper's corpus is counted and its words ranked, Sec. 2). Counts every id
 * of raw[0..T) in [0, V_raw) (other values are not counted), ranks the ids
 * by count, descending, ties by increasing raw id, and keeps the words with
 * count >= max(min_count, 1).
 *   ranked_counts device int64[V_raw]: count of the word of rank r for
 *                 r < V, 0 after (the counts argument of w2v_build_tables);
 *   rank_of       device int32[V_raw]: the new id of raw id x (its rank), or
 *                 -1 when x is dropped;
 *   v_kept        device int32[1]: V, the number of words kept;
 *   corpus_out    device int32[T] or NULL: raw rewritten in new ids, -1 for
 *                 dropped words and ids outside [0, V_raw) (the epoch skips
 *                 such positions before forming windows).
 * With ids ranked this way id 0 is the most frequent word, as the update
 * tiers of w2v_train_epoch assume. workspace: device, 256-byte aligned,
 * >= w2v_build_vocab_workspace_bytes(V_raw, T) bytes, caller-owned; up to
 * V_raw = 4,194,304 the ids are counted by id range without atomics to
 * device memory, which takes about 4.3 T bytes of it (the stream reordered
 * by id range, and partial counts). The call is asynchronous on `stream`.
 */
size_t w2v_build_vocab_workspace_bytes(int32_t V_raw, int64_t T);
int w2v_build_vocab(const int32_t* raw, int64_t T, int32_t V_raw,
                    int64_t min_count, int64_t* ranked_counts,
                    int32_t* rank_of, int32_t* v_kept, int32_t* corpus_out,
                    void* workspace, size_t workspace_bytes, void* stream);

/*
 * The minibatches w2v_train_epoch would form over [pos_begin, pos_end),
 * written out instead of applied (same arguments and readings as
 * w2v_train_epoch; the matrices are not needed): for every target word its
 * N input words and the K negatives they share (Sec. 1.1, negative sample
 * sharing; Alg. 1's problem statement: a target word, N input words, K
 * negatives drawn from V), with the sentence, window, subsampling, table and
 * learning-rate readings stated for w2v_train_epoch. This is the sampling
 * half of the epoch, exported so that it can be compared bit for bit with an
 * independent implementation. Outputs are indexed by raw
 * position r = p - pos_begin, P = pos_end - pos_begin:
 *   out_targets  device int32[P]: the target word, or -1 where position p
 *                forms no minibatch (not kept, or no input word);
 *   out_ctx      device int32[P][2*window]: input words in order, -1 padded;
 *   out_negs     device int32[P][K]; out_mask device uint8[P][K];
 *   out_alpha    device float[P].
 * Entries of out_ctx/out_negs/out_mask/out_alpha are written only where
 * out_targets != -1. stats as in w2v_train_epoch (may be NULL).
 */
int w2v_debug_minibatches(const int32_t* corpus, int64_t T, int64_t pos_begin,
                          int64_t pos_end, int32_t sentence_len, int32_t V,
                          int32_t window, int32_t K, const int32_t* neg_table,
                          int64_t table_size, const uint32_t* keep_thresh,
                          float alpha0, float min_alpha_frac, int32_t epoch,
                          int32_t n_epochs, uint64_t seed, int32_t* out_targets,
                          int32_t* out_ctx, int32_t* out_negs,
                          uint8_t* out_mask, float* out_alpha, int64_t* stats,
                          void* stream);

/* Bytes of workspace w2v_step_batch needs: the size of two fp64 V x ld
 * buffers, each rounded up to 256 bytes. */
size_t w2v_step_batch_workspace_bytes(int32_t V, int32_t ld);

/*
 * One deterministic batch of B independent HogBatch minibatches against given
 * matrices. Each minibatch is the step of Sec. 1.1 for one target word, its
 * N input words and K shared negatives (Alg. 1's problem statement:
 * given M_in, M_out, alpha, a target word and N input words): X = A O^T,
 * E = alpha (l - sigma(X)), M_in[inputs] += E O, M_out[target, negatives]
 * += E^T A. Every gradient is computed from the matrices as they were on
 * entry: the paper computes a minibatch's products from the rows as read and
 * writes the updates back when its matrix product is done (Sec. 1.1); here
 * the whole batch shares that snapshot, so the result does not depend on the
 * order of the minibatches (a deterministic counterpart of the Hogwild
 * epoch, not a step the paper runs as such). The per-minibatch updates are
 * summed per element in fp64 and each touched element becomes fp32(M + sum),
 * one rounding per element. Elements whose summed update is exactly 0 keep
 * their bits. How the sums are formed follows from the sizes: with fp64
 * atomics into delta buffers (in arrival order, so the last fp32 bit of an
 * element may differ from run to run), from staging rows, or from the
 * minibatches' errors; only w2v_step_batch_sorted promises the same bits on
 * every run. M_in and M_out may share elements (one matrix passed as both,
 * overlapping views): a shared element receives both updates, rounded one
 * after the other.
 * targets: device int32[B]; contexts: device int32[B][N], -1 = absent;
 * negatives: device int32[B][K]; a negative equal to its target is masked.
 * alpha: device float[B], or NULL to use alpha_scalar for every minibatch.
 * workspace: device, >= w2v_step_batch_workspace_bytes(V, ld) bytes, 256-byte
 * aligned, caller-owned scratch of no stated layout: its contents need not be
 * initialised, and calls that overlap in time must not share it. stats:
 * device int64[5] or NULL, as in w2v_train_epoch ([2] is not used).
 * Limits: 0 <= N <= W2V_MAX_BATCH_INPUTS, 0 <= K <= W2V_MAX_NEGATIVE,
 * 1 <= D <= W2V_MAX_DIM.
 */
int w2v_step_batch(int32_t B, int32_t N, int32_t K, const int32_t* targets,
                   const int32_t* contexts, const int32_t* negatives,
                   const float* alpha, float alpha_scalar, float* M_in,
                   float* M_out, int32_t V, int32_t D, int32_t ld,
                   void* workspace, size_t workspace_bytes, int64_t* stats,
                   void* stream);

/* The route that w2v_step_batch takes for these arguments, for tests of each
 * route (host only; the matrices are not read). A negative W2V_E* code on
 * invalid arguments. Matrices that share elements (one matrix passed as both,
 * overlapping views) take the atomic route. */
#define W2V_STEP_ROUTE_ATOMIC 0
#define W2V_STEP_ROUTE_STAGED 1
#define W2V_STEP_ROUTE_PULLED 2
int32_t w2v_debug_step_route(int32_t B, int32_t N, int32_t K, const float* M_in,
                             const float* M_out, int32_t V, int32_t D, int32_t ld);

/* Bytes of workspace w2v_step_batch_sorted needs for B minibatches of N
 * input slots and K negatives over V rows of stride ld (0 on invalid
 * arguments or a failed query): staging rows for every update, sort keys
 * and values, per-chunk partial sums and the sort's temporaries. */
size_t w2v_step_batch_sorted_workspace_bytes(int32_t B, int32_t N, int32_t K,
                                             int32_t V, int32_t ld);

/*
 * The step of w2v_step_batch (same arguments, readings and limits) with
 * every row's updates summed in one fixed order: each minibatch's updates
 * are written to staging rows, sorted by row id with a stable radix sort
 * (so a row's updates stay in minibatch order) and summed per row in fp64
 * in that order, in chunks of 64 whose partial sums are added in chunk
 * order (grouped 32 chunks at a time). The result is the same bits on every
 * run, and no atomics are used. w2v_step_batch gives the same bits where it
 * takes no atomics either, and may differ in the last fp32 bit of an element
 * where it does.
 * Additional limits: B (N + K + 1) must fit in int32, and M_in and M_out must
 * not share elements. workspace: device,
 * >= w2v_step_batch_sorted_workspace_bytes(B, N, K, V, ld) bytes, 256-byte
 * aligned, caller-owned, contents need not be initialised; calls that
 * overlap in time must not share it.
 */
int w2v_step_batch_sorted(int32_t B, int32_t N, int32_t K, const int32_t* targets,
                          const int32_t* contexts, const int32_t* negatives,
                          const float* alpha, float alpha_scalar, float* M_in,
                          float* M_out, int32_t V, int32_t D, int32_t ld,
                          void* workspace, size_t workspace_bytes, int64_t* stats,
                          void* stream);

/*
 * The vocabulary head: what a trained model answers with. Scores of contexts
 * against the rows of M_out are a matrix product; a smaller model learns
 * another one's distribution from its top scores; words are drawn from
 * scores. (Not in the paper, which ends with the trained vectors.)
 *
 * Matrices are row-major with unit column stride and a row stride in
 * elements, at least the number of columns, of any alignment that one element
 * has; row offsets are 64-bit. Element types:
 */
#define W2V_DTYPE_F32 0
#define W2V_DTYPE_BF16 1
#define W2V_DTYPE_F16 2

/* The `activation` argument of w2v_linear. */
#define W2V_ACTIVATION_NONE 0
#define W2V_ACTIVATION_RELU 1
#define W2V_ACTIVATION_GELU 2 /* z Phi(z), with the error function */
#define W2V_ACTIVATION_SILU 3 /* z sigma(z) */
#define W2V_ACTIVATION_TANH 4
#define W2V_ACTIVATION_SIGMOID 5

/*
 * y = act(x W^T + b) + residual, for x M x K, W N x K (a row per output, as
 * M_out holds a row per word) and y M x N.
 *   dtype         type of x, W and pre (W2V_DTYPE_*);
 *   out_dtype     type of y and residual: dtype or W2V_DTYPE_F32;
 *   bias          device float[N] or NULL;
 *   residual      device M x N or NULL; may be y itself (same stride);
 *   pre           device M x N or NULL: receives z = x W^T + b, which
 *                 w2v_linear_backward needs where there is an activation.
 * Sums and the epilogue are held in fp32 and each output is rounded once. The
 * order of a sum depends on the sizes alone: the same call gives the same
 * bits. workspace: device, 256-byte aligned, at least
 * w2v_linear_workspace_bytes(M, N, K, dtype) bytes (partial sums where a long k
 * is split; in 16 bits, for large outputs, copies of x and W with rows on
 * 64-byte lines, made if theirs are not; otherwise 0), contents need not be initialised; calls that overlap in time must
 * not share it. M = 0 is allowed and does nothing; N, K >= 1. y and pre must
 * not overlap any other argument (residual = y excepted).
 */
size_t w2v_linear_workspace_bytes(int32_t M, int32_t N, int32_t K, int32_t dtype);
int w2v_linear(const void* x, int64_t ldx, const void* w, int64_t ldw, const float* bias,
               const void* residual, int64_t ldr, void* y, int64_t ldy, void* pre,
               int64_t ldp, int32_t M, int32_t N, int32_t K, int32_t dtype,
               int32_t out_dtype, int32_t activation, void* workspace,
               size_t workspace_bytes, void* stream);

/*
 * Gradients of w2v_linear from dy (M x N):
 *   dz = dy * act'(pre), dx = dz W (M x K), dW = dz^T x (N x K),
 *   db = sum over the rows of dz (device float[N]);
 * the residual's gradient is dy itself. dx, dw and db may each be NULL (not
 * wanted). pre: z as w2v_linear wrote it, needed unless the activation is
 * W2V_ACTIVATION_NONE; relu's derivative at 0 is 0. All matrices are of
 * `dtype`. With an activation, dz is rounded once to `dtype` for dx and dW; db
 * sums it before that rounding. Sums are held in
 * fp32, in an order that depends on the sizes alone. M = 0 gives dW = 0 and
 * db = 0. workspace: as above, w2v_linear_backward_workspace_bytes bytes.
 * Outputs must not overlap any other argument.
 */
size_t w2v_linear_backward_workspace_bytes(int32_t M, int32_t N, int32_t K, int32_t dtype,
                                           int32_t activation);
int w2v_linear_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx,
                        const void* w, int64_t ldw, const void* pre, int64_t ldp, void* dx,
                        int64_t lddx, void* dw, int64_t lddw, float* db, int32_t M, int32_t N,
                        int32_t K, int32_t dtype, int32_t activation, void* workspace,
                        size_t workspace_bytes, void* stream);

/*
 * Distillation from a teacher's top logits. Per row, with s the student's V
 * scores, (id_k, t_k) the teacher's K entries and T the temperature:
 *   q   = softmax of t / T over the entries that are present,
 *   p_T = softmax(s / T), p_1 = softmax(s), both over all V words,
 *   loss = soft T^2 sum_k q_k (log q_k - log p_T(id_k)) - hard log p_1(label),
 * where a term of weight soft = 0 or hard = 0 is left out.
 *   logits     device rows x V of `dtype`, stride ld; -inf masks a word;
 *   ids        device int32[rows][K]: words, -1 = absent entry (its logit is
 *              not looked at); a row may have none (no soft term). Entries of
 *              one word add up;
 *   teacher    device [rows][K] of teacher_dtype: the teacher's logits; -inf
 *              gives q = 0, and a row of such entries alone has no soft term;
 *   labels     device int32[rows] or NULL (no hard term); -1 = none;
 *   row_weight device float[rows] or NULL (1): scales the row's gradient, not
 *              its loss;
 *   loss       device float[rows];
 *   stats      device float[rows][3]: the maximum m of s, log sum
 *              exp((s - m) / T), and log sum exp(s - m) (with labels, else 0):
 *              what w2v_distill_backward needs;
 *   grad       device rows x V of `dtype`, stride ldg, or NULL (not wanted):
 *              row_weight (soft T (Q p_T - q) + hard (p_1 - [label])), Q = 1 if
 *              the row has an entry above -inf, else 0. May be the logits' own
 *              memory (same stride), not overlap them otherwise.
 * A row whose scores are all -inf has loss 0 and gradient 0. NaN or +inf
 * among a row's scores makes its loss and its whole gradient NaN, whatever
 * terms the row has; among its present teacher logits, its soft term. A row
 * with an id or a label outside [-1, V) has loss 0 and gradient 0 and is
 * recorded in the device's error word. Sums, statistics and loss are held in
 * fp32; the gradient is rounded once. The same call gives the same bits.
 * Limits: 0 <= K <= W2V_MAX_TEACHER, temperature in [2^-20, 2^20], rows >= 0,
 * V >= 1. workspace: device, 256-byte aligned, at least
 * w2v_distill_workspace_bytes(rows, V, dtype) bytes, contents need not be
 * initialised; calls that overlap in time must not share it.
 */
#define W2V_MAX_TEACHER 1024

size_t w2v_distill_workspace_bytes(int32_t rows, int32_t V, int32_t dtype);
int w2v_distill_loss(const void* logits, int64_t ld, int32_t rows, int32_t V, int32_t dtype,
                     const int32_t* ids, const void* teacher, int32_t K,
                     int32_t teacher_dtype, const int32_t* labels, float temperature,
                     float soft, float hard, const float* row_weight, float* loss,
                     float* stats, void* grad, int64_t ldg, void* workspace,
                     size_t workspace_bytes, void* stream);

/* The gradient of w2v_distill_loss alone, from the stats that it wrote for
 * the same logits, temperature and labels: grad = dloss_n d loss_n / d s, with
 * dloss device float[rows]. */
int w2v_distill_backward(const float* dloss, const void* logits, int64_t ld, int32_t rows,
                         int32_t V, int32_t dtype, const int32_t* ids, const void* teacher,
                         int32_t K, int32_t teacher_dtype, const int32_t* labels,
                         float temperature, float soft, float hard, const float* stats,
                         void* grad, int64_t ldg, void* stream);

/*
 * Words drawn from scores by given random numbers. Per row, with z the V
 * scores and m their maximum: x_j = (z_j - m) / T, w_j = exp(x_j). Words are
 * ranked by score, equal ones by index. Kept are the words whose rank is
 * below top_k, for which the weight of the words ranked before them is below
 * top_p times the weight of the top_k words, and whose w_j >= min_p; the first
 * is always kept. Of these the word with the largest x_j - log(-log u_j) is
 * drawn (the lowest index of equal ones): word j with probability w_j over
 * the kept words' weight, if the u_j are independent and uniform in (0, 1).
 *   logits    device rows x V of `dtype`, stride ld; -inf masks a word;
 *   uniforms  device float rows x V, stride ldu; may be NULL if temperature
 *             is the scalar 0. Of a row with filters only the kept words'
 *             numbers are read;
 *   temperatures, top_ks, top_ps, min_ps  device arrays of `rows` settings,
 *             each NULL to use the scalar after it for every row.
 *             Temperature 0 takes the best-ranked word (others below 2^-126
 *             act as 2^-126); top_k 0, top_p >= 1 and min_p 0 are off; top_k
 *             is at most W2V_MAX_TOP_K, or >= V, which is off;
 *   ids       device int32[rows]; logprob device float[rows] or NULL: x - log
 *             sum of all w, the word's log-probability at T before the filters
 *             (0 at temperature 0).
 * A row without a word above -inf, or with NaN among its scores, gets id -1
 * and logprob NaN. Words at +inf weigh 1 each and all others 0. A row whose
 * setting in an array is invalid (temperature not finite or < 0, top_k < 0 or
 * between W2V_MAX_TOP_K and V, top_p <= 0 or NaN, min_p outside [0, 1]) gets
 * the same and is recorded in the device's error word; invalid scalars are
 * W2V_EINVAL. A u_j of 0 or NaN loses against every other word. Weights are
 * summed in 64-bit fixed point of at least 2^-31 of the first word's weight,
 * so nothing depends on an order. workspace: device, 256-byte aligned, at
 * least w2v_sample_workspace_bytes(rows, V) bytes (0 where a block does a
 * whole row), contents need not be initialised; calls that overlap in time
 * must not share it.
 */
#define W2V_MAX_TOP_K 1024

size_t w2v_sample_workspace_bytes(int32_t rows, int32_t V);
int w2v_sample_words(const void* logits, int64_t ld, const float* uniforms, int64_t ldu,
                     int32_t rows, int32_t V, int32_t dtype, const float* temperatures,
                     float temperature, const int32_t* top_ks, int32_t top_k,
                     const float* top_ps, float top_p, const float* min_ps, float min_p,
                     int32_t* ids, float* logprob, void* workspace, size_t workspace_bytes,
                     void* stream);

/*
 * A word model's ends: what brings words in and what answers with them, beside
 * the vocabulary head. Matrices, element types and workspaces as there. (Not in
 * the paper, which ends with the trained vectors.)
 *
 * Rows by word: y_i = scale W[id_i], for W V x D of `dtype` (M_in of a trained
 * model) and y n x D of `out_dtype`, any of the types. The product is one of fp32
 * numbers, rounded as such and then, where scale is not a power of two, again to a
 * 16-bit out_dtype.
 *   ids       device int32[n]: words; -1 = absent, whose row of y is 0. Any
 *             other id outside [0, V) gives a row of 0 too and is recorded in
 *             the device's error word.
 * y must not overlap any other argument. Limits: n >= 0, V >= 1,
 * 1 <= D <= 2^24, scale finite.
 */
int w2v_embed(const int32_t* ids, int32_t n, const void* weight, int64_t ldw, int32_t V,
              int32_t D, int32_t dtype, float scale, void* y, int64_t ldy, int32_t out_dtype,
              void* stream);

/*
 * Gradient of w2v_embed for the weight, from dy (n x D of `dtype`):
 *   grad[v] = scale sum of dy_i over the i with ids[i] = v, 0 for other words;
 *   accumulate = 1: that is added to grad, whose other rows are not touched (a
 *   negative scale makes it a step of gradient descent on the weight itself).
 * grad is V x D of `grad_dtype`, any of the types. Ids as in w2v_embed; absent
 * and out-of-range ones add nothing. Sums are held in fp32, over the positions
 * sorted by word, in an order that depends on the ids alone: the same call gives the
 * same bits. The sum times scale (and the old value, in one fused operation) is rounded
 * to fp32 and then to a 16-bit grad_dtype. Ids are read once. workspace: device, 256-byte
 * aligned, at least w2v_embed_backward_workspace_bytes(n, V, D) bytes (0 for n =
 * 0), contents need not be initialised; calls that overlap in time must not
 * share it. grad must not overlap any other argument.
 */
size_t w2v_embed_backward_workspace_bytes(int32_t n, int32_t V, int32_t D);
int w2v_embed_backward(const void* dy, int64_t lddy, const int32_t* ids, int32_t n,
                       int32_t dtype, float scale, void* grad, int64_t ldg, int32_t V, int32_t D,
                       int32_t grad_dtype, int32_t accumulate, void* workspace,
                       size_t workspace_bytes, void* stream);

/*
 * Dropout: y = [r >= B] x 2^32 / (2^32 - B) + residual, B = floor(p 2^32 + 1/2),
 * for x, residual and y rows x cols of `dtype`. The mask is not stored: the
 * backward pass is the same call on dy (without the residual, whose gradient is
 * dy). Element i = row cols + col (whatever the strides) has the 32-bit number
 * r_i = 2^16 h_i + l_i; h and l are halves of words of Philox4x32-10 (Salmon et
 * al., SC'11) with key (seed mod 2^32, seed / 2^32) and counter (b mod 2^32, b /
 * 2^32 + 2^31 s, o mod 2^32, o / 2^32), b = i / 8, s = 0 for h and 1 for l: half
 * i mod 8, a word's low half before its high one.
 *   o          offset + *offset_dev, modulo 2^64: a different number for every
 *              layer and step. offset_dev: device int64[1] or NULL (0), read by
 *              the kernel, so that a captured graph gets new numbers as the
 *              caller counts it up;
 *   residual   or NULL (0); y may be x or the residual itself (same stride) and
 *              must not overlap them otherwise.
 * Whatever a dropped element holds (NaN, infinities) does not reach y. The factor
 * 2^32 / (2^32 - B) is the nearest fp32 number; the product and the sum are formed in
 * fp32, rounded as one, and then to a 16-bit dtype. p = 0 keeps and p = 1 drops
 * everything. Limits: 0 <= p <= 1, rows >= 0, 1 <= cols <= 2^30.
 */
int w2v_dropout(const void* x, int64_t ldx, const void* residual, int64_t ldr, void* y,
                int64_t ldy, int32_t rows, int32_t cols, int32_t dtype, double p, uint64_t seed,
                uint64_t offset, const int64_t* offset_dev, void* stream);

/*
 * A matrix in 4 bits. W (N x K) has G = ceil(K / group) groups of columns, group
 * = 32, 64 or 128, and W_nk is held as scale_n,g (q - 8), q in [0, 15], with
 * bfloat16 scales: scale = max |W| of the group / 7, rounded, and q = W / scale
 * rounded to the nearest integer (even at ties), within [-8, 7], plus 8. A group
 * with NaN or infinities becomes NaN.
 * Layout: rows are in tiles of 16 (missing rows have q = 8 and scale 0), columns
 * in B = G group / 32 blocks of 32 (missing ones have q = 8), which lie in fours,
 * the rest (B mod 4) together:
 *   packed  uint32[ceil(N / 16)][B * 64]: of blocks 4 i to 4 i + 3, word
 *           [256 i + 4 l + j] is block 4 i + j's for lane l = 16 c + r, of the R
 *           others word [256 (B / 4) + R l + j]; it holds row r of the tile,
 *           columns 8 c to 8 c + 7 of the block: column 8 c + k in bits 2 k to 2
 *           k + 3 for even k, 2 k + 14 to 2 k + 17 for odd k;
 *   scales  bfloat16[ceil(N / 16)][G * 16]: of groups 4 i to 4 i + 3, [64 i + 4 r
 *           + j] is group 4 i + j's for row r, of the R others [64 (G / 4) + R r +
 *           j].
 * packed is of w2v_q4_packed_bytes bytes, scales of w2v_q4_scale_count elements
 * (0 on invalid arguments), both 16-byte aligned. K <= 2^24.
 */
size_t w2v_q4_packed_bytes(int32_t N, int32_t K, int32_t group);
size_t w2v_q4_scale_count(int32_t N, int32_t K, int32_t group);
int w2v_quantize_q4(const void* w, int64_t ldw, int32_t N, int32_t K, int32_t dtype,
                    int32_t group, void* packed, void* scales, void* stream);

/*
 * y = x W^T + bias for such a W, x M x K of `dtype` and y M x N of `out_dtype`
 * (dtype or W2V_DTYPE_F32); bias: device float[N] or NULL. Made for few rows:
 * the matrix is read once for every 64 of them (16-bit x) or 32 (fp32), or for
 * fewer with K in the thousands. Products x (q - 8) are exact and sums fp32: a
 * group's, which is multiplied with its scale, and the row's. A row of x with an
 * infinity gives NaN. The same call gives the same bits. M = 0 is allowed and does
 * nothing; M <= W2V_MAX_Q4_ROWS. y must not overlap any other argument.
 */
#define W2V_MAX_Q4_ROWS 524288

int w2v_linear_q4(const void* x, int64_t ldx, const void* packed, const void* scales,
                  const float* bias, void* y, int64_t ldy, int32_t M, int32_t N, int32_t K,
                  int32_t group, int32_t dtype, int32_t out_dtype, void* stream);

/*
 * A step of beam search over `batch` entries of `beams` beams each: of an entry's
 * pairs (beam b, word v), the `width` with the largest scores_b + log p_b(v), p_b
 * = softmax of row entry beams + b of the logits over all V words. Pairs of one
 * beam are ranked by logit, equal ones by word; of different beams by the sum,
 * formed in 64 bits from a sum of exponentials in fp32, equal ones by beam.
 *   logits       device (batch * beams) x V of `dtype`, stride ld; -inf masks a
 *                word;
 *   scores       device float[batch][beams], a beam's log-probability so far;
 *                -inf: the beam is none (a search starts with one beam per entry
 *                at 0 and the others at -inf), and its logits are not read;
 *   finished     device uint8[batch][beams] or NULL (none): a beam other than 0
 *                has ended. It is one pair, (b, end) at its score, and its logits
 *                are not read. Needs end >= 0;
 *   end          the word that ends a beam, or -1;
 *   words, parents  device int32[batch][width]: the pairs, best first; parents in
 *                [0, beams). Where there are fewer pairs than width: -1, score
 *                -inf;
 *   new_scores   device float[batch][width];
 *   new_finished device uint8[batch][width] or NULL: 1 where the parent had ended
 *                or the word is end.
 * An entry with a score of NaN or +inf, or with NaN or +inf among the logits of a
 * beam that goes on, gets words and parents -1, scores NaN and flags 0. Outputs
 * must not overlap any other argument. workspace: device, 256-byte aligned, at
 * least w2v_beam_step_workspace_bytes bytes, contents need not be initialised;
 * calls that overlap in time must not share it. Limits: 1 <= beams, width <=
 * W2V_MAX_BEAMS, batch >= 0, V >= 1.
 */
#define W2V_MAX_BEAMS 64

size_t w2v_beam_step_workspace_bytes(int32_t batch, int32_t beams, int32_t width, int32_t V,
                                     int32_t dtype);
int w2v_beam_step(const void* logits, int64_t ld, int32_t batch, int32_t beams, int32_t V,
                  int32_t dtype, const float* scores, const uint8_t* finished, int32_t end,
                  int32_t width, int32_t* words, int32_t* parents, float* new_scores,
                  uint8_t* new_finished, void* workspace, size_t workspace_bytes, void* stream);

/* A state of every beam: rows of row_bytes bytes (1 to W2V_MAX_STATE_BYTES), of
 * any meaning and alignment, row strides in bytes. */
typedef struct {
  const void* src; /* device, batch * beams rows */
  int64_t src_stride;
  void* dst; /* device, batch * width rows */
  int64_t dst_stride;
  int64_t row_bytes;
} w2v_beam_state;
#define W2V_MAX_BEAM_STATES 16
#define W2V_MAX_STATE_BYTES 17179869184 /* 2^34 */

/*
 * Moves states to where w2v_beam_step's pairs are: row entry width + j of dst is
 * row entry beams + parents[entry][j] of src; a row of zeros where the parent is
 * -1, or outside [-1, beams), which is recorded in the device's error word.
 * states: host, `count` <= W2V_MAX_BEAM_STATES of them, read before the call
 * returns. dst must not overlap any src.
 */
int w2v_beam_reorder(const w2v_beam_state* states, int32_t count, const int32_t* parents,
                     int32_t batch, int32_t beams, int32_t width, void* stream);

#ifdef __cplusplus
}
#endif
#endif
