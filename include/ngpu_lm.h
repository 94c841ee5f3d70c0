/*
 * ngpu_lm.h -- C ABI of the MI355X batched backoff n-gram language model.
 *
 * The library answers the query of Section 2.2 of the NGPU-LM paper
 * (arXiv 2505.22857): for a batch of B language-model states it returns the
 * score of every vocabulary token and the state reached after it,
 *     state[B] -> (scores[B, V], next_state[B, V]),
 * by walking the backoff chain of each state (Algorithm 1), and it fuses that
 * query into one greedy shallow-fusion decoding step (Section 2.3).
 *
 * Conventions shared by every call:
 *   - Weights are natural logarithms in fp32 (the paper stores "logarithms"
 *     without a base; an ARPA log10 value must be multiplied by ln 10 before it
 *     is passed in).  Scores are natural-log fp32.
 *   - A state is a context: the empty context (state 0) or a listed n-gram of
 *     order 1..N-1 (Section 2.1; highest-order n-grams have no state).  State ids
 *     are canonical: 0 is the empty context, then contexts ordered by
 *     (order ascending, token tuple lexicographically ascending) -- the order of
 *     arcs sorted by (from_state, token), Section 2.2.
 *   - Device memory is always owned by the caller.  The library never
 *     allocates device memory and never synchronises a stream except in
 *     ngpu_lm_check_states.  Calls taking `hip_stream` enqueue work on that
 *     hipStream_t (NULL = the null stream) and return once it is enqueued.
 *   - Queries launch on the current device, which must be the device whose
 *     memory holds the uploaded image (NGPU_E_INVALID_ARG otherwise).
 *   - Every call returns NGPU_OK (0) or a negative NGPU_E_* code and then sets a
 *     thread-local message readable with ngpu_lm_last_error().  No call throws.
 *   - A handle may be used from several threads for queries; build, upload and
 *     free must not race with other calls on the same handle.
 */
#ifndef NGPU_LM_H
#define NGPU_LM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define NGPU_LM_MAX_ORDER 10      /* the paper's models go up to order 10 */
#define NGPU_LM_MAX_VOCAB 8192    /* a V-wide score/state row (8 bytes per token) must fit in 64 KiB of LDS */
/* Most states a model may have: the kernels keep a state id in 30 bits of a
 * 32-bit word (the two high bits flag how a row slot was filled).  A larger
 * model is rejected with NGPU_E_TOO_LARGE. */
#define NGPU_LM_MAX_STATES ((int64_t)1 << 30)
/* Most hypotheses (or utterances) per call: the launch grid, 64 work-items per
 * hypothesis, must fit a 32-bit dispatch size.  Larger batches return
 * NGPU_E_INVALID_ARG; split them into several calls. */
#define NGPU_LM_MAX_BATCH ((int64_t)(1 << 26) - 256)

enum ngpu_status {
    NGPU_OK = 0,
    NGPU_E_INVALID_ARG = -1,      /* null pointer, bad size, misaligned buffer, bad mode */
    NGPU_E_TOKEN_RANGE = -2,      /* a token outside [0, V) */
    NGPU_E_ORDER_RANGE = -3,      /* an order outside [1, max_order] or max_order outside [1, 10] */
    NGPU_E_DUPLICATE_NGRAM = -4,  /* the same token tuple listed twice */
    NGPU_E_MISSING_PREFIX = -5,   /* an n-gram whose context (all but the last token) is not listed */
    NGPU_E_MISSING_SUFFIX = -6,   /* an n-gram whose suffix (all but the first token) is not listed */
    NGPU_E_MISSING_UNIGRAM = -7,  /* a token with no unigram and no <unk> weight given */
    NGPU_E_NOT_UPLOADED = -8,     /* a query before ngpu_lm_upload */
    NGPU_E_HIP = -9,              /* a HIP runtime error (message has the HIP error string) */
    NGPU_E_NONFINITE = -10,       /* a NaN/inf weight */
    NGPU_E_TOO_LARGE = -11,       /* vocabulary, order or count beyond the library's limits */
    NGPU_E_BAD_STATE = -12,       /* ngpu_lm_check_states found out-of-range input states */
    NGPU_E_NO_MEMORY = -13        /* host allocation failed */
};

typedef struct ngpu_lm ngpu_lm;   /* opaque; owns host arrays only */

/* An n-gram list, the array form of an ARPA file (Section 2.1).  Row i is the
 * n-gram tokens[i*max_order .. i*max_order + order[i] - 1] (context first,
 * predicted token last; the remaining entries of the row are ignored), with
 * log-probability logprob[i] and backoff weight backoff[i] (0 when the ARPA
 * line has none; ignored for order max_order).  Rows may come in any order.
 * The list must be closed: every n-gram of order k >= 2 needs its first k-1
 * tokens and its last k-1 tokens listed as n-grams too (KenLM output is). */
typedef struct {
    int64_t num_ngrams;
    int32_t max_order;            /* N, 1..NGPU_LM_MAX_ORDER */
    const int32_t *order;         /* [num_ngrams] */
    const int32_t *tokens;        /* [num_ngrams * max_order] */
    const float *logprob;         /* [num_ngrams] natural log */
    const float *backoff;         /* [num_ngrams] natural log */
} ngpu_ngram_list;

typedef struct {
    int64_t num_states;           /* S: 1 + number of n-grams of order < N */
    int64_t num_arcs;             /* arcs out of non-empty contexts (n-grams of order >= 2) */
    int32_t max_order;
    int32_t vocab_size;
    int64_t device_bytes;         /* size of the device image */
} ngpu_lm_info_t;

/* Build flag: the list also holds the sentence markers of an ARPA model, as
 * token V (<s>) and token V + 1 (</s>).  <s> may only open an n-gram and is
 * never scored (its unigram weight is ignored); the state of the context <s>
 * is the start state (ngpu_lm_start_state).  </s> may only close an n-gram;
 * n-grams ending in </s> are not arcs but give each state its final weight,
 * the </s> score folded through the backoff chain at build time (Section 2.3,
 * AED; ngpu_lm_final_weights, NGPU_FUSION_AED).  Both need a unigram (or, for
 * </s>, an <unk> weight). */
#define NGPU_BUILD_BOS_EOS 1u

/* Build flag: close a list that is not closed (a pruned ARPA model) instead of
 * rejecting it.  Every missing prefix and suffix of a listed n-gram (for an
 * n-gram ending in </s>, its prefix) is inserted with backoff weight 0 and the
 * weight the backoff rule of Section 2.1 gives it on the list without it; for
 * an inserted c + v of order >= 2 that is B(c) + W(c[1:] + v) in one fp32 add
 * (B(c) = 0 when c is inserted too), for an inserted unigram the <unk> weight
 * (NGPU_E_MISSING_UNIGRAM without one).  The score of every token after every
 * history is unchanged; the inserted contexts become states, so the state walk
 * reaches the longest listed context of a history as the backoff rule does. */
#define NGPU_BUILD_REPAIR_CLOSURE 2u

/* Build the trie from a closed n-gram list (Section 2.2): states numbered
 * canonically, arcs sorted by (from_state, token) with one contiguous range per
 * state, a dense row over all V tokens for the empty context (a token without a
 * unigram gets unk_logprob and leads to state 0; pass NaN when every token has
 * a unigram), and per state its backoff weight and backoff state (its context
 * minus the first token).  An arc of order < N leads to the state of its own
 * n-gram, an arc of order N to the state of its last N-1 tokens.  The image
 * stores this as one record per state holding its whole backoff chain (arc
 * ranges and the backoff weights already summed in Algorithm 1's order) and a
 * dense V-wide row per order-1 context (layout in csrc/trie.h).
 * vocab_size: 1..NGPU_LM_MAX_VOCAB; additionally ceil(log2 V') * N <= 128 with
 * V' = V (V + 2 with NGPU_BUILD_BOS_EOS), and at most NGPU_LM_MAX_STATES
 * states (NGPU_E_TOO_LARGE otherwise).
 * flags: NGPU_BUILD_BOS_EOS and/or NGPU_BUILD_REPAIR_CLOSURE (else
 * NGPU_E_MISSING_PREFIX / NGPU_E_MISSING_SUFFIX for a list that is not closed).
 * The list is read only during the call.
 * On success *out holds a new handle (free with ngpu_lm_free). */
int ngpu_lm_build(const ngpu_ngram_list *list, int32_t vocab_size, float unk_logprob,
                  uint32_t flags, ngpu_lm **out);

void ngpu_lm_free(ngpu_lm *lm);

int ngpu_lm_info(const ngpu_lm *lm, ngpu_lm_info_t *out);

/* Context tuple of a state: writes its order to *order_out (0 for state 0) and
 * its tokens to tokens_out[0 .. order-1] (capacity max_order - 1). */
int ngpu_lm_state_context(const ngpu_lm *lm, int64_t state, int32_t *tokens_out, int32_t *order_out);

/* The state decoding starts from: the context <s> for a model built with
 * NGPU_BUILD_BOS_EOS (and order >= 2), else the empty context 0. */
int ngpu_lm_start_state(const ngpu_lm *lm, int64_t *state);

/* Final weight of each state d_states[b] into d_final[b] (fp32): the </s>
 * score of the state (Section 2.3, AED), precomputed per state at build time
 * by the same fp32 fold as a query.  Needs NGPU_BUILD_BOS_EOS
 * (NGPU_E_INVALID_ARG otherwise).  Out-of-range states give NaN and are
 * counted for ngpu_lm_check_states.  Asynchronous on hip_stream. */
int ngpu_lm_final_weights(const ngpu_lm *lm, const int32_t *d_states, int64_t B, float *d_final,
                          void *hip_stream);

/* Bytes of device memory the trie image needs (also in ngpu_lm_info). */
size_t ngpu_lm_device_bytes(const ngpu_lm *lm);

/* Copy the trie image into dev_buf (caller-owned device memory of at least
 * ngpu_lm_device_bytes bytes, 256-byte aligned) with one asynchronous copy on
 * hip_stream, and remember dev_buf for later queries.  The host image stays
 * alive in the handle, so the copy needs no synchronisation by the caller
 * beyond stream order.  dev_buf must stay valid while queries are in flight.
 * Uploading again (e.g. to another buffer) replaces the remembered pointer. */
int ngpu_lm_upload(ngpu_lm *lm, void *dev_buf, size_t dev_bytes, void *hip_stream);

/* Batched full-vocabulary query (Algorithm 1, batched): for each b < B,
 * row b of d_scores ([B, V] fp32, row-major) and d_next ([B, V] int32) get the
 * score and the next state of every token v from state d_states[b].
 * The score is the fp32 left fold of Algorithm 1: an accumulator starting at 0
 * gains the backoff weight of each state left on the way down, and the first
 * level holding v adds its weight once.  Device pointers; d_scores and d_next
 * must not overlap.  States must lie in [0, num_states): an out-of-range state
 * yields a row of NaN scores and -1 next states and is counted for
 * ngpu_lm_check_states.  B = 0 is a no-op.  Asynchronous on hip_stream. */
int ngpu_lm_advance(const ngpu_lm *lm, const int32_t *d_states, int64_t B, float *d_scores,
                    int32_t *d_next, void *hip_stream);

enum ngpu_fusion_mode {
    NGPU_FUSION_PLAIN = 0,        /* argmax_v fma(lambda, lm[v], asr[v]) over v < V, then advance */
    NGPU_FUSION_CTC = 1,          /* blank / repeat / other groups (Section 2.3, CTC) */
    NGPU_FUSION_TRANSDUCER = 2,   /* two-stage selection (Section 2.3, transducers) */
    NGPU_FUSION_AED = 3           /* class V is <eos>, scored with the state's final weight (Section 2.3, AED) */
};

/* One greedy shallow-fusion step (Section 2.3) for B hypotheses.
 * d_asr: [B, asr_ld] fp32 ASR log-probabilities; row b holds classes 0..V-1
 *   (tokens) and, for CTC and transducer modes, class V = blank (AED: <eos>);
 *   asr_ld >= V (PLAIN) or >= V + 1.  Blank is always the last class, so no
 *   blank index is passed.
 * lambda: LM weight; the fused score of token v is fmaf(lambda, lm[v], asr[v])
 *   (single rounding), lm[v] being the advance score.
 * PLAIN: label = argmax over v < V of the fused score; state <- next[label].
 * CTC: a = argmax over all V + 1 classes of the raw ASR score.  If a is blank
 *   or equals d_prev[b] (a repeat, collapsed by CTC and not rescored), label = a
 *   and the state stays.  Otherwise label = argmax over v < V, v != d_prev[b]
 *   of the fused score, and state <- next[label].  Then d_prev[b] = label.
 * TRANSDUCER: a = raw argmax over V + 1 classes; blank stays blank with no state
 *   change; otherwise label = fused argmax over v < V and the state advances.
 * AED (model built with NGPU_BUILD_BOS_EOS): class V is <eos>; label = argmax
 *   over v <= V of the fused score, <eos> using the state's final weight as its
 *   LM score; <eos> leaves the state unchanged, a token advances it.
 * Ties go to the lowest index (-0 equals +0).  ASR scores may be -inf: a
 * candidate set entirely at -inf yields its first candidate, as a strict '>'
 * scan from index 0 does; a (quiet) NaN counts as -inf.  In/out: d_states[B] (int32), d_prev[B] (CTC
 * only; may be NULL otherwise).  Out: d_tokens[B] (int32 label, V = blank).
 * Out-of-range states give label -1, leave the state unchanged and are counted
 * for ngpu_lm_check_states.  Asynchronous on hip_stream. */
int ngpu_lm_fused_greedy_step(const ngpu_lm *lm, const float *d_asr, int64_t B, int64_t asr_ld,
                              int32_t mode, float lambda, int32_t *d_states, int32_t *d_prev,
                              int32_t *d_tokens, void *hip_stream);

#define NGPU_LM_MAX_TOPK 256

/* The k best tokens of the fused score fmaf(lambda, lm[v], asr[v]) over
 * v < V for each hypothesis -- the expansion step of a beam search with the
 * LM fused over the full vocabulary (Section 2.3: full-vocabulary scoring
 * before selection; the paper applies it to AED beam search).  Row b of the
 * outputs ([B, k] each, row-major) lists the k best in descending order of
 * the fused score, ties to the lower token index: d_tokens (int32), d_scores
 * (fp32 fused scores), d_next (int32 state after that token); when fewer
 * than k tokens score above -inf, the rest follow in index order (as a strict
 * '>' selection gives; a NaN score counts as -inf).  States are read only.
 * 1 <= k <= min(V, NGPU_LM_MAX_TOPK); cost per hypothesis: one pass over the V
 * tokens, then a selection whose cost hardly grows with k (a lower bound of the
 * k-th largest value, a short list of the tokens that reach it, and each
 * token's rank in that list).  An out-of-range state gives a
 * row of -1 tokens, NaN scores and -1 states and is counted for
 * ngpu_lm_check_states.  Asynchronous. */
int ngpu_lm_fused_topk(const ngpu_lm *lm, const float *d_asr, int64_t B, int64_t asr_ld, float lambda, int32_t k,
                       const int32_t *d_states, int32_t *d_tokens, float *d_scores, int32_t *d_next,
                       void *hip_stream);

/* A whole greedy decode (Section 2.3) in one launch: for each utterance b,
 * frames t = 0 .. len_b - 1 run the rule of ngpu_lm_fused_greedy_step on the
 * ASR row d_asr + b * stride_b + t * stride_t (strides in floats; the row holds
 * classes 0..V-1 and, for CTC and transducer, blank = V), carrying the state
 * and the previous label from frame to frame.
 * d_lengths: [B] int32 frame counts (clamped to [0, T]) or NULL for T.
 * In/out: d_states[B] (start states; final states on return), d_prev[B] (CTC:
 *   the label before frame 0, blank = V for a new utterance; the last label on
 *   return; may be NULL otherwise).  Passing the returned states and labels
 *   back continues a decode exactly where it stopped.
 * Out: d_labels[B, T] int32 (row b at d_labels + b * T): the label of each
 *   frame, -1 past the utterance's length; d_label_states[B, T] (or NULL): the
 *   state after each frame.  An out-of-range start state gives a row of -1 and
 *   is counted for ngpu_lm_check_states.  Asynchronous on hip_stream. */
int ngpu_lm_fused_greedy_decode(const ngpu_lm *lm, const float *d_asr, int64_t B, int64_t T, int64_t stride_b,
                                int64_t stride_t, const int32_t *d_lengths, int32_t mode, float lambda,
                                int32_t *d_states, int32_t *d_prev, int32_t *d_labels, int32_t *d_label_states,
                                void *hip_stream);

/* ------------------------------------------------------------------------
 * Speculative decoding with the n-gram model as the drafter.  One round over a
 * batch of sequences: ngpu_lm_draft proposes K tokens a sequence, the network
 * runs once over them, appending its keys and values to a paged cache
 * (ngpu_lm_kv_append) that its attention reads (ngpu_lm_attend), and
 * ngpu_lm_verify keeps a prefix of the draft and adds one token, so that the
 * tokens are distributed as the network's own.
 *
 * Random numbers are inputs.  A token is drawn from weights w >= 0 with unit
 * exponential noise e as the argmax of w / e (the lowest token of several),
 * which picks v with probability w[v] / sum(w).  A NaN counts as the lowest
 * value.
 * ------------------------------------------------------------------------ */

/* Most drafted tokens a sequence and round. */
#define NGPU_LM_MAX_DRAFT 63
/* Least temperature other than 0 (greedy). */
#define NGPU_LM_MIN_TEMPERATURE 1e-6f
/* Most sequences (ngpu_lm_verify, ngpu_lm_kv_append, ngpu_lm_attend) per call. */
#define NGPU_LM_MAX_SEQUENCES (1 << 20)

enum ngpu_dtype { NGPU_F32 = 0, NGPU_F16 = 1, NGPU_BF16 = 2 };

/* Draft K tokens (1..NGPU_LM_MAX_DRAFT) for each of B sequences from the n-gram
 * model alone: with x = lm / temperature over the V tokens,
 *   log p = x - max(x) - log sum exp(x - max(x)),
 *   token = argmax_v exp(x[v] - max(x)) / e[v],   state <- next[token],
 * K times.  temperature 0: token = argmax_v lm[v], the lowest of several.
 * d_states [B]: the states the sequences are in; not changed.
 * d_last [B] or NULL: a token each sequence takes before the draft starts (the
 *   one that the verification before added), -1 for none.
 * d_noise: unit exponential noise, V values at d_noise + b * noise_stride_b +
 *   k * noise_stride_k (elements); unused (may be NULL) at temperature 0.
 * d_tokens [B, K]; d_draft_states [B, K + 1]: the state before the draft, then the
 *   one after each of its tokens; d_logprobs [B, K, V]: log p, the rows that
 *   ngpu_lm_verify takes, or NULL; must be NULL at temperature 0, where the
 *   draft has all its mass on one token.
 * A state outside [0, num_states) or a last token outside [-1, V) gives -1
 * tokens and states and NaN rows and is counted for ngpu_lm_check_states. */
int ngpu_lm_draft(const ngpu_lm *lm, const int32_t *d_states, const int32_t *d_last, int64_t B, int32_t K,
                  float temperature, const float *d_noise, int64_t noise_stride_b, int64_t noise_stride_k,
                  int32_t *d_tokens, int32_t *d_draft_states, float *d_logprobs, void *hip_stream);

/* Verification of drafted tokens.  Strides are in elements; the last dimension
 * of logits, log-probabilities and noise has unit stride. */
typedef struct {
    int64_t B;                     /* sequences */
    int32_t K;                     /* drafted tokens a sequence, 0..NGPU_LM_MAX_DRAFT */
    int64_t V;                     /* vocabulary, 1..2^31 - 1 */
    int32_t dtype;                 /* of the logits, ngpu_dtype */
    const void *logits;            /* [B, K + 1, V]: row k scores the token at place k */
    int64_t logits_stride_b, logits_stride_k;
    const int32_t *tokens;         /* [B, K] drafted tokens; one outside [0, V) ends its sequence's draft */
    const int32_t *lengths;        /* [B] drafted tokens that count, clamped to [0, K], or NULL for K */
    const float *logprobs;         /* [B, K, V] natural-log probabilities the draft was drawn with, or NULL: each
                                    * token had probability 1 (greedy drafts) */
    int64_t logprobs_stride_b, logprobs_stride_k;
    const float *uniforms;         /* [B, K] uniform numbers in [0, 1) */
    const float *noise;            /* [B, V] unit exponential noise for the token that is added */
    int64_t noise_stride_b;
    float temperature;             /* of the network's softmax; 0: greedy, and logprobs, uniforms and noise are unused */
    const int32_t *draft_states;   /* [B, K + 1] as ngpu_lm_draft gives them, or NULL */
    int32_t *out_tokens;           /* [B, K + 1]: the kept tokens, the added one, then -1 */
    int32_t *accepted;             /* [B] kept tokens a sequence, 0..K */
    int32_t *states;               /* [B] draft_states at the kept tokens' end (the added token is not taken yet:
                                    * it is the next draft's last token), or NULL */
} ngpu_verify_t;

/* Device memory a verification needs, 16-byte aligned, not initialised; free
 * again when the call's work has run. */
size_t ngpu_lm_verify_workspace(int64_t B, int32_t K, int64_t V);

/* With p = softmax(logits / temperature) and q = exp(logprobs) (or 1 at the drafted
 * token): the token x at place k is kept while every one before it is and
 *   uniforms[k] * q[k][x] < p[k][x].
 * At the first place a whose token is not kept, the added token is drawn from
 * max(p[a] - q[a], 0) with the noise, at the draft's end (and where that leaves
 * nothing) from p[a].  temperature 0: x is kept while it is the row's argmax (the
 * lowest of several), and the added token is the argmax of row a.
 * A NaN logit counts as -inf; +inf logits share the row's whole mass; a row with
 * nothing above -inf gives every token p = 0, so nothing is kept there and
 * token 0 is added.  Classes that the draft does not know (an end-of-sequence class of the network's) have
 * log-probability -inf in its rows, which have V columns.  B = 0 is a no-op. */
int ngpu_lm_verify(const ngpu_verify_t *args, void *d_workspace, size_t workspace_bytes, void *hip_stream);

/* A paged cache of keys and values: pages of page_size tokens, each with `heads`
 * heads of `dim` elements (unit stride).  Strides in elements. */
typedef struct {
    int32_t dtype;                 /* NGPU_F16 or NGPU_BF16 */
    int32_t heads, dim;            /* dim: 1..NGPU_LM_MAX_HEAD_DIM */
    int32_t page_size;             /* tokens */
    int64_t num_pages;
    void *k, *v;
    int64_t k_stride_page, k_stride_token, k_stride_head;
    int64_t v_stride_page, v_stride_token, v_stride_head;
} ngpu_kv_cache_t;
#define NGPU_LM_MAX_HEAD_DIM 256

enum ngpu_rope_layout {
    NGPU_ROPE_HALF = 0,            /* pairs (i, i + rotary / 2) */
    NGPU_ROPE_INTERLEAVED = 1      /* pairs (2 i, 2 i + 1) */
};

/* New keys and values of S sequences, T tokens each (padded), for the cache. */
typedef struct {
    int64_t S, T;
    const void *k, *v;             /* [S, T, heads, dim], the cache's type, unit stride in the last dimension */
    int64_t k_stride_seq, k_stride_token, k_stride_head;
    int64_t v_stride_seq, v_stride_token, v_stride_head;
    const void *q;                 /* [S, T, q_heads, dim] queries to rotate too, or NULL */
    int32_t q_heads;
    int64_t q_stride_seq, q_stride_token, q_stride_head;
    void *q_out;                   /* [S, T, q_heads, dim] contiguous; must not overlap q */
    const int32_t *pages;          /* [S, pages_width] page tables, row stride pages_stride */
    int64_t pages_width, pages_stride;
    const int32_t *start;          /* [S] place of each sequence's first new token among its own tokens */
    const int32_t *lengths;        /* [S] new tokens that count, clamped to [0, T], or NULL for T */
    int32_t rotary;                /* rotated leading dimensions: even, 0..dim; 0: no rotation */
    int32_t layout;                /* ngpu_rope_layout */
    const int32_t *positions;      /* [S, T] row of the tables for each token, or NULL: start + t */
    const float *cos, *sin;        /* [positions_count, rotary / 2] contiguous */
    int64_t positions_count;
} ngpu_kv_append_t;

/* Token t of sequence s goes to place start[s] + t of its own tokens, that is to
 * entry (place mod page_size) of page pages[s][place / page_size], with its key's
 * (and query's) pairs (a, b) turned to (a cos - b sin, b cos + a sin) in fp32
 * and rounded once.  A token that does not count, or whose place lies outside
 * the table or on a page outside [0, num_pages), is not stored; its query is
 * rotated all the same where it counts, and rows of q_out that do not count are
 * zero.  A position outside [0, positions_count) gives NaN keys and queries.
 * Places must not repeat within a call (two sequences on one page entry). */
int ngpu_lm_kv_append(const ngpu_kv_cache_t *cache, const ngpu_kv_append_t *args, void *hip_stream);

/* Attention of S sequences with T query tokens each over the cache.  The
 * sequences come in G groups of S / G: those of one group share a prefix of
 * cached tokens, and each has tokens of its own after it. */
typedef struct {
    int64_t S, T;
    int32_t q_heads;               /* a multiple of the cache's heads; consecutive ones share a cache head */
    const void *q;                 /* [S, T, q_heads, dim], the cache's type, unit stride in the last dimension */
    int64_t q_stride_seq, q_stride_token, q_stride_head;
    const int32_t *q_lengths;      /* [S] query tokens that count, clamped to [0, T], or NULL for T */
    int64_t G;                     /* groups (divides S), 0: no shared prefix */
    const int32_t *prefix_pages;   /* [G, prefix_width] page tables of the prefixes */
    int64_t prefix_width, prefix_stride;
    const int32_t *prefix_lengths; /* [G] tokens, clamped to what the table holds */
    const int32_t *pages;          /* [S, pages_width] page tables of the own tokens, or NULL: none */
    int64_t pages_width, pages_stride;
    const int32_t *lengths;        /* [S] own tokens, the query tokens among them (the last ones), clamped alike */
    float scale;                   /* of the scores */
    void *out;                     /* [S, T, q_heads, dim] contiguous */
    float *lse;                    /* [S, T, q_heads] log of the softmax's sum, or NULL */
} ngpu_attend_t;

/* Device memory an attention needs, 16-byte aligned, not initialised.  To be asked with the call's own arguments:
 * it follows from the sizes, the strides, whether `pages` is NULL and the 16-byte alignment of k, v and out, and
 * is 0 for arguments that the call refuses (a cache without its pointers among them). */
size_t ngpu_lm_attend_workspace(const ngpu_kv_cache_t *cache, const ngpu_attend_t *args);

/* Query t < q_lengths[s] attends to every token of its group's prefix and to the
 * own tokens j < lengths[s] - q_lengths[s] + t + 1:
 *   out = sum_j softmax_j(scale * q . k_j) v_j,
 * the sums in fp32.  Keys on a page outside [0, num_pages) do not take part, nor
 * does anything else that a query does not attend to, whatever it holds.  A row
 * without any key, and one that does not count, is zero with lse = -inf.
 * The matrix cores take caches whose dim and strides are multiples of 8 elements, with k, v and out aligned to
 * 16 bytes, whose pages span no more than 2^34 elements (32 GiB; page stride times num_pages); a kernel that
 * reads element by element and each row's keys by themselves takes the others, many times slower. */
int ngpu_lm_attend(const ngpu_kv_cache_t *cache, const ngpu_attend_t *args, void *d_workspace,
                   size_t workspace_bytes, void *hip_stream);

/* A paged cache in 8 bits.  An element is an e4m3 value (1 sign, 4 exponent and 3 mantissa bits, largest 448, no
 * infinities) and stands for that times the scale of its block of tokens and its head: entry i of page p and head h has
 * scale [p][i / block][h].  Scales are finite and positive. */
typedef struct {
    ngpu_kv_cache_t cache;         /* k and v: bytes, as strides are; dtype: NGPU_F16 or NGPU_BF16, the type of the queries,
                                    * keys and values that go with it */
    int32_t block;                 /* tokens a scale, divides page_size; at most NGPU_LM_MAX_SCALE_BLOCK */
    float *k_scale, *v_scale;      /* [num_pages, page_size / block, heads] */
    int64_t k_scale_stride_page, k_scale_stride_block, k_scale_stride_head;
    int64_t v_scale_stride_page, v_scale_stride_block, v_scale_stride_head;
} ngpu_kv_cache8_t;
#define NGPU_LM_MAX_SCALE_BLOCK 65536

/* ngpu_lm_kv_append for a cache in 8 bits.  The rotated keys, in fp32, and the values are rounded once to e4m3.  A block's
 * scale for a head is the least power of two s (2^-100 at least) with 448 s no smaller than the new tokens' finite elements;
 * a block whose entries before the first new one are kept (that one is not its entry 0) keeps its scale where that holds the
 * new tokens and is 2^-100 at least, and else takes the new one, and the entries before are rounded again to it.  A scale there that is
 * not finite and positive counts as 2^-100.  What lies behind the last
 * new token of a block is no longer meaningful.  Elements that are not finite become NaN.  No two sequences of a call
 * may append to one block.  Scales that overlap, as with a stride of 0 or one array for keys and values, are refused. */
int ngpu_lm_kv_append8(const ngpu_kv_cache8_t *cache, const ngpu_kv_append_t *args, void *hip_stream);

/* ngpu_lm_attend over a cache in 8 bits: keys and values are the elements times their scales, in fp32.
 * The matrix cores take caches whose dim and strides are multiples of 16 elements, with k, v and out aligned to 16 bytes,
 * whose pages span no more than 2^35 elements; an element kernel takes the others, many times slower. */
size_t ngpu_lm_attend8_workspace(const ngpu_kv_cache8_t *cache, const ngpu_attend_t *args);
int ngpu_lm_attend8(const ngpu_kv_cache8_t *cache, const ngpu_attend_t *args, void *d_workspace,
                    size_t workspace_bytes, void *hip_stream);

/* ---------------------------------------------------------------------------
 * Beam search.  One step over a batch of utterances: ngpu_lm_beam_step selects
 * the best continuations of each utterance's hypotheses, ngpu_lm_kv_fork makes
 * their page tables from their parents' and gives them pages to write into, and
 * ngpu_lm_kv_copy (in each layer's cache) copies what two of them would
 * otherwise write into.  ngpu_lm_kv_compact moves a pool's used pages together.
 * ------------------------------------------------------------------------ */

/* Most hypotheses an utterance, before a step and after it. */
#define NGPU_LM_MAX_BEAMS 64

/* Strides in elements; rows of asr have unit stride and hold V classes, outside plain fusion V + 1. */
typedef struct {
    int64_t B;                     /* utterances */
    int32_t W, k;                  /* hypotheses before and after, 1..NGPU_LM_MAX_BEAMS each */
    int32_t mode;                  /* NGPU_FUSION_PLAIN, _TRANSDUCER or _AED */
    float lambda;
    const float *asr;              /* [B, W, classes]; a stride may be 0 (one frame for all hypotheses) */
    int64_t asr_stride_b, asr_stride_w;
    const int32_t *states;         /* [B, W] */
    const float *scores;           /* [B, W] sums so far; -inf (and NaN): no hypothesis, and its state is not looked at */
    const int32_t *last;           /* [B, W] last classes (AED): a hypothesis whose last is V has ended; NULL: none has */
    int32_t *out_tokens;           /* [B, k] class */
    int32_t *out_parents;          /* [B, k] place among the W */
    float *out_scores;             /* [B, k] */
    int32_t *out_states;           /* [B, k] */
} ngpu_beam_step_t;

/* Device memory a step needs, 16-byte aligned, not initialised; free again when the call's work has run. */
size_t ngpu_lm_beam_step_workspace(int64_t B, int32_t W, int32_t k);

/* The k continuations with the largest sums of each utterance, over all its
 * hypotheses w and classes c, in descending order:
 *   total[w][c] = scores[w] + fma(lambda, lm[w][c], asr[w][c]),
 * ties to the lowest w, then the lowest c.  lm is the query's score; class V is
 * <eos> in AED mode, with the state's final weight, and blank in transducer
 * mode, with lm = 0; it keeps the state.  A hypothesis that has ended continues
 * as itself alone (class V, score and state unchanged).  A NaN total counts as
 * -inf, and continuations at -inf are not selected: places that are left over
 * hold token -1, parent -1, score -inf and state 0.  A state outside [0,
 * num_states) of a hypothesis that is looked at gives no continuation and is
 * counted for ngpu_lm_check_states.  B = 0 is a no-op.  CTC needs prefixes to be merged and is refused. */
int ngpu_lm_beam_step(const ngpu_lm *lm, const ngpu_beam_step_t *args, void *d_workspace, size_t workspace_bytes,
                      void *hip_stream);

/* A pool of num_pages pages: refs[p] page tables hold page p, a page with 0 is free.
 * Each row of a page table holds one reference for each of its entries in [0, num_pages); other entries are empty. */
typedef struct {
    int64_t G;                     /* groups (utterances) */
    int64_t W, K;                  /* hypotheses of a group before (W) and after (K), at most NGPU_LM_MAX_FORK each */
    const int32_t *pages;          /* [G * W, width] page tables, row stride pages_stride */
    int64_t width, pages_stride;
    const int32_t *lengths;        /* [G * W] tokens, clamped to what the table holds */
    const int32_t *parents;        /* [G, K] place among the W; any other value: none */
    const int32_t *tokens;         /* [G, K] tokens that will be appended, negative ones count as 0, or NULL: T each */
    int64_t T;
    int32_t page_size;
    int64_t num_pages;
    int32_t *refs;                 /* [num_pages], updated */
    int32_t *out_pages;            /* [G * K, width] contiguous; must not overlap pages */
    int32_t *out_lengths;          /* [G * K] */
    int32_t *copies;               /* [G * K, 3] for ngpu_lm_kv_copy */
} ngpu_kv_fork_t;
#define NGPU_LM_MAX_FORK 4096
#define NGPU_LM_MAX_PAGES ((int64_t)1 << 28)

size_t ngpu_lm_kv_fork_workspace(int64_t G, int64_t K, int64_t num_pages);

/* Continuations take over their parents' tokens, and the old rows end.
 *  1. Row (g, j) gets the first ceil(lengths / page_size) entries of its parent's row, and -1 behind; refs go down by one
 *     for every entry of an old row (those behind its length too) and up by one for every entry of a new one.
 *  2. A row that will append (tokens > 0) and whose last page is filled in part takes a fresh page for it where others
 *     hold that page too: where refs, less the rows before it in its group that decided on that page, is above 1.
 *     copies[row] = {that page, the fresh one, entries that are filled}; for other rows {-1, -1, 0}.
 *  3. It takes fresh pages for the places of its new tokens behind.
 * Fresh pages are the free ones of after step 1, the lowest to the first row (its copy first), each with refs 1.  A row
 * whose pages, with those of the rows before, are not there, or whose tokens would not fit the table, is dropped: its
 * entries are given back and -1, its length -1, no copy; the caller has to end that hypothesis, as a later call takes a length
 * below 0 for 0.  out_lengths: the parent's (without the new tokens), 0 without parent.  The lengths are counted in tokens the table holds, so rejected tokens are given up by passing shorter ones.
 * Freeing is a fork without children: K = 0, or parents of -1.  A new sequence is a row of -1 entries and length 0 that
 * is forked with as many tokens as its prompt has.  G = 0 is a no-op. */
int ngpu_lm_kv_fork(const ngpu_kv_fork_t *args, void *d_workspace, size_t workspace_bytes, void *hip_stream);

/* For each of n rows {from, to, entries} of `copies`: entries [0, entries) of page `from` of the cache, keys and values,
 * are copied to page `to`; entries are clamped to the page, and rows with a page outside [0, num_pages) or from = to do
 * nothing.  No page may be the `to` of two rows, or one row's `to` and another's `from`. */
int ngpu_lm_kv_copy(const ngpu_kv_cache_t *cache, const int32_t *copies, int64_t n, void *hip_stream);

/* The same for a cache in 8 bits; all scales of the page are copied with the entries.  A stride of 0, and one array of scales
 * for keys and values, are taken; scales that overlap otherwise are refused. */
int ngpu_lm_kv_copy8(const ngpu_kv_cache8_t *cache, const int32_t *copies, int64_t n, void *hip_stream);

/* Device memory a compaction needs, 16-byte aligned, not initialised. */
size_t ngpu_lm_kv_compact_workspace(int64_t num_pages);

/* With n pages in use (refs other than 0), the i-th used page from n on moves to the i-th free one below n, in
 * ascending order: copies[i] = {from, to, page_size}, {-1, -1, 0} behind the last of the num_pages / 2 rows; moved[p] is
 * page p's new place (p itself where it stays or is free).  refs follow.  The tables are then to be put through
 * ngpu_lm_kv_move, the caches through ngpu_lm_kv_copy. */
int ngpu_lm_kv_compact(int32_t *refs, int64_t num_pages, int32_t page_size, int32_t *copies, int32_t *moved,
                       void *d_workspace, size_t workspace_bytes, void *hip_stream);

/* pages[r][i] = moved[pages[r][i]] for the entries in [0, num_pages) of a table [rows, width], row stride pages_stride
 * (at least width where rows > 1).  A second time changes nothing: each new place was free, and moved has it stay. */
int ngpu_lm_kv_move(int32_t *pages, int64_t rows, int64_t width, int64_t pages_stride, const int32_t *moved,
                    int64_t num_pages, void *hip_stream);

/* Synchronises hip_stream, then reports (and clears) how many out-of-range
 * input states the queries enqueued since the last check met.  Returns
 * NGPU_E_BAD_STATE when the count is non-zero. */
int ngpu_lm_check_states(const ngpu_lm *lm, void *hip_stream, int64_t *bad_count);

/* The same check without the count: synchronises hip_stream and returns
 * NGPU_E_BAD_STATE (clearing the count) when queries enqueued since the last
 * check met out-of-range input states, else NGPU_OK.  Every query kernel
 * performs the range check itself (one compare per hypothesis), so no build
 * flag enables it. */
int ngpu_lm_sync_check(const ngpu_lm *lm, void *hip_stream);

/* Algorithmic memory traffic of ngpu_lm_advance on host-side states h_states[B]:
 *   *hbm_bytes   = 8V (output row) + the state's chain record (16 bytes per
 *                  order, 16 for state 0) + 12 bytes per arc of each state of
 *                  order >= 2 on its backoff chain,
 *   *total_bytes = *hbm_bytes + 8V (the dense row of the order-1 ancestor, or
 *                  of the empty context),
 * summed over the batch.  The dense rows are shared by all hypotheses and
 * mostly served from the caches, hence the two figures.  Host-only. */
int ngpu_lm_query_bytes(const ngpu_lm *lm, const int32_t *h_states, int64_t B,
                        int64_t *hbm_bytes, int64_t *total_bytes);

/* Read-only view of the host copy of the trie image (the bytes that
 * ngpu_lm_upload copies), valid until ngpu_lm_free.  Its layout belongs to this
 * library build; it is exposed for saving an image and for white-box tests. */
int ngpu_lm_host_image(const ngpu_lm *lm, const void **data, size_t *bytes);

/* ARPA text (Section 2.1: "W context token B" lines, base-10 logarithms, as
 * KenLM writes them) parsed into an n-gram list for ngpu_lm_build.
 * vocab[0..V-1]: the scored vocabulary as words (NUL-terminated, distinct,
 * without <unk>, <s>, </s>); every other word of the file is an error
 * (NGPU_E_TOKEN_RANGE).  Weights become natural logarithms: x * ln 10 in
 * double, rounded once to fp32.  The <unk> unigram's weight is returned as
 * the <unk> weight; longer n-grams containing <unk> are dropped.  With
 * NGPU_BUILD_BOS_EOS, <s> and </s> become tokens V and V + 1; without it,
 * n-grams containing them are dropped (a closed file stays closed either
 * way).  The header's n-gram counts must match the file.  text need not be
 * NUL-terminated; it is read only during the call.  On success *out owns the
 * list (free with ngpu_arpa_free). */
typedef struct ngpu_arpa ngpu_arpa;
int ngpu_arpa_parse(const char *text, size_t len, const char *const *vocab, int32_t V, uint32_t flags,
                    ngpu_arpa **out);

/* The parsed list (arrays owned by a, valid until ngpu_arpa_free) and the
 * <unk> weight (NaN when the file has no <unk> unigram). */
int ngpu_arpa_list(const ngpu_arpa *a, ngpu_ngram_list *list, float *unk_logprob);

void ngpu_arpa_free(ngpu_arpa *a);

/* Message of the last failing call on this thread ("" if none). */
const char *ngpu_lm_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* NGPU_LM_H */
