/*
 * toktier_model.h — C ABI of the operators that stand next to the tokenizer,
 * on both sides of a model: the plan of a step's tokens (what a model needs
 * besides the IDs of tt_encode_batch and of session appends) and the scores of
 * given tokens (what comes back from the model about them).
 *
 * Conventions
 *  - Those of toktier.h: int64_t sizes, int32_t token IDs, TT_OK or a negative
 *    TT_ERR_* code, `stream` a hipStream_t as void*.
 *  - Every pointer is HIP device memory of the current device, which is also
 *    the stream's.  The calls only enqueue work on `stream`: they allocate
 *    nothing, keep nothing between calls and do not synchronise, so that they
 *    may be captured into a graph and replayed on new contents.
 *  - Arguments that the host can see are checked before anything is enqueued.
 *    A call that returns an error has written nothing.
 *  - Outputs must not overlap inputs, except where stated.
 *  - A workspace is the caller's memory, aligned to 256 bytes, of at least the
 *    size that the matching *_workspace function gives; its contents mean
 *    nothing before and after a call.  Calls that share one must be ordered.
 *  - Rows and columns count elements; a stride is the distance between the
 *    first elements of two rows, at least the row's length.  Rows need no
 *    alignment beyond their element's.
 *  - Results do not depend on timing: nothing is summed in an order that
 *    varies between calls.
 */
#ifndef TOKTIER_MODEL_H
#define TOKTIER_MODEL_H

#include "toktier.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The current device of the calling thread, on which the calls below enqueue;
 * TT_ERR_HIP if there is none. */
int32_t tt_current_device(void);

/* ---- plan of a step -------------------------------------------------------- */
/* One step of a server with a paged cache: request r has cached[r] tokens in
 * the cache and brings fresh[r] new ones (either may be 0).  The new tokens of
 * all requests stand one after the other, request 0's first: token t of
 * request r, with i = t - offsets[r], gets
 *   position  cached[r] + i
 *   slot      page * page_size + position % page_size, where page is entry
 *             position / page_size of the request's table
 *   target    ids[t + 1], or -1 for the request's last token
 * and a request whose pages do not hold cached[r] + fresh[r] tokens gets more
 * from the top of the stack of free pages, in order of requests.
 *
 * A session that repairs its tail (tt_session_append) has cached = info.kept
 * and may hold more pages than its kept tokens fill: held[] says how many.
 *
 * All arrays are device memory; result reports errors that only the device can
 * see.  The free list and its count are read, not changed: a caller that goes
 * on uses result[1] as the next count. */
typedef struct {
  int32_t n_requests;
  int32_t page_size;            /* tokens of a page, at least 1                              */
  int32_t table_width;          /* entries of a table that may be used                       */
  int64_t table_stride;
  int64_t max_tokens;           /* entries of the per-token arrays, below 2^31               */
  int64_t n_free;               /* entries of free_pages, below 2^31                         */
  /* inputs */
  const int32_t* cached;        /* [n_requests]                                              */
  const int32_t* fresh;         /* [n_requests]                                              */
  const int32_t* held;          /* [n_requests] pages in each table; NULL: cached tokens'    */
  const int32_t* ids;           /* [max_tokens] the new tokens; NULL with targets            */
  const int32_t* free_pages;    /* [n_free] stack of free page numbers, the top last         */
  const int64_t* free_count;    /* [1] entries on the stack, at most n_free                  */
  /* updated in place */
  int32_t* tables;              /* [n_requests][table_stride]: new pages are added           */
  /* outputs */
  int32_t* offsets;             /* [n_requests + 1] first token of each request              */
  int32_t* lengths;             /* [n_requests] cached + fresh                               */
  int32_t* pages;               /* [n_requests] pages held after the step                    */
  int64_t* slots;               /* [max_tokens]; -1 past the last token                      */
  int32_t* positions;           /* [max_tokens];  0 past the last token                      */
  int32_t* requests;            /* [max_tokens] request of each token; -1 past the last      */
  int32_t* targets;             /* [max_tokens]; -1 past the last token; NULL with ids       */
  int64_t* result;              /* [2]: number of tokens, free pages left                    */
} tt_step;

/* result[0] is negative where the device found an error; the tables are then
 * unchanged, result[1] is *free_count, offsets and lengths are 0, pages is what
 * was held and the per-token arrays hold what they hold past the last token:
 *  TT_ERR_BAD_ARG  a negative length, a request that needs (or holds) more than
 *                  table_width pages or 2^31 tokens, more new tokens than
 *                  max_tokens, a count outside [0, n_free];
 *  TT_ERR_OOM      fewer free pages than the step needs. */
int tt_step_plan(const tt_step* step, void* stream);

/* ---- scores of given tokens ------------------------------------------------ */
/* Element types of the tensors. */
enum { TT_F32 = 0, TT_BF16 = 1, TT_F16 = 2 };

/* The most alternatives of a row. */
#define TT_MAX_ALTERNATIVES 64

/* With x = scale * logits[row], m the largest x / scale, s the sum of
 * exp(x - scale * m), t = targets[row]:
 *   logprobs[row]   x_t - scale * m - log s; 0 where t is negative (no token is
 *                   given: the end of a document), NaN where t >= vocab
 *   stats[row]      {m, log s}: what the gradient needs
 *   entropy[row]    -sum p log p, p = exp(x - scale * m) / s
 *   alternatives    the n_alt largest logits, the lowest ID first among equal
 *                   ones, and their log probabilities, in descending order
 * A logit of -inf has probability 0 and is no alternative; places without one
 * get ID -1 and -inf.  A row of nothing but -inf has no distribution: logprob
 * -inf (0 where no token is given), stats {-inf, -inf}, entropy 0, no
 * alternatives, gradient 0.  A row with a NaN or +inf has NaN for all of these
 * (ID -1), its whole gradient included.
 * log s comes from the sum of the other entries next to the largest one: where a
 * row is nearly sure of a token, log s, the token's log probability and the
 * entropy are good to some 2^-17 of their own small values (the error of logits
 * from hidden states included), and with them the token's gradient.
 * Sums are kept in 32 bits; scale is a positive number (1 / temperature). */

/* Workspace of tt_token_scores in bytes, or a negative error code. */
int64_t tt_token_scores_workspace(int64_t rows, int64_t vocab, int32_t n_alt);

/* Scores from stored logits [rows][vocab] (any of the three types).
 *  targets        [rows]; NULL: no token is given anywhere
 *  logprobs, entropy  [rows] float; stats [rows][2] float; each may be NULL
 *  alt_ids, alt_logprobs  [rows][n_alt]; NULL where n_alt is 0 */
int tt_token_scores(const void* logits, int32_t type, int64_t rows, int64_t vocab, int64_t stride, float scale,
                    const int32_t* targets, float* logprobs, float* stats, float* entropy, int32_t n_alt,
                    int32_t* alt_ids, float* alt_logprobs, void* workspace, int64_t workspace_bytes, void* stream);

/* Gradient with respect to the logits, of any function of the log
 * probabilities and entropies (the alternatives pass none on):
 *   grad_logits_j = scale * (g_l ([j = t] - p_j) - g_e p_j (log p_j + entropy))
 * with g_l = grad_logprobs[row] (0 where no token is given) and
 * g_e = grad_entropy[row]; either array may be NULL (zeros).  Rounded once, to
 * the type of the logits.  grad_logits may be the logits themselves (same
 * stride).  stats and entropy are those of tt_token_scores (entropy may be NULL
 * with grad_entropy).  A row whose g_l and g_e are both 0 gets zeros. */
int tt_token_scores_grad(const void* logits, int32_t type, int64_t rows, int64_t vocab, int64_t stride, float scale,
                         const int32_t* targets, const float* stats, const float* entropy,
                         const float* grad_logprobs, const float* grad_entropy, void* grad_logits,
                         int64_t grad_stride, void* stream);

/* The same scores of logits = hidden weight^T that are never stored:
 * hidden [rows][width], weight [vocab][width], both TT_BF16 or both TT_F16;
 * products are summed in 32 bits and the logits are not rounded. */
int64_t tt_head_scores_workspace(int64_t rows, int64_t vocab, int64_t width);
int tt_head_scores(const void* hidden, int64_t hidden_stride, const void* weight, int64_t weight_stride, int32_t type,
                   int64_t rows, int64_t vocab, int64_t width, float scale, const int32_t* targets, float* logprobs,
                   float* stats, float* entropy, void* workspace, int64_t workspace_bytes, void* stream);

/* Gradients with respect to hidden and weight (either may be NULL: not
 * wanted), rounded once to their type.  The logits are computed again; the
 * gradient with respect to them is rounded to the type of hidden before it is
 * multiplied by weight and hidden, and those products are summed in 32 bits.  It
 * is scaled before that, so that a gradient that many rows share is not rounded;
 * for TT_F16 the largest possible value of all rows comes to 2^12 to 2^13: entries
 * below 2^-27 of it lose bits, below 2^-38 they are 0.  For up to 256 rows what the
 * rounding takes off is kept too and multiplied with the rest: the results' error
 * is then their own rounding, and with more rows some 1.4 times that in the norm.
 *   grad_hidden = G weight, grad_weight = G^T hidden, G as in
 *   tt_token_scores_grad.
 * The workspace function gives the least size, which works through the
 * vocabulary in pieces of 256 entries, or with `ample` the size up to which
 * more room helps; any size between is used. */
int64_t tt_head_scores_grad_workspace(int64_t rows, int64_t vocab, int64_t width, int32_t ample);
int tt_head_scores_grad(const void* hidden, int64_t hidden_stride, const void* weight, int64_t weight_stride,
                        int32_t type, int64_t rows, int64_t vocab, int64_t width, float scale,
                        const int32_t* targets, const float* stats, const float* entropy,
                        const float* grad_logprobs, const float* grad_entropy, void* grad_hidden,
                        int64_t grad_hidden_stride, void* grad_weight, int64_t grad_weight_stride, void* workspace,
                        int64_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* TOKTIER_MODEL_H */
