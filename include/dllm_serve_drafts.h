/*
 * dllm_serve_drafts.h - operators for decoding from drafts and with several
 * continuations, next to those of dllm_serve.h and on its tables.
 *
 * A step that checks drafts takes for every request a tree of new tokens: the
 * token it decided on last and, behind it, drafts of what follows, several for
 * one place where there are several guesses.  After dllm_serve_plan (not
 * causal, or causal for trees whose tokens see none behind them):
 *   dllm_serve_tree            who sees whom, and positions, from the parents
 *   in every layer
 *   dllm_serve_qk_norm_rope    at the tree's positions
 *   dllm_serve_tree_attention  attention by the bits of dllm_serve_tree
 *   and at the end
 *   dllm_serve_logits          the decisions (and dllm_serve_logprobs)
 *   dllm_serve_accept          the path of the tree that they bear out
 *   dllm_serve_compact         its keys and values, side by side in all layers
 * The next plan's lengths are those before plus the path's.  Between steps
 * dllm_serve_fork lets requests continue others (beams, samples of one
 * prompt): full pages are shared, not copied.
 *
 * Conventions: those of dllm_serve.h.
 */
#ifndef DLLM_SERVE_DRAFTS_H
#define DLLM_SERVE_DRAFTS_H

#include "dllm_serve.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Further bits of dllm_serve_tables.status[0]. */
enum {
    DLLM_SERVE_TREE = 128,  /* a parent that is not an earlier token of its request, a tree of more tokens than its rows
                             * have bits, or kept places that do not ascend or are not there: request left out */
    DLLM_SERVE_SHARED = 256 /* a plan that would give back or write to a page that requests share, or a compaction that
                             * would write to one: request refused */
};

/* Bits and positions of the plan's new tokens.  parent (dev int32 [rows], rows
 * those of the plan) numbers the tokens of each request from 0: parent[row] is
 * the token that this one follows, an earlier one of the same request, or -1:
 * it follows the cached ones.  Token t sees itself and all that it follows:
 * bit j % 32 of mask[row][j / 32] (dev uint32 [rows][words]) says whether it
 * sees token j.  The tables' pos of a row becomes the request's first position
 * plus the number of tokens that this one follows.  A request whose tree is
 * wrong, or has more than 32 * words tokens, keeps the plan's positions; its
 * bits, and those of padding, are 0.  words 1 to 1024 (a token walks to its
 * root: a chain of 32768 takes 0.2 s). */
int dllm_serve_tree(const dllm_serve_config* cfg, const dllm_serve_tables* t, const int32_t* parent, uint32_t* mask, int words,
                    int rows, void* stream);

/* dllm_serve_attention with bits: a row sees the prefix, the keys of its
 * request that were cached before the plan, and of the request's new tokens
 * those whose bit of mask[row] (dev uint32 [rows][words]) is set; tokens past
 * the row's bits it does not see, and bits past the request's tokens say
 * nothing.  After a causal plan it sees of these only those up to itself.
 * words 1 to 2^16.  As there, the softmax's weights are rounded to dtype before
 * the product with v: out is 0.0023 off 64 bits in bf16, 0.0017 for an fp32
 * softmax rounded once (f16: 2.7e-4, 2.1e-4). */
int dllm_serve_tree_attention(const dllm_serve_config* cfg, const dllm_serve_tables* t, const void* q, int64_t ldq,
                              const void* kc, const void* vc, const int32_t* prefix_pages, int n_prefix, float scale,
                              const uint32_t* mask, int words, void* out, float* lse, int rows, void* stream);

/* The path of each request's tree that the decisions bear out.  parent as
 * above, ids (dev int32 [rows]) the tokens, x0 (dev int32 [rows]) what follows
 * each of them as decided.  The path begins at token 0 and goes on to the first
 * later token that follows its last one and whose id is the last one's x0, up to
 * max_len tokens.  keep[b][0 .. n[b]) (dev int32 [batch][max_len]): the path's
 * tokens, then -1; next[b]: x0 of its last token.  A request without new
 * tokens, one that the plan has refused, and one whose tree dllm_serve_tree has
 * found wrong since the plan have no path: n = 0, next -1 (so that the lengths
 * that follow count no position that was not written).  batch: the plan's; rows
 * past it have none. */
int dllm_serve_accept(const dllm_serve_config* cfg, const dllm_serve_tables* t, const int32_t* parent, const int32_t* ids,
                      const int32_t* x0, int batch, int rows, int max_len, int32_t* keep, int32_t* n, int32_t* next,
                      void* stream);

/* Keys and values moved together: own position first[b] + keep[b][i] of request
 * b < batch goes to first[b] + i, for i < n[b] (keep dev int32 [batch][keep_ld];
 * first, n dev int32 [batch]), in the n_layers caches kc[i], vc[i] (host arrays
 * of device pointers, n_layers 1 to 128, all different).  keep ascends, so that
 * places only move down; a list that does not, that names places which the
 * request does not hold, or that would write to pages which others share, leaves
 * its caches as they were.  Lengths and pages stay: the next plan's len says what is left.
 * (Paths belong into rows of up to 128: wider ones are taken for long lists.) */
int dllm_serve_compact(const dllm_serve_config* cfg, const dllm_serve_tables* t, void* const* kc, void* const* vc, int n_layers,
                       const int32_t* first, const int32_t* keep, int keep_ld, const int32_t* n, int batch, void* stream);

/* Requests continue others: request b < batch holds what src[b] (of any of the
 * max_batch requests; itself to stay, or to be cut) held up to len[b] own
 * positions (both dev int32 [batch]); len[b] = 0 ends it.  Full pages become
 * pages of several requests.  The last, partly filled page is copied, in the
 * n_layers caches kc[i], vc[i] (as above), to a page from the ring's front,
 * unless nobody else is left to hold it; the first of several requests that
 * continue on the same page keeps it.  Copies take pages in order of requests;
 * pages that nobody holds any more go to the ring's end in ascending order, so
 * that a page given back is handed out again at the next plan or fork at the
 * earliest.  n_keys[b] becomes len[b].  status[1 .. 3] as after a plan.  The
 * last plan's rows and work list stay: a plan comes before the next attention.
 * The call is carried out whole or not at all: where a src or a len is wrong
 * (DLLM_SERVE_LENGTHS), or the copies are more than the free pages
 * (DLLM_SERVE_PAGES), tables and caches stay as they were and status[1] is batch.
 * What requests share is in the tables' shared, which each fork makes anew from
 * all rows (one of requests onto themselves, at their own lengths, serves to do
 * that alone).  While a page is shared, a plan refuses (DLLM_SERVE_SHARED) to
 * give it back or to write to it: requests that share pages are ended, or cut by
 * more than their last page, by a fork. */
int dllm_serve_fork(const dllm_serve_config* cfg, const dllm_serve_tables* t, void* const* kc, void* const* vc, int n_layers,
                    const int32_t* src, const int32_t* len, int batch, void* stream);

/* Log probabilities under softmax(logits) over all ids but mask_id, natural
 * logarithms, from logits of one read.  With m the largest logit (NaN passed
 * over) and O the sum of exp(z - m) over all ids but one that has it:
 *   lse     = m + log1p(O)
 *   entropy = log1p(O) - sum exp(z - m) (z - m) / (1 + O)
 *   lp      = (z - m) - log1p(O) for tokens[row][i]; -inf for ids outside the
 *             vocabulary and for mask_id
 *   top_ids, top_lp: the n_top largest logits in descending order (ties: lowest
 *             id), without NaN and -inf; past them id -1, -inf
 * so that peaked rows keep their digits (exponentials below 2^-126 are 0).  A
 * row of nothing but -inf: lse -inf, entropy 0, lp -inf.  A NaN (not mask_id's)
 * makes the row's lse, lp and entropy NaN; logits of +inf make lse +inf, entropy
 * NaN, lp NaN for those ids and -inf for the others.  Rows that begin at 16
 * bytes (logits, and ld a multiple of 8 values, of 4 for DLLM_F32) take half to
 * a third of the time of others. */
typedef struct {
    const void* logits;    /* dev dtype [rows][ld] */
    int64_t ld;            /* elements, >= vocab */
    int dtype;             /* DLLM_F32, DLLM_BF16 or DLLM_F16 */
    int rows, vocab;       /* vocab <= 2^28 */
    int mask_id;           /* -1: none */
    const int32_t* tokens; /* dev [rows][n_tokens] */
    int n_tokens;          /* 0 to 2^20 */
    int n_top;             /* 0 to 32 */
    float* lp;             /* dev [rows][n_tokens] (with n_tokens) */
    float* entropy;        /* dev [rows], nullable, and so is lse */
    float* lse;
    int32_t* top_ids;      /* dev [rows][n_top] (with n_top) */
    float* top_lp;
} dllm_serve_logprobs_args;

int dllm_serve_logprobs(const dllm_serve_logprobs_args* a, void* stream);

#ifdef __cplusplus
}
#endif
#endif
