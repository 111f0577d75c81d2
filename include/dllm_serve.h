/*
 * dllm_serve.h - operators that serve a batch of requests of unequal lengths
 * over a paged K/V cache, under a prefix that all of them share.
 *
 * dllm.h decodes a batch in lockstep over one dense cache slice per sequence.
 * Here each request has its own number of cached and of new tokens (one, a
 * window, a prompt), its keys and values live in pages of a common pool, and a
 * long prompt in front of all of them is stored, and read, once.  A step is
 *   dllm_serve_plan          pages, slots and positions from the lengths
 *   then, in every layer,
 *   dllm_serve_qk_norm_rope  q and k normalised and rotated, k and v stored
 *   dllm_serve_attention     attention over the prefix and the own pages
 *   and at its end
 *   dllm_serve_logits        penalties, biases, grammar, and the decision.
 *
 * Conventions: those of dllm.h for return codes, error messages
 * (dllm_last_error(NULL)) and pointers, with these differences.  Every call is
 * asynchronous on the caller's stream, allocates nothing, and can be captured
 * in a CUDA graph.  Device memory, workspaces included, is the caller's; the
 * buffers of one dllm_serve_tables are for one stream at a time.  What a kernel
 * finds wrong (lengths, a pool that ran out, a wait that ran out) it records in
 * the tables' status words, which dllm_serve_check reads: no such case writes
 * outside the buffers or disturbs the other requests.  Device pointers that a
 * call takes as arrays of 16-bit values are 16-byte aligned, their strides (in
 * elements) multiples of 8; those of 32-bit values are 4-byte aligned; what
 * differs is said at the call.  Other ones are refused.
 */
#ifndef DLLM_SERVE_H
#define DLLM_SERVE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { DLLM_BF16 = 0, DLLM_F16 = 1, DLLM_F32 = 2 };

/* Limits and shapes.  The cache of a layer is two arrays kc and vc of dtype
 * [n_pages][n_kv_heads][page][head_dim], page_stride elements from page to
 * page.  Slot s of the pool is place s % page of page s / page.
 * Constraints: max_batch <= 4096; page one of 16, 32, 64, 128, 256;
 * n_pages * page < 2^31; max_pages * page < 2^31; max_rows <= 2^22;
 * head_dim 64 or 128; n_heads <= 65536; n_kv_heads divides n_heads,
 * n_heads / n_kv_heads <= 128;
 * dtype DLLM_BF16 or DLLM_F16. */
typedef struct {
    int max_batch;  /* requests */
    int max_rows;   /* new tokens of a step, all requests together */
    int page;       /* positions of a page */
    int n_pages;    /* pages of the pool */
    int max_pages;  /* pages that one request may hold */
    int n_heads, n_kv_heads, head_dim;
    int dtype;             /* of q, kc, vc and the attention's output */
    int64_t page_stride;   /* 0: n_kv_heads * page * head_dim */
} dllm_serve_config;

/* Device buffers, carved by dllm_serve_layout from one piece of memory.  The
 * first four are the state of the pool, kept from step to step; a program may
 * read all of them, and write the state between steps (a page belongs to one
 * request's row of table, to the ring, or to the program). */
typedef struct {
    int32_t* table;      /* [max_batch][max_pages]: pages of a request in order; past held: -1 */
    int32_t* held;       /* [max_batch]: pages that a request holds */
    int32_t* ring;       /* [n_pages]: free pages, oldest first, from ring_pos[0] on (cyclic) */
    int32_t* ring_pos;   /* [2]: place of the oldest free page, number of free pages */
    int32_t* row_start;  /* [max_batch + 1]: first row of a request in the step's packed rows */
    int32_t* n_keys;     /* [max_batch]: own keys after the step (0: refused) */
    int32_t* slot;       /* [max_rows]: where a row's key and value go (-1: nowhere) */
    int32_t* pos;        /* [max_rows]: its position */
    int32_t* req;        /* [max_rows]: its request (-1: padding) */
    int32_t* status;     /* [4]: DLLM_SERVE_* bits; requests refused, pages taken and given back by the last plan */
    int32_t* work;       /* the attention's work list (opaque) */
    float* partials;     /* the attention's workspace (opaque) */
} dllm_serve_tables;

/* Bits of status[0], kept until dllm_serve_check. */
enum {
    DLLM_SERVE_TIMEOUT = 1,   /* a bounded wait ran out: outputs are not valid */
    DLLM_SERVE_LENGTHS = 2,   /* a negative length, more pages than max_pages, or more than 2^31 - 1 positions with
                               * the prefix: request refused */
    DLLM_SERVE_PAGES = 4,     /* the pool ran out: request refused */
    DLLM_SERVE_ROWS = 8,      /* the new tokens are more than the plan's rows: the last ones are left out */
    DLLM_SERVE_PREFIX = 16,   /* fewer prefix pages than the plan's prefix_len needs, or one outside the pool */
    DLLM_SERVE_SLOT = 32,     /* a slot outside the pool: its row was not stored */
    DLLM_SERVE_STATE = 64     /* table, held or ring_pos are not what a plan leaves (request refused, or its keys read
                               * as zeros), or an attention after another config's plan (zeros, as after a reset and
                               * no plan, which sets no bit) */
};

/* Bytes of the buffers for cfg (bytes nullable) and, with mem (16-byte aligned
 * device memory of so many bytes), the pointers into it (out nullable). */
int dllm_serve_layout(const dllm_serve_config* cfg, void* mem, dllm_serve_tables* out, size_t* bytes);

/* Nothing held, every page free (in ascending order), status clear, no plan. */
int dllm_serve_reset(const dllm_serve_config* cfg, const dllm_serve_tables* t, void* stream);

/* The step's plan.  Request b < batch has len[b] own positions cached (after
 * the shared prefix) and q_len[b] new tokens (both dev int32 [batch], apart from
 * the tables but for len, which may be their n_keys: what the last plan left); it
 * needs ceil((len + q_len) / page) pages.  Those it holds beyond that go to the
 * ring's end, in order of requests and pages; those it lacks come from the ring's
 * front in order of requests, so a page given back is handed out again at the
 * next plan at the earliest.  len = q_len = 0 ends a request.  A request whose
 * lengths are wrong, or that needs pages when the needs of the requests up to
 * it pass what was free, is refused: it keeps what it held, its rows get slot
 * -1 and position 0 and its n_keys is 0.
 * New tokens are packed, request after request: row_start[b] .. row_start[b + 1].
 * rows (<= max_rows): the rows of the step's arrays; rows past the last new
 * token are padding (slot -1, position 0, request -1).  Token t of request b has
 * position prefix_len + len[b] + t and slot table[b][(len[b] + t) / page] * page
 * + (len[b] + t) % page.
 * The plan also cuts the attention's work, for a prefix of prefix_len positions
 * and, with causal != 0, own keys only up to a row's own position (else all
 * n_keys of its request: a window's rows see one another, Sec. 2.1). */
int dllm_serve_plan(const dllm_serve_config* cfg, const dllm_serve_tables* t, const int32_t* len,
                    const int32_t* q_len, int batch, int rows, int prefix_len, int causal, void* stream);

/* Queries and keys of rows 0 .. rows - 1: RMSNorm of each head,
 * y = x * rsqrt(mean(x^2) + eps) * gain (gain dev fp32 [head_dim], 16-byte
 * aligned, null: ones; the norm itself is always applied),
 * then rotate-half RoPE: features j and j + head_dim / 2 turned by
 * pos[row] * theta[j] (theta dev fp32 [head_dim / 2]).  q, k, v dev of in_dtype
 * (the config's dtype, or DLLM_F32): row r at r * ldq, r * ldk, r * ldv
 * elements, heads one after another.  q goes to q_out [rows][n_heads][head_dim]
 * (ld_out elements from row to row), k and v to their slots in kc and vc; a row
 * of slot -1 is not stored.  q_out may be q itself (same type and stride).
 * rows: no more than the plan's (slots past them are an earlier plan's). */
int dllm_serve_qk_norm_rope(const dllm_serve_config* cfg, const dllm_serve_tables* t, const void* q, const void* k,
                            const void* v, int in_dtype, int64_t ldq, int64_t ldk, int64_t ldv, const float* q_gain,
                            const float* k_gain, float eps, const float* theta, void* q_out, int64_t ld_out, void* kc,
                            void* vc, int rows, void* stream);

/* Attention of the plan's rows: softmax(scale * q k^T) v over the plan's
 * prefix_len prefix positions (pages prefix_pages dev int32 [n_prefix], in
 * order, of the same pool) and the own keys that the row sees.  Query head h
 * reads K/V head h / (n_heads / n_kv_heads).  q row r at r * ldq, out
 * [rows][n_heads * head_dim], 32-byte aligned; lse dev fp32 [rows][n_heads], nullable: the
 * natural logarithm of the row's softmax sum.  A row that sees no key, and
 * padding, gives zeros (lse -inf).  Keys and values past a request's n_keys,
 * or past the prefix, may hold anything, infinities and NaN included; so may
 * those that a row does not see, for that row.
 * rows: those of the plan.  scale > 0.  Scores, sums and out's accumulation
 * are fp32; the softmax's weights are rounded to dtype before the product with
 * v (out's error is 1.4 times that of an fp32 softmax rounded once). */
int dllm_serve_attention(const dllm_serve_config* cfg, const dllm_serve_tables* t, const void* q, int64_t ldq,
                         const void* kc, const void* vc, const int32_t* prefix_pages, int n_prefix, float scale,
                         void* out, float* lse, int rows, void* stream);

/* Waits for the stream, clears status[0] and reports it: DLLM_OK,
 * DLLM_ETIMEOUT, DLLM_ECAPACITY (DLLM_SERVE_PAGES) or DLLM_EINVAL (the other
 * bits).  bits: status[0], nullable. */
int dllm_serve_check(const dllm_serve_tables* t, int* bits, void* stream);

/* Logits of rows 0 .. rows - 1 and the decision from them.  Row n belongs to
 * request r = req[n] (null: r = n; negative: none, no penalties and biases).
 * For each id v, with c = how often v stands in hist[r][0 .. hist_len[r]):
 *   c > 0:  z = (z > 0 ? z / rep[r] : z * rep[r]) - (freq[r] * c + pres[r])
 *   v among bias_ids[r][0 .. bias_len[r]):  z = z + bias[r][i] (of several the last i)
 *   grammar_row[n] = g >= 0 and bit v % 32 of grammar[g][v / 32] clear, or g >= n_grammar:  z = -inf
 * in fp32, in this order, each operation rounded on its own.  out: z, rounded to
 * dtype (nullable; may be logits itself).  The decision, as dllm_op_lmhead: x0 =
 * argmax without mask_id (ties: lowest id; -1: every id is -inf), conf =
 * softmax(z)[x0], tokconf = softmax(z)[cur[n]] (0 when cur is mask_id or no
 * id), both over all ids but mask_id.  A NaN that no mask hides is passed over
 * by x0 and makes conf and tokconf NaN. */
typedef struct {
    const void* logits;   /* dev dtype [rows][ld] */
    void* out;            /* dev dtype [rows][ld_out], or null */
    int64_t ld, ld_out;   /* elements, >= vocab (any alignment) */
    int dtype;            /* DLLM_F32, DLLM_BF16 or DLLM_F16 */
    int rows, vocab;
    int mask_id;          /* -1: none */
    int n_req;            /* rows of the arrays per request */
    const int32_t* req;   /* dev [rows], nullable */
    const int32_t* hist;  /* dev [n_req][hist_ld], nullable: no penalties; ids outside the vocabulary are skipped */
    const int32_t* hist_len; /* dev [n_req] (null: hist_ld) */
    int hist_ld;          /* < 2^20 */
    const float *rep, *freq, *pres; /* dev [n_req]; null: 1, 0, 0 */
    const int32_t* bias_ids; /* dev [n_req][bias_ld], nullable */
    const float* bias;       /* dev [n_req][bias_ld] */
    const int32_t* bias_len; /* dev [n_req] (null: bias_ld) */
    int bias_ld;             /* < 4096 */
    const uint32_t* grammar; /* dev [n_grammar][(vocab + 31) / 32], nullable */
    const int32_t* grammar_row; /* dev [rows] */
    int n_grammar;
    const int32_t* cur;      /* dev int32 [rows], nullable: tokconf is not written */
    int32_t* x0;             /* dev [rows], nullable, and so are conf and tokconf */
    float *conf, *tokconf;
    void* ws;                /* dev, 16-byte aligned, dllm_serve_logits_bytes */
    size_t ws_bytes;
} dllm_serve_logits_args;

int dllm_serve_logits_bytes(int rows, int vocab, size_t* bytes);
int dllm_serve_logits(const dllm_serve_logits_args* a, void* stream);

#ifdef __cplusplus
}
#endif
#endif
