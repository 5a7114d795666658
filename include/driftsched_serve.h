/*
 * driftsched_serve.h - C ABI of one decode step of a dispatched batch on AMD
 * Instinct MI355X (gfx950), beside the admission path of driftsched.h and in
 * the same library.
 *
 * The admission path decides which requests run (ds_order) and how many
 * tokens each is expected to hold (ds_score's budget). These calls run the
 * memory side of the step that follows, over a paged key-value cache:
 *
 *   ds_decode_attention  attention of the batch's new tokens over the cache,
 *                        and the weight every cached token received
 *   ds_cache_evict       requests that drifted past their budget keep the
 *                        tokens of the largest accumulated weight
 *   ds_verify_draft      drafted tokens against the target's probabilities;
 *                        the counts add to the observed output lengths that
 *                        ds_calibrate reads
 *
 * Everything stated in driftsched.h under "Conventions shared by every entry
 * point" holds here too: device arrays, host parameter structs, workspaces of
 * the caller, enqueueing on the caller's stream, status codes, DS_VALIDATE.
 * `rows` names the batch: rows[i] is the request of row i, e.g. the first
 * n_rows entries of a ds_order permutation; NULL: row i is request i. What a
 * call writes lies apart from what it reads, but where it says otherwise. A
 * workspace of 256 bytes is used by DS_VALIDATE only and may be NULL without
 * that flag.
 */
#ifndef DRIFTSCHED_SERVE_H
#define DRIFTSCHED_SERVE_H

#include "driftsched.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
typedef enum {
    DS_F32 = 0,
    DS_F16 = 1,
    DS_BF16 = 2,
    DS_E4M3 = 3             /* 8-bit float: 4 exponent, 3 mantissa bits, no infinities */
} ds_dtype;

#define DS_MAX_HEAD_DIM 256
#define DS_MAX_NEW_TOKENS 16
#define DS_MAX_QUERY_ROWS 1024   /* new tokens times query heads per key-value head */
#define DS_MAX_MASS_TOKENS (1u << 24)   /* visible tokens of a request whose weights are gathered */
#define DS_MAX_DRAFTS 63
#define DS_MAX_VOCAB (1u << 24)

/*
 * A paged key-value cache. Token j of request r lies in page
 * table[r * max_pages + j / page_size] at slot j % page_size; its key for
 * head h starts at element
 *     page * page_stride + slot * token_stride + h * head_stride
 * of k (its value: of v) and is head_dim elements long. Pages may be shared
 * between requests (each request reads them for itself); any order of the axes
 * page, slot and head fits.
 *
 *  k, v       device, 16-byte aligned; strides in elements, multiples of 16 bytes
 *  k_scale,   device, n_kv float, or NULL for ones; DS_E4M3 only (else NULL):
 *  v_scale      the values that the stored ones of head h are multiplied with
 *  table      device, n_requests * max_pages uint32; contract: entries that
 *             hold tokens are < n_pages
 *  len        device, n_requests uint32: cached tokens per request; contract:
 *             <= max_pages * page_size
 *  head_dim   a multiple of 8 (DS_E4M3: of 16), at most DS_MAX_HEAD_DIM
 *  type       DS_F16, DS_BF16 or DS_E4M3
 * n_requests, max_pages, n_pages, page_size, n_kv >= 1; max_pages * page_size
 * <= DS_MAX_ITEMS.
 * Tokens whose page is out of range are taken as absent. Pages are memory as a
 * whole: every slot of a page that holds a token may be read, and those of
 * page 0.
 */
typedef struct {
    void *k, *v;
    const float *k_scale, *v_scale;
    const uint32_t *table;
    uint32_t *len;
    uint32_t n_requests, max_pages, n_pages, page_size, n_kv, head_dim;
    uint64_t page_stride, token_stride, head_stride;
    ds_dtype type;
} ds_kv_cache;

/* Parameters of ds_decode_attention. */
typedef struct {
    uint32_t n_q;           /* query heads, a multiple of n_kv; head h reads head h / (n_q / n_kv) */
    uint32_t n_tokens;      /* new tokens per row, 1..DS_MAX_NEW_TOKENS, the same for every row of a call */
    ds_dtype q_type;        /* of q and out: DS_F16 or DS_BF16; the cache's own type unless that is DS_E4M3 */
    uint64_t q_row_stride, q_token_stride, q_head_stride;   /* elements, multiples of 8 */
    double scale;           /* of the products q.k; finite */
    uint32_t window;        /* tokens a query sees back, itself included; 0: all */
    uint32_t sinks;         /* first tokens that stay visible behind the window */
    uint32_t max_len;       /* contract: len <= max_len for the batch's requests; 0: max_pages * page_size.
                               Sizes the launch and the workspace, whatever the requests hold */
    uint64_t mass_len;      /* entries of mass per request and head, >= max_len; unused without mass */
} ds_decode_params;

/*
 * Attention of the last n_tokens tokens of each row's request over its cache
 * (their keys and values are in it already, and counted by len). With n =
 * len[r], query t of row i stands at position p = n - n_tokens + t and sees
 * the tokens j <= p with window == 0, j > p - window, or j < sinks:
 *     w_j = softmax_j(scale * q . k_j),   out = sum_j w_j v_j
 * A query that sees no token (p < 0 among them), or only scores of -inf,
 * gives zeros. What lies in masked places, NaN and infinities included, does
 * not reach the result.
 *
 * mass, if given, gathers the weight that each cached token received: for
 * token j of request r and head h, the sum of w_j over the row's queries of
 * head h's group is stored in mass[(r * n_kv + h) * mass_len + j] for the
 * n_tokens newest tokens, and added to what stands there for the others.
 * Nothing is written from entry n on. Rows with different numbers of new
 * tokens (drafts, say) therefore go in one call per number, each with its part
 * of the batch as `rows`: given more queries than it has new tokens, a row
 * would lose what its older tokens had gathered and count their queries again.
 *
 * Up to 1,024 rows a call splits long requests over the chip by the lengths of
 * the whole batch; with more, one workgroup per head takes all of a request.
 *
 * Scores, softmax and sums are held in 32 bits; the weights enter the second
 * product as two parts of q's type, which hold a weight to 2^-17 (bfloat16) or
 * 2^-22 (float16, and to 2^-40 of the query's largest weight), so that out is
 * rounded once, at the end. The same inputs give the same bits on every run.
 *
 *  q    device, q_type, element (i, t, h, d) at i * q_row_stride + t *
 *       q_token_stride + h * q_head_stride + d; 16-byte aligned
 *  out  device, q_type, n_rows * n_tokens * n_q * head_dim; written, and apart from q
 *  mass device, float, or NULL. With mass a request may stand in one row only
 *       (DS_VALIDATE checks it), and a query may see at most DS_MAX_MASS_TOKENS tokens (else DS_ERR_SIZE)
 *  ws   workspace of ds_decode_workspace_bytes(cache, params, n_rows, mass != NULL)
 */
ds_status ds_decode_attention(const ds_kv_cache *cache, const ds_decode_params *params,
                              uint32_t n_rows, const uint32_t *rows, const void *q, void *out,
                              float *mass, void *ws, size_t ws_bytes, uint32_t flags,
                              ds_stream stream);

/* Workspace of ds_decode_attention; 0 if it would refuse the structs. */
size_t ds_decode_workspace_bytes(const ds_kv_cache *cache, const ds_decode_params *params,
                                 uint32_t n_rows, int with_mass);

/* Parameters of ds_cache_evict. */
typedef struct {
    uint32_t sinks;         /* first tokens that always stay */
    uint32_t recent;        /* last tokens that always stay */
    uint32_t slack;         /* tokens a request may hold above its budget before it is cut */
    uint32_t max_len;       /* as in ds_decode_params; above 24,576 the workspace takes, per row and head,
                               8 KB for each 8,192 tokens (at most 2 MB) and 4 bytes for each that may be kept */
    uint64_t mass_len;      /* entries of mass and mass_out per request and head, >= max_len */
    uint64_t kept_len;      /* entries of kept per row and head */
} ds_evict_params;

/*
 * Cuts the requests that hold more tokens than their budget. For row i, its
 * request r, n = src->len[r] and keep = max(floor(budget[r]), sinks + recent):
 * if n > keep + slack, each head keeps its first `sinks` tokens, its last
 * `recent` ones, and of the others the keep - sinks - recent with the largest
 * mass (ties: the earlier token; NaN counts as less than any number). The
 * kept tokens' keys and values are copied, in their order, to the tokens 0 ..
 * keep-1 of row i of dst, and dst->len[i] = keep. Otherwise nothing is copied
 * and dst->len[i] = n. Pages of src are only read, so they may be shared
 * between requests; the pages that dst's table names for the rows that are
 * cut must be distinct and not among those that hold the batch's tokens. k and
 * v of dst may be those of src (one pool), and the caller then enters dst's
 * pages in the request's own table.
 *  dst->len may not overlap src->len (DS_ERR_ARG): the caller takes the new
 *  lengths over together with the pages.
 *
 *  src, dst   same page_size, n_kv, head_dim, type and strides; dst has one
 *             request per row (dst->n_requests >= n_rows) and len is written
 *  budget     device, n_requests double, e.g. from ds_score; NaN: not cut
 *  mass       device, n_requests * n_kv * mass_len float, as ds_decode_attention leaves it
 *  mass_out   device, like mass, mass itself or apart from it: its entries 0 .. keep-1
 *             receive the kept tokens' masses for the requests that are cut;
 *             nothing else is written
 *  kept       device, n_rows * n_kv * kept_len uint32: entries 0 .. keep-1 of
 *             the rows that are cut receive the kept tokens' indices; nothing
 *             else is written
 * A row whose keep exceeds kept_len or dst's max_pages * page_size is not cut
 * (DS_VALIDATE reports it). A request may stand in one row only.
 *  ws         workspace of ds_evict_workspace_bytes(src, dst, params, n_rows)
 */
ds_status ds_cache_evict(const ds_kv_cache *src, const ds_kv_cache *dst,
                         const ds_evict_params *params, uint32_t n_rows, const uint32_t *rows,
                         const double *budget, const float *mass, float *mass_out, uint32_t *kept,
                         void *ws, size_t ws_bytes, uint32_t flags, ds_stream stream);

/* Workspace of ds_cache_evict; 0 if it would refuse the structs. */
size_t ds_evict_workspace_bytes(const ds_kv_cache *src, const ds_kv_cache *dst,
                                const ds_evict_params *params, uint32_t n_rows);

/* Parameters of ds_verify_draft. */
typedef struct {
    uint32_t n_drafts;      /* drafted tokens per row at most, 0..DS_MAX_DRAFTS */
    uint32_t vocab;         /* 1..DS_MAX_VOCAB */
    uint32_t n_requests;    /* entries of observed and len */
    ds_dtype type;          /* of target and draft: DS_F32, DS_F16 or DS_BF16 */
    uint64_t target_row_stride, target_pos_stride;   /* elements */
    uint64_t draft_row_stride, draft_pos_stride;
} ds_verify_params;

/*
 * Verification of drafted tokens. Row i has m = n_draft[i] drafts x_0 ..
 * x_{m-1}; p_t is the target's distribution at position t (0 .. n_drafts),
 * q_t the one that draft t was drawn from. Draft t is accepted while
 *     u[i][t] * q_t(x_t) < p_t(x_t)
 * and with a the number of accepted drafts one more token is drawn: from
 * max(p_a - q_a, 0) if a < m (from p_a where that is zero everywhere), else
 * from p_a. The drawn token is the lowest j with sum_{i <= j} w_i > u_sample[i]
 * * sum_i w_i, in 64-bit arithmetic; entries that are not > 0 (NaN among them)
 * count as 0, and if rounding leaves no such j it is the last one with w_j > 0.
 * If every weight is 0 no token is drawn.
 *
 *  target     device, (n_rows, n_drafts + 1, vocab)
 *  draft      device, (n_rows, n_drafts, vocab), or NULL: the drafts were not
 *             drawn (q_t is 1 at x_t and 0 elsewhere)
 *  tokens     device, n_rows * n_drafts int32; contract: 0 <= x < vocab (others are rejected)
 *  n_draft    device, n_rows uint32 <= n_drafts, or NULL: n_drafts in every row
 *  u          device, n_rows * n_drafts float in [0, 1)
 *  u_sample   device, n_rows float in [0, 1)
 *  out        device, n_rows * (n_drafts + 1) int32: the accepted drafts, the
 *             drawn token, then -1
 *  n_emitted  device, n_rows uint32: tokens of the row before the -1s
 *  observed   device, n_requests uint32, or NULL: n_emitted[i] is added to
 *             observed[rows[i]], the output tokens ds_calibrate reads
 *  len        device, n_requests uint32, or NULL: the rejected drafts m - a
 *             are taken off len[rows[i]] (not below 0). With len a request may
 *             stand in one row only
 *  ws         workspace of ds_verify_workspace_bytes(params, n_rows)
 */
ds_status ds_verify_draft(const ds_verify_params *params, uint32_t n_rows, const uint32_t *rows,
                          const void *target, const void *draft, const int32_t *tokens,
                          const uint32_t *n_draft, const float *u, const float *u_sample,
                          int32_t *out, uint32_t *n_emitted, uint32_t *observed, uint32_t *len,
                          void *ws, size_t ws_bytes, uint32_t flags, ds_stream stream);

/* Workspace of ds_verify_draft; 0 if it would refuse the struct. */
size_t ds_verify_workspace_bytes(const ds_verify_params *params, uint32_t n_rows);

#ifdef __cplusplus
}
#endif

#endif /* DRIFTSCHED_SERVE_H */
