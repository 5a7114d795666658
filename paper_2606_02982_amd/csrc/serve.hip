// C ABI of the decode step (driftsched_serve.h): argument checks, workspace
// carving and kernel launches on the caller's stream.
#include <math.h>

#include "apiutil.h"
#include "serve.h"

using namespace ds;

namespace {

// workgroups of a launch: its threads are counted in 32 bits
constexpr uint64_t kMaxGrid = 0xFFFFFFFFull / 256, kMaxGrid1024 = 0xFFFFFFFFull / 1024;
constexpr uint32_t kMaxTokens = DS_MAX_ITEMS;   // of a request; windows and sinks beyond act like it

uint32_t clamp32(uint32_t x, uint32_t most) { return x < most ? x : most; }

// The structs' own checks; the pointers' come with the call.
ds_status view_of(const ds_kv_cache *c, uint32_t max_len, KvView &v)
{
    if (!c) return DS_ERR_NULL;
    const int type = enum_int(c->type);
    if (type != DS_F16 && type != DS_BF16 && type != DS_E4M3) return DS_ERR_ARG;
    const uint32_t unit = type == DS_E4M3 ? 16 : 8;      // elements of 16 bytes
    if (!c->n_requests || !c->max_pages || !c->n_pages || !c->page_size || !c->n_kv || !c->head_dim) return DS_ERR_ARG;
    if (c->head_dim % unit || c->head_dim > DS_MAX_HEAD_DIM) return DS_ERR_ARG;
    if (c->page_stride % unit || c->token_stride % unit || c->head_stride % unit) return DS_ERR_ALIGN;
    if (type != DS_E4M3 && (c->k_scale || c->v_scale)) return DS_ERR_ARG;
    const uint64_t cap = (uint64_t)c->max_pages * c->page_size;
    if (cap > kMaxTokens || c->n_kv > 65536) return DS_ERR_SIZE;
    if (max_len > cap) return DS_ERR_ARG;
    v.k = static_cast<uint8_t *>(c->k);
    v.v = static_cast<uint8_t *>(c->v);
    v.k_scale = c->k_scale;
    v.v_scale = c->v_scale;
    v.table = c->table;
    v.len = c->len;
    v.n_requests = c->n_requests;
    v.max_pages = c->max_pages;
    v.n_pages = c->n_pages;
    v.page_size = c->page_size;
    v.n_kv = c->n_kv;
    v.dim = c->head_dim;
    v.cap = max_len ? max_len : (uint32_t)cap;
    v.page_stride = c->page_stride;
    v.token_stride = c->token_stride;
    v.head_stride = c->head_stride;
    v.type = type;
    v.page_shift = c->page_size & (c->page_size - 1) ? -1 : __builtin_ctz(c->page_size);
    return DS_OK;
}

ds_status pointers_of(const KvView &v)
{
    if (!v.k || !v.v || !v.table || !v.len) return DS_ERR_NULL;
    if (!aligned(v.k, 16) || !aligned(v.v, 16) || !aligned(v.table, 4) || !aligned(v.len, 4) || !aligned(v.k_scale, 4) ||
        !aligned(v.v_scale, 4))
        return DS_ERR_ALIGN;
    return DS_OK;
}

bool overlap(const void *a, uint64_t a_bytes, const void *b, uint64_t b_bytes)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y ? y - x < a_bytes : x - y < b_bytes;
}

ds_status decode_args(const ds_kv_cache *cache, const ds_decode_params *p, uint32_t n_rows, DecodeArgs &a)
{
    if (!p) return DS_ERR_NULL;
    a = DecodeArgs{};
    ds_status st = view_of(cache, p->max_len, a.c);
    if (st != DS_OK) return st;
    a.q_type = enum_int(p->q_type);
    if (a.q_type != DS_F16 && a.q_type != DS_BF16) return DS_ERR_ARG;
    if (a.c.type != DS_E4M3 && a.c.type != a.q_type) return DS_ERR_ARG;
    if (!p->n_q || p->n_q % a.c.n_kv || !p->n_tokens || p->n_tokens > DS_MAX_NEW_TOKENS) return DS_ERR_ARG;
    if (!isfinite(p->scale)) return DS_ERR_ARG;
    const float scale2 = (float)(p->scale * 1.4426950408889634);   // log2(e)
    if (!isfinite(scale2)) return DS_ERR_ARG;
    a.scale2 = scale2;
    a.group = p->n_q / a.c.n_kv;
    a.tokens = p->n_tokens;
    if ((uint64_t)a.group * a.tokens > DS_MAX_QUERY_ROWS) return DS_ERR_SIZE;
    if (p->q_row_stride % 8 || p->q_token_stride % 8 || p->q_head_stride % 8) return DS_ERR_ALIGN;
    a.q_row = p->q_row_stride;
    a.q_token = p->q_token_stride;
    a.q_head = p->q_head_stride;
    a.window = clamp32(p->window, kMaxTokens);
    a.sinks = clamp32(p->sinks, kMaxTokens);
    a.mass_len = p->mass_len;
    a.n_rows = n_rows;
    if (n_rows == 0) return DS_OK;
    if (n_rows > DS_MAX_ITEMS || (uint64_t)n_rows * a.c.n_kv * a.group * a.tokens > kMaxGrid) return DS_ERR_SIZE;
    decode_plan(a);
    if (attend_grid(a) > kMaxGrid ||
        (uint64_t)n_rows * a.c.n_kv * (a.score_len / 1024 + 2 + a.group * a.tokens) > kMaxGrid)
        return DS_ERR_SIZE;
    return DS_OK;
}

ds_status evict_args(const ds_kv_cache *src, const ds_kv_cache *dst, const ds_evict_params *params, uint32_t n_rows, EvictArgs &a)
{
    if (!params) return DS_ERR_NULL;
    a = EvictArgs{};
    ds_status st = view_of(src, params->max_len, a.src);
    if (st == DS_OK) st = view_of(dst, 0, a.dst);
    if (st != DS_OK) return st;
    if (a.src.type != a.dst.type || a.src.page_size != a.dst.page_size || a.src.n_kv != a.dst.n_kv || a.src.dim != a.dst.dim ||
        a.src.page_stride != a.dst.page_stride || a.src.token_stride != a.dst.token_stride ||
        a.src.head_stride != a.dst.head_stride)
        return DS_ERR_ARG;
    if (params->mass_len < a.src.cap || n_rows > a.dst.n_requests) return DS_ERR_ARG;
    a.mass_len = params->mass_len;
    a.kept_len = params->kept_len;
    a.n_rows = n_rows;
    a.sinks = params->sinks;
    a.recent = params->recent;
    a.slack = params->slack;
    evict_plan(a);
    if ((uint64_t)n_rows * a.src.n_kv * (a.n_chunks ? a.n_chunks : 1) > kMaxGrid1024) return DS_ERR_SIZE;
    return DS_OK;
}

// A workspace of the flag alone is used by DS_VALIDATE only.
ds_status check_scratch(void *ws, size_t ws_bytes, size_t need, uint32_t flags)
{
    return need || (flags & DS_VALIDATE) ? check_ws(ws, ws_bytes, kFlagBytes + need) : DS_OK;
}

ds_status verify_args(const ds_verify_params *p, uint32_t n_rows, VerifyArgs &v)
{
    if (!p) return DS_ERR_NULL;
    v = VerifyArgs{};
    v.type = enum_int(p->type);
    if (v.type != DS_F32 && v.type != DS_F16 && v.type != DS_BF16) return DS_ERR_ARG;
    if (p->n_drafts > DS_MAX_DRAFTS || p->vocab == 0) return DS_ERR_ARG;
    if (p->vocab > DS_MAX_VOCAB || n_rows > DS_MAX_ITEMS || (uint64_t)n_rows * cdiv(p->vocab, 1024) > kMaxGrid) return DS_ERR_SIZE;
    v.n_drafts = p->n_drafts;
    v.vocab = p->vocab;
    v.n_requests = p->n_requests;
    v.t_row = p->target_row_stride;
    v.t_pos = p->target_pos_stride;
    v.d_row = p->draft_row_stride;
    v.d_pos = p->draft_pos_stride;
    v.n_rows = n_rows;
    return DS_OK;
}

}  // namespace

extern "C" {

size_t ds_decode_workspace_bytes(const ds_kv_cache *cache, const ds_decode_params *params, uint32_t n_rows, int with_mass)
{
    DecodeArgs a;
    if (decode_args(cache, params, n_rows, a) != DS_OK) return 0;
    if (n_rows && with_mass && a.score_len > DS_MAX_MASS_TOKENS) return 0;
    return kFlagBytes + (n_rows ? decode_ws_bytes(a, with_mass != 0) : 0);
}

ds_status ds_decode_attention(const ds_kv_cache *cache, const ds_decode_params *params, uint32_t n_rows,
                              const uint32_t *rows, const void *q, void *out, float *mass, void *ws, size_t ws_bytes,
                              uint32_t flags, ds_stream stream)
{
    DecodeArgs a;
    ds_status st = decode_args(cache, params, n_rows, a);
    if (st != DS_OK) return st;
    if (mass && a.mass_len < a.c.cap) return DS_ERR_ARG;
    if (n_rows == 0) return DS_OK;
    if (mass && a.score_len > DS_MAX_MASS_TOKENS) return DS_ERR_SIZE;
    if (!rows && n_rows > a.c.n_requests) return DS_ERR_ARG;
    st = pointers_of(a.c);
    if (st != DS_OK) return st;
    if (!q || !out) return DS_ERR_NULL;
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(rows, 4) || !aligned(mass, 4)) return DS_ERR_ALIGN;
    st = check_scratch(ws, ws_bytes, decode_ws_bytes(a, mass != nullptr), flags);
    if (st != DS_OK) return st;
    a.rows = rows;
    a.q = q;
    a.out = out;
    a.mass = mass;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return run(ws, flags, s, [&](uint32_t *flag) { return flag ? decode_check(a, flag, s) : decode_launch(a, after_flag(ws), s); });
}

size_t ds_evict_workspace_bytes(const ds_kv_cache *src, const ds_kv_cache *dst, const ds_evict_params *params, uint32_t n_rows)
{
    EvictArgs a;
    if (evict_args(src, dst, params, n_rows, a) != DS_OK) return 0;
    return kFlagBytes + evict_ws_bytes(a);
}

ds_status ds_cache_evict(const ds_kv_cache *src, const ds_kv_cache *dst, const ds_evict_params *params, uint32_t n_rows,
                         const uint32_t *rows, const double *budget, const float *mass, float *mass_out, uint32_t *kept,
                         void *ws, size_t ws_bytes, uint32_t flags, ds_stream stream)
{
    EvictArgs a;
    ds_status st = evict_args(src, dst, params, n_rows, a);
    if (st != DS_OK) return st;
    if (n_rows == 0) return DS_OK;
    if (!rows && n_rows > a.src.n_requests) return DS_ERR_ARG;
    st = pointers_of(a.src);
    if (st == DS_OK) st = pointers_of(a.dst);
    if (st != DS_OK) return st;
    if (!budget || !mass || !mass_out || !kept) return DS_ERR_NULL;
    if (!aligned(budget, 8) || !aligned(mass, 4) || !aligned(mass_out, 4) || !aligned(kept, 4) || !aligned(rows, 4))
        return DS_ERR_ALIGN;
    st = check_scratch(ws, ws_bytes, evict_ws_bytes(a), flags);
    if (st != DS_OK) return st;
    // every launch looks up again which rows are cut: their lengths may not change on the way
    if (overlap(a.src.len, (uint64_t)a.src.n_requests * 4, a.dst.len, (uint64_t)n_rows * 4)) return DS_ERR_ARG;
    a.rows = rows;
    a.budget = budget;
    a.mass = mass;
    a.mass_out = mass_out;
    a.kept = kept;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return run(ws, flags, s, [&](uint32_t *flag) { return flag ? evict_check(a, flag, s) : evict_launch(a, after_flag(ws), s); });
}

size_t ds_verify_workspace_bytes(const ds_verify_params *params, uint32_t n_rows)
{
    VerifyArgs v;
    if (verify_args(params, n_rows, v) != DS_OK) return 0;
    return kFlagBytes + verify_ws_bytes(n_rows, v.vocab);
}

ds_status ds_verify_draft(const ds_verify_params *params, uint32_t n_rows, const uint32_t *rows, const void *target,
                          const void *draft, const int32_t *tokens, const uint32_t *n_draft, const float *u,
                          const float *u_sample, int32_t *out, uint32_t *n_emitted, uint32_t *observed, uint32_t *len,
                          void *ws, size_t ws_bytes, uint32_t flags, ds_stream stream)
{
    VerifyArgs v;
    ds_status st = verify_args(params, n_rows, v);
    if (st != DS_OK) return st;
    if (n_rows == 0) return DS_OK;
    if ((observed || len) && !rows && n_rows > v.n_requests) return DS_ERR_ARG;
    if (!target || !u_sample || !out || !n_emitted || (v.n_drafts && (!tokens || !u))) return DS_ERR_NULL;
    const size_t elem = v.type == DS_F32 ? 4 : 2;
    if (!aligned(target, elem) || !aligned(draft, elem) || !aligned(tokens, 4) || !aligned(n_draft, 4) || !aligned(u, 4) ||
        !aligned(u_sample, 4) || !aligned(out, 4) || !aligned(n_emitted, 4) || !aligned(observed, 4) || !aligned(len, 4) ||
        !aligned(rows, 4))
        return DS_ERR_ALIGN;
    st = check_ws(ws, ws_bytes, kFlagBytes + verify_ws_bytes(n_rows, v.vocab));
    if (st != DS_OK) return st;
    v.rows = rows;
    v.target = target;
    v.draft = draft;
    v.tokens = tokens;
    v.n_draft = n_draft;
    v.u = u;
    v.u_sample = u_sample;
    v.out = out;
    v.n_emitted = n_emitted;
    v.observed = observed;
    v.len = len;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return run(ws, flags, s, [&](uint32_t *flag) { return flag ? verify_check(v, flag, s) : verify_launch(v, after_flag(ws), s); });
}

}  // extern "C"
