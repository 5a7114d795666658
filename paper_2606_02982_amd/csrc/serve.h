// Internal interface of the decode-step kernels: arguments and launchers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/driftsched_serve.h"

namespace ds {

// A cache as the kernels see it. cap: the most tokens a request is taken to
// hold (a larger length is clamped to it).
struct KvView {
    uint8_t *k, *v;
    const float *k_scale, *v_scale;
    const uint32_t *table;
    uint32_t *len;
    uint32_t n_requests, max_pages, n_pages, page_size, n_kv, dim, cap;
    uint64_t page_stride, token_stride, head_stride;   // elements
    int type;
    int page_shift;        // log2(page_size), or -1
};

struct DecodeArgs {
    KvView c;
    const uint32_t *rows;
    const void *q;
    void *out;
    float *mass;
    uint64_t q_row, q_token, q_head, mass_len;
    uint32_t n_rows, group, tokens, window, sinks;
    float scale2;          // scale * log2(e)
    int q_type;
    // The split. A slot is a run of blocks of one row; it has n_kv pairs
    // (slot, head), and a pair one unit per tile of 16 or 32 query rows. Which
    // blocks a slot holds follows on the device from the batch's lengths.
    uint32_t n_tiles;      // tiles per pair
    uint32_t n_slots;      // most slots of a batch of this size
    uint32_t slot_goal;    // slots wanted where the caches are long enough; 0: one per row
    uint32_t slot_blocks;  // and blocks that are not cut further
    int spread;            // order of the pairs (attend_kernel)
    uint32_t part_rows;    // query rows of a unit's partial result
    uint32_t score_len;    // tokens of a row of scores
    float *part_o;         // (unit, part_rows, padded dim): mean values; a row in one slot has none
    float *part_ml;        // (unit, part_rows, 2): running maximum and sum
    uint32_t *row_slots;   // (row, 2): its first slot and their number
    float *scores;         // (row, head, query row, score_len), for mass
};

struct EvictArgs {
    KvView src, dst;
    const uint32_t *rows;
    const double *budget;
    const float *mass;
    float *mass_out;
    uint32_t *kept;
    uint64_t mass_len, kept_len;
    uint32_t n_rows, sinks, recent, slack;
    // long requests: the selection split into chunks of tokens
    uint32_t chunk_tokens, n_chunks;   // n_chunks 0: one workgroup selects for a (row, head)
    uint32_t most_kept;                // the most tokens that a request can keep
    uint32_t *counts;                  // (row, head, chunk, 2048): masses by their first digit
    uint32_t *starts;                  // (row, head, chunk, 2): kept and equal tokens before the chunk
    uint32_t *bars;                    // (row, head, 2): smallest kept key, how many of it stay
    float *kept_mass;                  // (row, head, most_kept)
};

struct VerifyArgs {
    const uint32_t *rows;
    const void *target, *draft;
    const int32_t *tokens;
    const uint32_t *n_draft;
    const float *u, *u_sample;
    int32_t *out;
    uint32_t *n_emitted, *observed, *len;
    uint64_t t_row, t_pos, d_row, d_pos;
    uint32_t n_rows, n_drafts, vocab, n_requests;
    int type;
    double *sums;          // (row, chunk, 2): of the weights and of the target
    uint32_t *accepted;    // per row
};

constexpr uint32_t kBlockTokens = 32;   // tokens of one step of the attention loop

// Width that a head's dimensions are padded to in registers.
inline uint32_t padded_dim(uint32_t dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }
// 16-row tiles that one wave carries.
inline uint32_t unit_tiles(uint32_t dim, uint32_t query_rows) { return query_rows > 16 && dim <= 128 ? 2 : 1; }

// Blocks of 32 tokens that a row of n tokens visits: those with a sink token,
// then those from the window's start on.
struct Span {
    uint32_t sink_blocks, first_block, total;
};
__host__ __device__ inline Span span_of(uint32_t n, uint32_t tokens, uint32_t window, uint32_t sinks)
{
    Span s;
    const uint32_t lo = window && n > tokens && n - tokens >= window ? n - tokens - window + 1 : 0;
    s.first_block = lo / kBlockTokens;
    const uint32_t sb = sinks / kBlockTokens + (sinks % kBlockTokens != 0);
    s.sink_blocks = sb < s.first_block ? sb : s.first_block;
    s.total = s.sink_blocks + (n + kBlockTokens - 1) / kBlockTokens - s.first_block;
    return s;
}

enum { kHeadsFirst, kSlotsFirst, kDieOfSlot };   // DecodeArgs.spread

// Workgroups of the attention kernel.
inline uint64_t attend_grid(const DecodeArgs &a)
{
    const uint64_t n_kv = a.c.n_kv, slots = a.spread == kSlotsFirst ? a.n_slots | 1u : a.n_slots;
    return a.spread == kDieOfSlot ? (slots + 7) / 8 * 8 * n_kv * a.n_tiles : (slots * n_kv + 7) / 8 * 8 * a.n_tiles;
}

// Sets the split of a; the largest grid and the workspace bytes follow from it.
void decode_plan(DecodeArgs &a);
size_t decode_ws_bytes(const DecodeArgs &a, bool with_mass);
hipError_t decode_launch(DecodeArgs a, void *ws, hipStream_t s);
hipError_t decode_check(const DecodeArgs &a, uint32_t *flag, hipStream_t s);
// Requests, lengths and pages of a batch; once: no request twice.
hipError_t cache_check(const KvView &c, const uint32_t *rows, uint32_t n_rows, bool once, uint32_t *flag, hipStream_t s);

hipError_t decode_attend_bf16(const DecodeArgs &a, hipStream_t s);
hipError_t decode_attend_f16(const DecodeArgs &a, hipStream_t s);
hipError_t decode_attend_bf16_e4m3(const DecodeArgs &a, hipStream_t s);
hipError_t decode_attend_f16_e4m3(const DecodeArgs &a, hipStream_t s);

// Sets the chunks of a.
void evict_plan(EvictArgs &a);
size_t evict_ws_bytes(const EvictArgs &a);
hipError_t evict_launch(EvictArgs a, void *ws, hipStream_t s);
hipError_t evict_check(const EvictArgs &a, uint32_t *flag, hipStream_t s);

size_t verify_ws_bytes(uint32_t n_rows, uint32_t vocab);
hipError_t verify_launch(VerifyArgs a, void *ws, hipStream_t s);
hipError_t verify_check(const VerifyArgs &a, uint32_t *flag, hipStream_t s);

}  // namespace ds
