// Attention of the newest tokens over a paged cache: the kernel (included by
// one source per element type, attend_*.hip).
//
// With q scaled by scale * log2(e), every query keeps the running maximum m
// of its scores s_j, the sum l = sum_j 2^(s_j - m) and o = sum_j 2^(s_j - m)
// v_j, and rescales l and o when m grows; out = o / l. Splits of the cache
// and the four waves of a workgroup hold (m, l, o / l) of their own tokens and
// are joined by the same rule: o / l is a mean of values and so no larger than
// the largest of them, while o of values near the type's end may pass it.
//
// The work is reading the cache once: 4 dim bytes per token and head in 16
// bits against 4 dim flops per query row. So the loop is laid out for loads:
// a wave takes 32 tokens at a time straight from memory into the operand
// layout of the matrix instructions, with no pass through shared memory.
//  - scores: S^T = K Q^T in 16x16x32 steps. Lane (m, g) of K holds token m,
//    dimensions 8 g .. of each 32 (16 g .. of each 64 in 8 bits: the order of
//    a sum's terms is free, so a load is always 16 bytes).
//  - S^T leaves the tokens 4 g + i of column m (a query) in lane (m, g); this
//    is taken as the order of the 32 tokens in the second product, so the
//    weights are its operand where they stand.
//  - O^T = V^T P^T: lane (m, g) loads dimensions 8 m .. 8 m + 7 of its eight
//    tokens, a row of V by 16 lanes, and swaps 16-bit halves between its own
//    registers to get one dimension of eight tokens.
// Weights are split into two 16-bit parts (value and remainder), so that
// rounding them adds nothing to out's own rounding; the matrix units are idle
// most of the time anyway. float16 has no step below 2^-24, so there the
// weights are taken times 2^15 (at most 32,768): what both parts lose is below
// 2^-40 of the largest weight instead of 2^-25.
#pragma once

#include "common.h"
#include "serve.h"

namespace ds {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
typedef uint32_t uintx2 __attribute__((ext_vector_type(2)));

struct Bf16 {
    static constexpr float kWeight = 1.0f;         // what weights are multiplied with before they are split
    typedef __bf16 x8 __attribute__((ext_vector_type(8)));
    typedef __bf16 x2 __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ floatx4 mfma(uintx4 a, uintx4 b, floatx4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b)
    {
        const floatx2 v = {a, b};
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, x2));
    }
    static __device__ __forceinline__ float lo(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
    static __device__ __forceinline__ float hi(uint32_t w) { return __builtin_bit_cast(float, w & 0xFFFF0000u); }
    // two 8-bit floats, exact
    template <bool kHigh>
    static __device__ __forceinline__ uint32_t from_e4m3(uint32_t w)
    {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, kHigh));
    }
};

struct F16 {
    static constexpr float kWeight = 32768.0f;
    typedef _Float16 x8 __attribute__((ext_vector_type(8)));
    typedef _Float16 x2 __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ floatx4 mfma(uintx4 a, uintx4 b, floatx4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b)
    {
        const floatx2 v = {a, b};
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, x2));
    }
    static __device__ __forceinline__ float lo(uint32_t w) { return (float)__builtin_bit_cast(x2, w)[0]; }
    static __device__ __forceinline__ float hi(uint32_t w) { return (float)__builtin_bit_cast(x2, w)[1]; }
    template <bool kHigh>
    static __device__ __forceinline__ uint32_t from_e4m3(uint32_t w)
    {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, kHigh));
    }
};

// The largest of x over lanes m, m + 16, m + 32, m + 48.
__device__ __forceinline__ float max_over_groups(float x)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    x = fmaxf(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]));
    const uint32_t w = __builtin_bit_cast(uint32_t, x);
    const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)b[0]), __builtin_bit_cast(float, (uint32_t)b[1]));
}

__device__ __forceinline__ float finite_or_zero(float m) { return m == -__builtin_inff() ? 0.0f : m; }

typedef const __attribute__((address_space(4))) uint32_t *ScalarU32;   // read-only during the launch: scalar loads

// Rows whose lengths every workgroup looks through. Above it every row is one
// slot: looking through more rows costs more than the split gives where
// lengths are alike, and a row far longer than the others then takes the time
// of one workgroup per head (2 heads of 128 dimensions in 16 bits, up to 400
// tokens, 1,025 rows split / not: 75 / 45 us, 2,048 rows 152 / 79 us; one
// head, one row of 32,768 tokens among 1,025 of 64: 34 / 430 us).
constexpr uint32_t kBalancedRows = 1024;

__device__ __forceinline__ uint32_t length_of(const DecodeArgs &a, uint32_t row, uint32_t &req)
{
    req = a.rows ? a.rows[row] : row;
    const uint32_t n = req < a.c.n_requests ? a.c.len[req] : 0;
    return n < a.c.cap ? n : a.c.cap;
}

struct Slots {
    uint32_t row;          // kNone: there is no such slot
    uint32_t first, count; // the row's slots
    uint32_t req, n;       // its request and length
};
constexpr uint32_t kNone = 0xFFFFFFFFu;

// The row that slot `want` belongs to. Rows differ in length, so slots are
// cut from the batch's blocks as a whole: of all rows' blocks a slot gets at
// most ceil(blocks / slot_goal), at least slot_blocks, and a row is cut
// into equal slots of at most that. Every workgroup of 256 threads finds this
// by itself, looking through the rows' lengths (a launch before would cost
// more than the few hundred cycles).
__device__ inline Slots find_slots(const DecodeArgs &a, uint32_t want)
{
    if (a.slot_goal == 0) {
        Slots s{want < a.n_rows ? want : kNone, want, 1, 0, 0};
        if (s.row != kNone) s.n = length_of(a, want, s.req);
        return s;
    }
    __shared__ uint64_t sm_blocks[4];
    __shared__ uint32_t sm_slots[4], sm_found[5];
    const uint32_t each = (a.n_rows + 255) / 256, r0 = threadIdx.x * each;
    const uint32_t r1 = r0 + each < a.n_rows ? r0 + each : a.n_rows;
    const int wave = threadIdx.x >> 6;
    uint64_t blocks = 0;
    uint32_t total = 0, n = 0, req = 0;                 // of the last row looked at
    auto look = [&](uint32_t r) {
        n = length_of(a, r, req);
        total = span_of(n, a.tokens, a.window, a.sinks).total;
    };
    for (uint32_t r = r0; r < r1; r++) {
        look(r);
        blocks += total;
    }
    uint64_t all = blocks;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) all += __shfl_xor(all, d, 64);
    if (lane_id() == 0) sm_blocks[wave] = all;
    if (threadIdx.x == 0) sm_found[0] = kNone;
    __syncthreads();
    all = sm_blocks[0] + sm_blocks[1] + sm_blocks[2] + sm_blocks[3];
    // all < 2^37: a float holds the quotient to far less than a slot
    uint32_t most = (uint32_t)((float)all / (float)a.slot_goal) + 1;
    most = most > a.slot_blocks ? most : a.slot_blocks;
    auto slots_of = [&](uint32_t t) { return t <= most ? 1u : (t + most - 1) / most; };
    uint32_t own = 0;
    for (uint32_t r = r0; r < r1; r++) {
        if (each > 1) look(r);
        own += slots_of(total);
    }
    const uint32_t incl = wave_incl_scan_dpp(own);
    if (lane_id() == 63) sm_slots[wave] = incl;
    __syncthreads();
    uint32_t first = incl - own;
    for (int w = 0; w < wave; w++) first += sm_slots[w];
    if (want - first < own)
        for (uint32_t r = r0; r < r1; r++) {
            if (each > 1) look(r);
            const uint32_t count = slots_of(total);
            if (want - first < count) {
                sm_found[0] = r;
                sm_found[1] = first;
                sm_found[2] = count;
                sm_found[3] = req;
                sm_found[4] = n;
            }
            first += count;
        }
    __syncthreads();
    auto same = [&](int k) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)sm_found[k]); };
    return Slots{same(0), same(1), same(2), same(3), same(4)};
}

// One wave's share of a unit: steps wave, wave + 4, ... of the slot's blocks
// (see DecodeArgs for slots and units).
// kDim: padded dimensions; kTiles: 16-row tiles of queries. kPath: kAnyPage,
// addresses are per lane; kPages16, a page holds a multiple of 16 tokens, so
// half a block lies in one page, its address is the same for the whole wave,
// and a lane's place in it is a 32-bit offset; kWhole, that and all kDim
// dimensions are there. (32 rows of 2,000 to 10,000 tokens, 8 heads in 16
// bits: 128 dimensions 133 us, in pages of 24 tokens 148; 80 dimensions 116
// us, in pages of 24 tokens 128.)
enum { kAnyPage, kPages16, kWhole };

// A step takes two blocks where one is 8 KB of keys and values or less and
// there is one tile of query rows, else one (32 KB for 256 dimensions in 16
// bits): the chain of a step (products, maximum over the lanes, exponentials,
// products) is as long for few bytes as for many, and a second tile needs the
// registers of the second block.
template <int kDim, int kElem, int kTiles>
constexpr int kSubBlocks = kDim * kElem >= 256 || kTiles > 1 ? 1 : 2;

template <typename T, bool kE4m3, int kDim, int kTiles, int kPath, bool kStream>
struct Attender {
    static constexpr bool kFast = kPath >= kPages16;
    static constexpr int kElem = kE4m3 ? 1 : 2;
    static constexpr bool kWideValues = !kE4m3 && T::kWeight == 1.0f;   // bfloat16
    static constexpr int kStepsK = kDim / 32;                  // matrix steps per score
    static constexpr int kLoadsK = kE4m3 ? kDim / 64 : kDim / 32;
    static constexpr int kParts = kDim > 128 ? kDim / 128 : 1; // V: pieces of a row
    static constexpr int kVd = kDim / 16 / kParts;             // V: dimensions per lane and piece
    static constexpr int kVw = kVd * kElem / 4;                // V: 32-bit words per lane, token and piece
    static constexpr int kOut = kDim / 16;                     // 16-dimension tiles of O^T
    static constexpr int kSub = kSubBlocks<kDim, kElem, kTiles>;       // blocks of 32 tokens per step

    // Where a block's tokens are.
    struct Place {
        int j0;
        uint32_t seen;          // tokens that exist, by bit
        uint64_t base[2];       // kFast: element offset of each half (the same in all lanes)
        uint64_t at;            // else: of token (lane & 31)
    };

    const DecodeArgs &a;
    Span span;
    uint32_t n;
    int m, g, first_pos, lo;
    float scale;
    float down;                                                // what kCareful multiplies values with
    ScalarU32 table;
    const uint8_t *kh, *vh;
    __amdgpu_buffer_rsrc_t score_rsrc;                         // this tile's rows of scores
    uint32_t score_lane[kTiles];
    uint32_t k_lane, v_lane, token_bytes;                      // kFast: this lane's byte offsets in half a block

    uintx4 q[kTiles][kStepsK];
    int pos[kTiles];
    float mx[kTiles], sum[kTiles];
    floatx4 acc[kTiles][kOut];
    uintx4 kr[kSub][2][kLoadsK];
    uint32_t vr[kSub][8][kParts][kVw];
    uint32_t page[kSub][2];                                    // kFast: of the step after next

    __device__ __forceinline__ uint32_t block_of(uint32_t v) const
    {
        return v < span.sink_blocks ? v : span.first_block + (v - span.sink_blocks);
    }
    __device__ __forceinline__ uint32_t page_of(uint32_t j) const
    {
        return a.c.page_shift >= 0 ? j >> a.c.page_shift : j / a.c.page_size;
    }

    // The pages of the halves of blocks v, v + 1, .. (kFast; no page where there is no token).
    __device__ __forceinline__ void pages(uint32_t v, uint32_t v1)
    {
#pragma unroll
        for (int b = 0; b < kSub; b++) {
            const uint32_t j0 = block_of(v + b) * kBlockTokens;
#pragma unroll
            for (int i = 0; i < 2; i++)
                page[b][i] = v + b < v1 && j0 + 16 * i < n ? table[page_of(j0 + 16 * i)] : 0xFFFFFFFFu;
        }
    }

    __device__ __forceinline__ Place place(uint32_t v, uint32_t v1, const uint32_t *page) const
    {
        Place p;
        p.j0 = (int)(block_of(v) * kBlockTokens);
        p.seen = 0xFFFFFFFFu;
        if constexpr (kFast) {
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const bool ok = page[i] < a.c.n_pages;
                if (!ok) p.seen &= i ? 0x0000FFFFu : 0xFFFF0000u;
                const uint32_t j = (uint32_t)p.j0 + 16 * i, slot = j - page_of(j) * a.c.page_size;
                p.base[i] = (ok ? page[i] : 0u) * a.c.page_stride + slot * a.c.token_stride;
            }
        } else {
            const uint32_t j = (uint32_t)p.j0 + (lane_id() & 31);
            const uint32_t pg = v < v1 && j < n ? ((const uint32_t *)a.c.table)[(uint64_t)req * a.c.max_pages + page_of(j)] : 0xFFFFFFFFu;
            const bool ok = pg < a.c.n_pages;
            p.seen = (uint32_t)__ballot(ok);
            p.at = (ok ? pg : 0u) * a.c.page_stride + (j - page_of(j) * a.c.page_size) * a.c.token_stride;
        }
        const int left = v < v1 ? (int)n - p.j0 : 0;
        if (left < 32) p.seen &= (1u << left) - 1u;
        return p;
    }
    __device__ __forceinline__ uint64_t at_of(const Place &p, int token) const
    {
        return ((uint64_t)(uint32_t)__shfl((int)(uint32_t)(p.at >> 32), token, 64) << 32) |
               (uint32_t)__shfl((int)(uint32_t)p.at, token, 64);
    }

    // kStream: whole cache lines that no other unit of the pair reads go past
    // the caches (16 heads of 128 dimensions in 16 bits: 380 -> 370 us for 2.1
    // GB, 8 heads of 256: 348 -> 336 us, 20 query rows 216 -> 199 us; in 8
    // bits 217 -> 222 us, 40 query rows, whose two units read the same, 268 ->
    // 365 us). Not where dimensions are missing: heads share lines, and the
    // first dimensions are read again in place of the last (8 heads of 80: 116
    // us, streamed 160; of 192: 228 and 276).
    // Which requests share pages the host does not know, and such pages would
    // gain from the caches (32 requests of 8,192 tokens, 8 heads of 128
    // dimensions in 16 bits, streamed / not: none shared 176 / 193 us, the
    // first half 161 / 123, all 145 / 83; 8 heads of 256, 16 requests: 175 /
    // 185, 141 / 132 and 116 / 102).
    template <typename W>
    static __device__ __forceinline__ W fetch(const uint8_t *p)
    {
        if constexpr (kStream)
            return __builtin_nontemporal_load(reinterpret_cast<const W *>(p));
        else
            return *reinterpret_cast<const W *>(p);
    }

    // Dimension d of a token if there is one, else the first. What is read in
    // its place is taken out of the keys where they are used, so that no load
    // is waited for early, and gives values that are never written.
    __device__ __forceinline__ uint32_t within(uint32_t d) const { return kPath == kWhole || d < a.c.dim ? d : 0; }

    __device__ __forceinline__ void load_k(const Place &p, uintx4 (&kr)[2][kLoadsK])
    {
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const uint8_t *base = kFast ? kh + p.base[i] * kElem + k_lane : kh + at_of(p, 16 * i + m) * kElem;
#pragma unroll
            for (int s = 0; s < kLoadsK; s++) {
                if constexpr (kPath == kWhole)
                    kr[i][s] = fetch<uintx4>(base + s * 64);
                else
                    kr[i][s] = fetch<uintx4>(base + within(kE4m3 ? s * 64 + g * 16 : s * 32 + g * 8) * kElem);
            }
        }
    }

    // dimensions kVd m .. of each piece, for the lane's eight tokens, as stored
    __device__ __forceinline__ void load_v(const Place &p, uint32_t (&vr)[8][kParts][kVw])
    {
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const uint8_t *base;
            if constexpr (kFast)
                base = vh + p.base[j >> 2] * kElem + (j & 3) * token_bytes + v_lane;
            else
                base = vh + at_of(p, (j >> 2) * 16 + g * 4 + (j & 3)) * kElem;
#pragma unroll
            for (int h = 0; h < kParts; h++) {
                const uint8_t *src = kPath == kWhole ? base + h * 128 * kElem : base + within(h * 128 + m * kVd) * kElem;
                if constexpr (kVw == 4) {
                    const uintx4 x = fetch<uintx4>(src);
#pragma unroll
                    for (int w = 0; w < 4; w++) vr[j][h][w] = x[w];
                } else if constexpr (kVw == 2) {
                    const uintx2 x = fetch<uintx2>(src);
                    vr[j][h][0] = x[0];
                    vr[j][h][1] = x[1];
                } else {
                    vr[j][h][0] = fetch<uint32_t>(src);
                }
            }
        }
    }

    // All blocks of the wave. Keys of the next block are loaded as soon as
    // the scores have used the present ones, values as soon as the second
    // product has: while one is waited for the other is under way.
    // kCareful: 0 * inf or 0 * NaN of a token that some queries do not see
    // must not reach their sums, so every product is made only where the
    // weight is not 0, and with values small enough for their sum (taken
    // where the first pass gave a number that is not finite).
    template <bool kCareful>
    __device__ __forceinline__ void pass(uint32_t v, uint32_t v1)
    {
#pragma unroll
        for (int t = 0; t < kTiles; t++) {
            mx[t] = -__builtin_inff();
            sum[t] = 0.0f;
#pragma unroll
            for (int x = 0; x < kOut; x++) acc[t][x] = floatx4{0, 0, 0, 0};
        }
        if (v >= v1) return;
        if (kFast) pages(v, v1);
        Place here[kSub];
#pragma unroll
        for (int b = 0; b < kSub; b++) {
            here[b] = place(v + b, v1, page[b]);
            load_k(here[b], kr[b]);
        }
#pragma unroll
        for (int b = 0; b < kSub; b++) load_v(here[b], vr[b]);
        if (kFast) pages(v + 4 * kSub, v1);
        for (;;) {
            floatx4 s[kTiles][2 * kSub];
#pragma unroll
            for (int i = 0; i < 2 * kSub; i++)
#pragma unroll
                for (int t = 0; t < kTiles; t++) {
                    s[t][i] = floatx4{0, 0, 0, 0};
#pragma unroll
                    for (int st = 0; st < kStepsK; st++) {
                        uintx4 kf;
                        if constexpr (kE4m3) {
                            const uint32_t w0 = kr[i >> 1][i & 1][st >> 1][(st & 1) * 2], w1 = kr[i >> 1][i & 1][st >> 1][(st & 1) * 2 + 1];
                            kf = uintx4{T::template from_e4m3<false>(w0), T::template from_e4m3<true>(w0),
                                        T::template from_e4m3<false>(w1), T::template from_e4m3<true>(w1)};
                        } else {
                            kf = kr[i >> 1][i & 1][st];
                        }
                        if constexpr (kPath != kWhole)
                            if ((kE4m3 ? (st >> 1) * 64 + g * 16 : st * 32 + g * 8) >= (int)a.c.dim) kf = uintx4{0, 0, 0, 0};
                        s[t][i] = T::mfma(kf, q[t][st], s[t][i]);
                    }
                }
            const bool more = v + 4 * kSub < v1;
            Place next[kSub];
            if (more) {
#pragma unroll
                for (int b = 0; b < kSub; b++) {
                    next[b] = place(v + 4 * kSub + b, v1, page[b]);
                    load_k(next[b], kr[b]);
                }
                if (kFast) pages(v + 8 * kSub, v1);
            }

            // which tokens any query sees; whether every query sees all
            uint32_t seen[kSub];
            bool full[kSub];
#pragma unroll
            for (int b = 0; b < kSub; b++) {
                const int j0 = here[b].j0;
                seen[b] = here[b].seen;
                full[b] = seen[b] == 0xFFFFFFFFu && j0 + 31 <= first_pos &&
                          (a.window == 0 || j0 > (int)n - 1 - (int)a.window || j0 + 31 < (int)a.sinks);
                if (!full[b]) {
                    uint32_t near = 0xFFFFFFFFu;        // at or behind the window's start
                    if (lo > j0) near = lo - j0 < 32 ? ~((1u << (lo - j0)) - 1u) : 0u;
                    uint32_t sink = 0;
                    if ((int)a.sinks > j0) sink = (int)a.sinks - j0 < 32 ? (1u << ((int)a.sinks - j0)) - 1u : 0xFFFFFFFFu;
                    seen[b] &= near | sink;
#pragma unroll
                    for (int t = 0; t < kTiles; t++)
#pragma unroll
                        for (int i = 0; i < 2; i++)
#pragma unroll
                            for (int e = 0; e < 4; e++) {
                                const int bit = 16 * i + g * 4 + e, j = j0 + bit;
                                const bool on = ((seen[b] >> bit) & 1u) && j <= pos[t] &&
                                                (a.window == 0 || j > pos[t] - (int)a.window || j < (int)a.sinks);
                                s[t][2 * b + i][e] = on ? s[t][2 * b + i][e] * scale : -__builtin_inff();
                            }
                } else {
#pragma unroll
                    for (int t = 0; t < kTiles; t++)
#pragma unroll
                        for (int i = 0; i < 2; i++)
#pragma unroll
                            for (int e = 0; e < 4; e++) s[t][2 * b + i][e] *= scale;
                }
            }
            // without conditions, so that the loads under way are still
            // counted behind it: rows past the last one, blocks past the
            // split's end, and all of it where no weights are gathered, lie
            // outside the buffer and are dropped
#pragma unroll
            for (int t = 0; t < kTiles; t++)
#pragma unroll
                for (int i = 0; i < 2 * kSub; i++)
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(uintx4, s[t][i]), score_rsrc,
                                                           v + i / 2 < v1 ? score_lane[t] + 64 * i : 0xFFFFFFF0u,
                                                           v * (kBlockTokens * 4), 0);
            // softmax step: s becomes the weights
            uintx4 p_hi[kTiles][kSub], p_lo[kTiles][kSub];
#pragma unroll
            for (int t = 0; t < kTiles; t++) {
                float top = -__builtin_inff();
#pragma unroll
                for (int i = 0; i < 2 * kSub; i++)
#pragma unroll
                    for (int e = 0; e < 4; e++) top = fmaxf(top, s[t][i][e]);
                top = max_over_groups(top);
                if (__any(top > mx[t])) {
                    const float grown = fmaxf(mx[t], top);
                    const float f = __builtin_amdgcn_exp2f(mx[t] - finite_or_zero(grown));
                    mx[t] = grown;
                    sum[t] *= f;
#pragma unroll
                    for (int x = 0; x < kOut; x++)
#pragma unroll
                        for (int e = 0; e < 4; e++) acc[t][x][e] *= f;
                }
                const float base = finite_or_zero(mx[t]);
#pragma unroll
                for (int i = 0; i < 2 * kSub; i++)
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        s[t][i][e] = __builtin_amdgcn_exp2f(s[t][i][e] - base);
                        sum[t] += s[t][i][e];
                        if constexpr (T::kWeight != 1.0f) s[t][i][e] *= T::kWeight;
                    }
#pragma unroll
                for (int i = 0; i < 2 * kSub; i++)
#pragma unroll
                    for (int e = 0; e < 4; e += 2) {
                        const uint32_t w = T::pack(s[t][i][e], s[t][i][e + 1]);
                        p_hi[t][i >> 1][(i & 1) * 2 + e / 2] = w;
                        p_lo[t][i >> 1][(i & 1) * 2 + e / 2] = T::pack(s[t][i][e] - T::lo(w), s[t][i][e + 1] - T::hi(w));
                    }
            }
#pragma unroll
            for (int b = 0; b < kSub; b++) {
                if (!full[b]) {
#pragma unroll
                    for (int j = 0; j < 8; j++) {
                        const bool on = (seen[b] >> ((j >> 2) * 16 + g * 4 + (j & 3))) & 1u;
#pragma unroll
                        for (int h = 0; h < kParts; h++)
#pragma unroll
                            for (int w = 0; w < kVw; w++) vr[b][j][h][w] = on ? vr[b][j][h][w] : 0u;
                    }
                }
#pragma unroll
                for (int h = 0; h < kParts; h++)
#pragma unroll
                    for (int d = 0; d < kVd; d += 2) {
                        uint32_t pair[8];               // dimensions d, d + 1 of the eight tokens
#pragma unroll
                        for (int j = 0; j < 8; j++) {
                            if constexpr (kE4m3)
                                pair[j] = (d & 2) ? T::template from_e4m3<true>(vr[b][j][h][d >> 2])
                                                  : T::template from_e4m3<false>(vr[b][j][h][d >> 2]);
                            else
                                pair[j] = vr[b][j][h][d >> 1];
                        }
#pragma unroll
                        for (int o = 0; o < 2; o++) {
                            const int x = h * kVd + d + o;
                            const uint32_t sel = o ? 0x07060302u : 0x05040100u;
                            uintx4 vf;
#pragma unroll
                            for (int w = 0; w < 4; w++) vf[w] = __builtin_amdgcn_perm(pair[2 * w + 1], pair[2 * w], sel);
                            if constexpr (!kCareful) {
#pragma unroll
                                for (int t = 0; t < kTiles; t++) {
                                    acc[t][x] = T::mfma(vf, p_hi[t][b], acc[t][x]);
                                    acc[t][x] = T::mfma(vf, p_lo[t][b], acc[t][x]);
                                }
                            } else {
                                // lane (m, g) adds dimensions 4 g + i of column m
#pragma unroll 1
                                for (int from = 0; from < 4; from++)
#pragma unroll
                                    for (int j = 0; j < 8; j++)
#pragma unroll
                                        for (int t = 0; t < kTiles; t++) {
                                            const float pw = __shfl(s[t][2 * b + (j >> 2)][j & 3], from * 16 + m, 64);
#pragma unroll
                                            for (int i = 0; i < 4; i++) {
                                                const uint32_t w = (uint32_t)__shfl((int)vf[j >> 1], from * 16 + g * 4 + i, 64);
                                                const float val = ((j & 1) ? T::hi(w) : T::lo(w)) * down;
                                                if (pw != 0.0f) acc[t][x][i] += pw * val;
                                            }
                                        }
                            }
                        }
                    }
            }
            if (!more) break;
#pragma unroll
            for (int b = 0; b < kSub; b++) {
                here[b] = next[b];
                load_v(here[b], vr[b]);
            }
            v += 4 * kSub;
        }
    }
    uint32_t req;
};

// Waves per SIMD that the registers are limited to: as many as fit without
// spilling vector registers (scalar ones are spilled into lanes of these in
// most of the kernels, up to 33). kFast: kWhole, and kPages16 with two tiles of
// query rows (24 rows, 8 heads of 80 dimensions, 671 MB: 161 us, with one wave
// less 171; of 48, 302 MB: 98 and 99 us, in 8 bits 72 and 71; for one tile of
// 80 125 us for 481 MB, with one wave less 116).
template <int kWidth, int kSub, bool kFast>
constexpr int kWaves = kWidth <= 64 ? (kSub == 1 || kFast ? 3 : 2) : kWidth <= 128 ? (kSub == 1 && kFast ? 3 : 2) : kWidth <= 256 && kFast ? 2 : 1;

template <typename T, bool kE4m3, int kDim, int kTiles, int kPath, bool kStream>
__global__ __launch_bounds__(256, (kWaves<kDim == 256 ? 512 : kDim * kTiles, kSubBlocks<kDim, kE4m3 ? 1 : 2, kTiles>, kPath == kWhole || (kPath == kPages16 && kTiles > 1)>))
void attend_kernel(const DecodeArgs a)
{
    typedef Attender<T, kE4m3, kDim, kTiles, kPath, kStream> A;
    constexpr int kRows = 16 * kTiles;
    constexpr int kPitch = kDim + 4;

    __shared__ float sm_m[4][kRows], sm_l[4][kRows];
    __shared__ __align__(16) float sm_o[4][kRows * kPitch];

    const KvView &c = a.c;
    const int lane = lane_id(), m = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    // Workgroups go round the eight dies, each with a cache of its own. Units
    // of one pair, which read the same keys and values, go to one die. Which
    // pairs are under way at one time:
    //  - all heads of a slot on one die where a token's key is at most 128
    //    bytes, a cache line (8-bit, 8 heads: 64 dimensions 92 -> 69 us for
    //    268 MB, 128 dimensions 119 -> 116 us for 537 MB), or ends inside a
    //    line (8 heads of 80 dimensions in 16 bits 128 -> 116 us for 481 MB,
    //    of 96 130 -> 118 us for 577 MB), and there are 64 slots, eight for
    //    each die (80 dimensions in 16 bits, requests of 2,048 tokens, a die
    //    per slot / slots first: 128 slots 26 / 31 us, 64 slots 17 / 20, 32
    //    slots 15 / 17, 8 slots 14 / 15; with one slot one die has it all);
    //  - all slots of few heads, up to 8 heads (8 heads of 128 dimensions in
    //    16 bits: 192 -> 177 us for 1.07 GB, three long rows 241 -> 222 us
    //    for 1.33 GB); the odd number of slots spreads a slot's heads over
    //    the dies;
    //  - else all heads of few slots (16 heads: ragged rows up to 2,048 62 us
    //    for 292 MB, slots first 62 to 83; long rows 371 and 357 us).
    const uint32_t of_slot = a.spread == kDieOfSlot ? c.n_kv : 1;
    const uint32_t round = blockIdx.x / (8 * a.n_tiles * of_slot), within = blockIdx.x % (8 * a.n_tiles * of_slot);
    const uint32_t tile = within / 8 % a.n_tiles;
    const uint32_t at = (round * 8 + within % 8) * of_slot + within / 8 / a.n_tiles, per_head = a.n_slots | 1;
    const uint32_t slot = a.spread == kSlotsFirst ? at % per_head : at / c.n_kv;
    const uint32_t head = a.spread == kSlotsFirst ? at / per_head : at % c.n_kv;
    if (slot >= a.n_slots || head >= c.n_kv) return;
    const uint32_t pair = slot * c.n_kv + head;
    const Slots slots = find_slots(a, slot);
    const uint32_t row = slots.row;
    if (row == kNone) return;
    const uint32_t req = slots.req, n = slots.n;
    if (a.row_slots && slot == slots.first && head == 0 && tile == 0 && threadIdx.x == 0)
        *reinterpret_cast<uintx2 *>(a.row_slots + 2 * row) = uintx2{slots.first, slots.count};
    const Span span = span_of(n, a.tokens, a.window, a.sinks);
    const uint32_t per = slots.count == 1 ? span.total : (span.total + slots.count - 1) / slots.count;
    const uint32_t v0 = (slot - slots.first) * per;
    const uint32_t v1 = v0 + per < span.total ? v0 + per : span.total;
    const uint32_t query_rows = a.group * a.tokens;
    const int first_pos = (int)n - (int)a.tokens;       // of the first query

    A w{a};
    w.span = span;
    w.req = req;
    w.n = n;
    w.m = m;
    w.g = g;
    w.first_pos = first_pos;
    w.lo = a.window && first_pos >= (int)a.window ? first_pos - (int)a.window + 1 : 0;
    // sums of float16 and of 8-bit values are far from the end of 32 bits
    w.down = 1.0f;
    if constexpr (A::kWideValues) w.down = __builtin_amdgcn_ldexpf(1.0f, __builtin_clz((v1 - v0) * kBlockTokens | 1) - 32);
    w.scale = a.scale2 * (kE4m3 && c.k_scale ? c.k_scale[head] : 1.0f);
    w.table = (ScalarU32)(uint64_t)(c.table + (uint64_t)req * c.max_pages);
    w.kh = c.k + head * c.head_stride * A::kElem;
    w.vh = c.v + head * c.head_stride * A::kElem;
    w.token_bytes = (uint32_t)c.token_stride * A::kElem;
    w.k_lane = m * w.token_bytes + (kPath == kWhole ? g * 16 : 0);
    w.v_lane = g * 4 * w.token_bytes + (kPath == kWhole ? m * A::kVd * A::kElem : 0);
    {
        const uint32_t rows = query_rows - tile * kRows < (uint32_t)kRows ? query_rows - tile * kRows : kRows;
        const uint64_t first = (((uint64_t)row * c.n_kv + head) * query_rows + tile * kRows) * a.score_len;
        w.score_rsrc = __builtin_amdgcn_make_buffer_rsrc(a.scores + (a.scores ? first : 0), 0,
                                                         a.scores ? (int)(rows * a.score_len * 4) : 0, 0x00027000);
#pragma unroll
        for (int t = 0; t < kTiles; t++) w.score_lane[t] = ((t * 16 + m) * a.score_len + g * 4) * 4;
    }
    // this lane's queries (one column of each tile)
#pragma unroll
    for (int t = 0; t < kTiles; t++) {
        const uint32_t r = tile * kRows + t * 16 + m;
        const uint32_t tok = r / a.group, h = r % a.group;
        w.pos[t] = r < query_rows ? first_pos + (int)tok : -1;
        const uint16_t *src = static_cast<const uint16_t *>(a.q) + row * a.q_row + tok * a.q_token +
                              ((uint64_t)head * a.group + h) * a.q_head;
#pragma unroll
        for (int s = 0; s < A::kStepsK; s++) {
            const uint32_t d = kE4m3 ? (s >> 1) * 64 + g * 16 + (s & 1) * 8 : s * 32 + g * 8;
            w.q[t][s] = uintx4{0, 0, 0, 0};
            if (r < query_rows && d < c.dim) w.q[t][s] = *reinterpret_cast<const uintx4 *>(src + d);
        }
    }

    w.template pass<false>(v0 + wave * A::kSub, v1);
    bool odd = false;
#pragma unroll
    for (int t = 0; t < kTiles; t++)
#pragma unroll
        for (int x = 0; x < A::kOut; x++)
#pragma unroll
            for (int e = 0; e < 4; e++) odd = odd || !(fabsf(w.acc[t][x][e]) < __builtin_inff());
    if (__any(odd)) w.template pass<true>(v0 + wave * A::kSub, v1);
    auto &mx = w.mx;
    auto &sum = w.sum;
    auto &acc = w.acc;
    constexpr int kVd = A::kVd;
    const float times = T::kWeight * (__any(odd) ? w.down : 1.0f);      // acc is o times this
    // the waves' results side by side; they are joined as they are read
#pragma unroll
    for (int t = 0; t < kTiles; t++) {
        sum[t] += __shfl_xor(sum[t], 16, 64);
        sum[t] += __shfl_xor(sum[t], 32, 64);
        const float inv = sum[t] == 0.0f ? 0.0f : 1.0f / (sum[t] * times);
        if (g == 0) {
            sm_m[wave][t * 16 + m] = mx[t];
            sm_l[wave][t * 16 + m] = sum[t];
        }
#pragma unroll
        for (int h = 0; h < A::kParts; h++)
#pragma unroll
            for (int e = 0; e < 4; e++)
#pragma unroll
                for (int x = h * kVd; x < (h + 1) * kVd; x += 4)
                    *reinterpret_cast<floatx4 *>(&sm_o[wave][(t * 16 + m) * kPitch + h * 128 + (g * 4 + e) * kVd + x % kVd]) =
                        floatx4{acc[t][x][e] * inv, acc[t][x + 1][e] * inv, acc[t][x + 2][e] * inv, acc[t][x + 3][e] * inv};
    }
    __syncthreads();
    const uint32_t rows_here = query_rows - tile * kRows < (uint32_t)kRows ? query_rows - tile * kRows : kRows;
    for (uint32_t i = threadIdx.x; i < rows_here * (kDim / 4); i += 256) {
        const uint32_t rr = i / (kDim / 4), d = i % (kDim / 4) * 4;
        float top = sm_m[0][rr], l = 0.0f;
#pragma unroll
        for (int k = 1; k < 4; k++) top = fmaxf(top, sm_m[k][rr]);
        float share[4];
#pragma unroll
        for (int k = 0; k < 4; k++) {
            // a wave without tokens has a share of 0 and means of 0
            share[k] = sm_l[k][rr] * __builtin_amdgcn_exp2f(sm_m[k][rr] - finite_or_zero(top));
            l += share[k];
        }
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        floatx4 o = {0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const floatx4 x = *reinterpret_cast<const floatx4 *>(&sm_o[k][rr * kPitch + d]);
#pragma unroll
            for (int e = 0; e < 4; e++) o[e] += x[e] * (share[k] * inv);
        }
        const uint64_t at = ((uint64_t)pair * a.n_tiles + tile) * a.part_rows + rr;
        if (a.part_ml && d == 0) *reinterpret_cast<floatx2 *>(a.part_ml + 2 * at) = floatx2{top, l};
        if (slots.count > 1) {
            *reinterpret_cast<floatx4 *>(a.part_o + at * kDim + d) = o;
        } else if (d < c.dim) {
            const float times = kE4m3 && c.v_scale ? c.v_scale[head] : 1.0f;
            const uint32_t r = tile * kRows + rr, tok = r / a.group, h = r % a.group;
            uint16_t *to = static_cast<uint16_t *>(a.out) +
                           (((uint64_t)row * a.tokens + tok) * c.n_kv * a.group + (uint64_t)head * a.group + h) * c.dim + d;
            *reinterpret_cast<uintx2 *>(to) = uintx2{T::pack(o[0] * times, o[1] * times), T::pack(o[2] * times, o[3] * times)};
        }
    }
}

template <typename T, bool kE4m3, int kDim, int kTiles, bool kStream>
hipError_t attend_page(const DecodeArgs &a, hipStream_t s)
{
    const uint64_t grid = attend_grid(a);
    // lane offsets in half a block take 32 bits
    const bool pages16 = a.c.page_size % 16 == 0 && a.c.token_stride < (1u << 26);
    const bool whole = a.c.dim == kDim;
    if (pages16 && whole)
        attend_kernel<T, kE4m3, kDim, kTiles, kWhole, kStream><<<(uint32_t)grid, 256, 0, s>>>(a);
    else if (pages16)
        attend_kernel<T, kE4m3, kDim, kTiles, kPages16, false><<<(uint32_t)grid, 256, 0, s>>>(a);
    else if (kStream && whole)
        attend_kernel<T, kE4m3, kDim, kTiles, kAnyPage, kStream><<<(uint32_t)grid, 256, 0, s>>>(a);
    else
        attend_kernel<T, kE4m3, kDim, kTiles, kAnyPage, false><<<(uint32_t)grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T, bool kE4m3>
hipError_t attend(const DecodeArgs &a, hipStream_t s)
{
    const uint32_t dim = padded_dim(a.c.dim), tiles = unit_tiles(a.c.dim, a.group * a.tokens);
    if (dim == 64) return tiles == 1 ? attend_page<T, kE4m3, 64, 1, false>(a, s) : attend_page<T, kE4m3, 64, 2, false>(a, s);
    if (dim == 128 && tiles == 1) return attend_page<T, kE4m3, 128, 1, !kE4m3>(a, s);
    if (dim == 128) return a.n_tiles == 1 ? attend_page<T, kE4m3, 128, 2, !kE4m3>(a, s) : attend_page<T, kE4m3, 128, 2, false>(a, s);
    if constexpr (!kE4m3)
        if (a.n_tiles == 1) return attend_page<T, kE4m3, 256, 1, true>(a, s);
    return attend_page<T, kE4m3, 256, 1, false>(a, s);
}

}  // namespace ds
