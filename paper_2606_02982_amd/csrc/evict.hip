// Eviction from the paged cache by accumulated attention weight.
//
// Per (row, head) the kept set is a selection: the k-th largest of the masses
// that compete is found digit by digit (11, 11 and 10 bits from the top,
// counting the values that agree with the digits found so far), then one walk
// in token order keeps what is larger, and of what is equal the earliest. One
// workgroup does that; where requests may be long, three launches: digit
// counts per chunk of tokens, the sought key per (row, head) from the counts
// and the few masses that share its first digit, and the walk per chunk. The
// copy of the kept keys and values is a launch over all tokens of all rows,
// and bound by memory: 16 bytes per thread, read and written once.
#include "common.h"
#include "serve.h"

namespace ds {

constexpr int kSelect = 1024;              // threads of one selection
constexpr int kSelectWaves = kSelect / 64;

struct Cut {
    uint32_t req, n, keep;                 // keep == n: not cut
};

// What becomes of row i: its request, length and the tokens it keeps.
__device__ inline Cut cut_of(const EvictArgs &a, uint32_t row, bool *refused = nullptr)
{
    Cut x;
    x.req = a.rows ? a.rows[row] : row;
    x.n = x.req < a.src.n_requests ? a.src.len[x.req] : 0;
    if (x.n > a.src.cap) x.n = a.src.cap;
    x.keep = x.n;
    const double budget = x.req < a.src.n_requests ? a.budget[x.req] : __builtin_nan("");
    if (budget < (double)x.n) {            // false for NaN
        uint64_t keep = budget > 0.0 ? (uint64_t)budget : 0;
        const uint64_t least = (uint64_t)a.sinks + a.recent;
        keep = keep > least ? keep : least;
        if (x.n > keep + a.slack) {
            const bool fits = keep <= a.kept_len && keep <= (uint64_t)a.dst.max_pages * a.dst.page_size;
            if (fits) x.keep = (uint32_t)keep;
            if (!fits && refused) *refused = true;
        }
    }
    return x;
}

// A float as an unsigned integer in the same order; NaN below everything,
// -0 as +0.
__device__ __forceinline__ uint32_t mass_key(float x)
{
    if (x != x) return 0u;
    const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);
    return (u >> 31) ? ~u : (u | 0x80000000u);
}

typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
typedef uint32_t uintx2 __attribute__((ext_vector_type(2)));

constexpr int kBins = 2048;
constexpr int kCopies = 4;                 // of the digit counts: sixteen lanes share one, equal masses
                                           // (zeros are common) meet in an atomic no more often
constexpr int kCopyPitch = kBins + 16;     // the copies of a bin lie in different banks
// Requests that may be longer are selected from in chunks (with the copy of
// half of 16 dimensions, 8 heads; one row / 8 rows, in one workgroup and in
// chunks: 16,384 tokens 29 / 90 and 33 / 95 us, 24,576 38 / 133 and 38 / 134,
// 32,768 48 / 179 and 44 / 176, 100,000 139 / 564 and 98 / 537 us).
constexpr uint32_t kLongTokens = 24576;
constexpr uint32_t kMaxChunks = 256;
constexpr uint32_t kCopyGroups = 1u << 23; // workgroups of a copy, where there are no more (row, head)
constexpr int kAhead = 8;                  // groups of 64 tokens under way per wave
constexpr uint32_t kList = 8192;           // masses with the first digit sought that fit into LDS
struct Select {
    uintx4 hist4[kCopyPitch * kCopies / 4];
    uint32_t list[kList], listed, wave_total[kSelectWaves], pick[3], gt_of[kSelectWaves], eq_of[kSelectWaves];
};

// The largest digit d such that `want` of the counted values have a digit of
// at least d: pick[0] = d, pick[1] = how many of digit d itself are wanted,
// pick[2] = how many have it.
__device__ inline void pick_digit(Select &sm, uint32_t want)
{
    // thread t adds up bins 2047 - 2 t and 2046 - 2 t
    const int wave = threadIdx.x >> 6, top = kBins - 1 - 2 * (int)threadIdx.x;
    uint32_t h[2] = {0, 0};
#pragma unroll
    for (int c = 0; c < kCopies; c++) {
        const uintx2 x = *reinterpret_cast<const uintx2 *>(reinterpret_cast<const uint32_t *>(sm.hist4) + c * kCopyPitch + top - 1);
        h[0] += x[1];
        h[1] += x[0];
    }
    const uint32_t incl = wave_incl_scan_dpp(h[0] + h[1]);
    if (lane_id() == 63) sm.wave_total[wave] = incl;
    __syncthreads();
    uint32_t before = incl - h[0] - h[1];
    for (int w = 0; w < wave; w++) before += sm.wave_total[w];
#pragma unroll
    for (int k = 0; k < 2; k++) {
        if (before < want && want <= before + h[k]) {
            sm.pick[0] = top - k;
            sm.pick[1] = want - before;
            sm.pick[2] = h[k];
        }
        before += h[k];
    }
    __syncthreads();
}

// The selection of one (row, head) by 16 waves. Each wave owns a run of
// tokens in groups of 64. The masses that have
// the first digit sought are listed in LDS if they fit there, and the other
// digits found from the list. Its time goes into the passes over the masses
// on one compute unit (24 selections of 60,000 to 100,000 tokens 90 us; 256
// of 2,048 to 6,144 17 us) and, for few tokens, into a chain of barriers
// (700 tokens 9 us; with all counts of a bin in one bank 21 us).
// A request that stands in two rows, against the contract, is compacted in
// place by one workgroup while another still selects, so that what one pass
// counted the next may not find again: places in the list, in kept and among
// the masses are therefore held in their bounds one by one.
__device__ inline void select_tokens(const EvictArgs &a, const Cut &x, const float *mass, float *mass_out, uint32_t *kept, Select &sm)
{
    const uint32_t n = x.n, lo = a.sinks, span = n - a.recent - a.sinks;   // the tokens that compete
    uint32_t want = x.keep - a.sinks - a.recent;                           // how many of them stay
    const int wave = threadIdx.x >> 6, lane = lane_id();
    const uint32_t run = (uint32_t)align_up(cdiv(n, kSelectWaves), 64);
    const uint32_t w0 = wave * run < n ? wave * run : n, w1 = w0 + run < n ? w0 + run : n;

    // f(token, mass) for every group of 64 tokens, one per lane, in order;
    // tokens from n on come with any mass. The loads of kAhead groups are
    // issued at once and without conditions, so that one wait serves them all.
    auto groups = [&](auto &&f) {
#pragma unroll 1
        for (uint32_t j = w0; j < w1; j += 64 * kAhead) {
            float v[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; i++) {
                const uint32_t at = j + i * 64 + lane;
                v[i] = mass[at < n ? at : n - 1];
            }
#pragma unroll
            for (int i = 0; i < kAhead; i++)
                if (j + i * 64 < w1) f(j + i * 64 + lane, v[i]);
        }
    };
    auto clear = [&]() {
        for (int i = threadIdx.x; i < kCopyPitch * kCopies / 4; i += kSelect) sm.hist4[i] = uintx4{0, 0, 0, 0};
        __syncthreads();
    };
    auto count = [&](uint32_t digit) {
        atomicAdd(reinterpret_cast<uint32_t *>(sm.hist4) + (lane & (kCopies - 1)) * kCopyPitch + digit, 1u);
    };

    uint32_t bar = 0xFFFFFFFFu;            // the smallest kept key; of it the first `want` stay
    if (want) {
        if (threadIdx.x == 0) sm.listed = 0;
        clear();
        groups([&](uint32_t j, float v) {
            if (j - lo < span) count(mass_key(v) >> 21);
        });
        __syncthreads();
        pick_digit(sm, want);
        uint32_t found = sm.pick[0];       // the digits of bar so far
        want = sm.pick[1];
        const bool fits = sm.pick[2] <= kList;
        if (fits) {
            groups([&](uint32_t j, float v) {
                const uint32_t key = mass_key(v);
                const bool on = j - lo < span && key >> 21 == found;
                const uint64_t all = __ballot(on);
                if (!all) return;
                uint32_t to = 0;
                if (lane == 0) to = atomicAdd(&sm.listed, (uint32_t)__popcll(all));
                to = readlane32(to, 0) + (uint32_t)__popcll(all & lanemask_lt());
                if (on && to < kList) sm.list[to] = key;
            });
            __syncthreads();
        }
        const uint32_t listed = sm.listed < kList ? sm.listed : kList;
#pragma unroll 1
        for (int shift = 10; shift >= 0; shift -= 10) {
            // bits 20 .. 10, then 9 .. 0
            const uint32_t mask = shift ? 2047u : 1023u;
            const int above = shift ? 21 : 10;
            clear();
            auto look = [&](uint32_t key) {
                if (key >> above == found) count((key >> shift) & mask);
            };
            if (fits)
                for (uint32_t i = threadIdx.x; i < listed; i += kSelect) look(sm.list[i]);
            else
                groups([&](uint32_t j, float v) {
                    if (j - lo < span) look(mass_key(v));
                });
            __syncthreads();
            pick_digit(sm, want);
            found = found << (shift ? 11 : 10) | sm.pick[0];
            want = sm.pick[1];
        }
        bar = found;
    }

    // kept tokens in their order: of every wave's run how many, then where
    auto state = [&](uint32_t j, float v, bool &gt, bool &eq) {
        const uint32_t key = mass_key(v);
        const bool competes = j - lo < span;
        gt = competes ? key > bar : j < n;
        eq = competes && want && key == bar;
    };
    uint32_t n_gt = 0, n_eq = 0;
    groups([&](uint32_t j, float v) {
        bool gt, eq;
        state(j, v, gt, eq);
        n_gt += (uint32_t)__popcll(__ballot(gt));
        n_eq += (uint32_t)__popcll(__ballot(eq));
    });
    if (lane == 0) {
        sm.gt_of[wave] = n_gt;
        sm.eq_of[wave] = n_eq;
    }
    __syncthreads();
    uint32_t at = 0, eq_at = 0;
    for (int w = 0; w < wave; w++) {
        const uint32_t left = eq_at < want ? want - eq_at : 0;
        at += sm.gt_of[w] + (sm.eq_of[w] < left ? sm.eq_of[w] : left);
        eq_at += sm.eq_of[w];
    }
    const bool direct = mass_out != mass;
    groups([&](uint32_t j, float v) {
        bool stays, eq;
        state(j, v, stays, eq);
        if (const uint64_t eqs = __ballot(eq)) {
            stays = stays || (eq && eq_at + (uint32_t)__popcll(eqs & lanemask_lt()) < want);
            eq_at += (uint32_t)__popcll(eqs);
        }
        const uint64_t all = __ballot(stays);
        const uint32_t to = at + (uint32_t)__popcll(all & lanemask_lt());
        if (stays && to < x.keep) {
            kept[to] = j;
            if (direct) mass_out[to] = v;
        }
        at += (uint32_t)__popcll(all);
    });
    if (direct) return;
    // kept[i] >= i: reading a piece before writing it is enough
    __syncthreads();
    constexpr int kPiece = 8;
    for (uint32_t i = 0; i < x.keep; i += kSelect * kPiece) {
        float v[kPiece];
#pragma unroll
        for (int k = 0; k < kPiece; k++) {
            const uint32_t p = i + k * kSelect + threadIdx.x;
            const uint32_t from = p < x.keep ? kept[p] : 0;
            v[k] = from < n ? mass[from] : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kPiece; k++) {
            const uint32_t p = i + k * kSelect + threadIdx.x;
            if (p < x.keep) mass_out[p] = v[k];
        }
        __syncthreads();
    }
}

// The same in chunks. Every chunk is a multiple of 1,024 tokens; all
// workgroups have 16 waves.
struct ChunkOf {
    uint32_t chunk, head, row;
    uint64_t pair;
};
__device__ inline ChunkOf chunk_of(const EvictArgs &a)
{
    ChunkOf c;
    c.chunk = blockIdx.x % a.n_chunks;
    c.pair = blockIdx.x / a.n_chunks;
    c.head = (uint32_t)(c.pair % a.src.n_kv);
    c.row = (uint32_t)(c.pair / a.src.n_kv);
    return c;
}

__global__ __launch_bounds__(kSelect) void count_kernel(const EvictArgs a)
{
    __shared__ uintx4 hist4[kCopyPitch * kCopies / 4];
    uint32_t *hist = reinterpret_cast<uint32_t *>(hist4);
    const ChunkOf c = chunk_of(a);
    const Cut x = cut_of(a, c.row);
    if (threadIdx.x == 0 && c.head == 0 && c.chunk == 0) a.dst.len[c.row] = x.keep;
    const uint32_t j0 = c.chunk * a.chunk_tokens, j1 = j0 + a.chunk_tokens < x.n ? j0 + a.chunk_tokens : x.n;
    if (x.keep == x.n || j0 >= x.n) return;
    for (int i = threadIdx.x; i < kCopyPitch * kCopies / 4; i += kSelect) hist4[i] = uintx4{0, 0, 0, 0};
    __syncthreads();
    const float *mass = a.mass + ((uint64_t)x.req * a.src.n_kv + c.head) * a.mass_len;
    const uint32_t span = x.n - a.recent - a.sinks;
    for (uint32_t j = j0; j < j1; j += kSelect * kAhead) {
        float v[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; i++) {
            const uint32_t at = j + i * kSelect + threadIdx.x;
            v[i] = mass[at < x.n ? at : x.n - 1];
        }
#pragma unroll
        for (int i = 0; i < kAhead; i++) {
            const uint32_t at = j + i * kSelect + threadIdx.x;
            if (at < j1 && at - a.sinks < span)
                atomicAdd(&hist[(threadIdx.x & (kCopies - 1)) * kCopyPitch + (mass_key(v[i]) >> 21)], 1u);
        }
    }
    __syncthreads();
    uint32_t *to = a.counts + (c.pair * a.n_chunks + c.chunk) * kBins;
    for (int b = threadIdx.x; b < kBins; b += kSelect) {
        uint32_t h = 0;
#pragma unroll
        for (int k = 0; k < kCopies; k++) h += hist[k * kCopyPitch + b];
        to[b] = h;
    }
}

struct Threshold {
    Select s;
    uint32_t gt[kMaxChunks], eq[kMaxChunks];
    uint32_t token[kList];
};

__global__ __launch_bounds__(kSelect) void threshold_kernel(const EvictArgs a)
{
    __shared__ Threshold sm;
    const uint32_t row = blockIdx.x / a.src.n_kv, head = blockIdx.x % a.src.n_kv;
    const Cut x = cut_of(a, row);
    if (x.keep == x.n) return;
    const int wave = threadIdx.x >> 6, lane = lane_id();
    const float *mass = a.mass + ((uint64_t)x.req * a.src.n_kv + head) * a.mass_len;
    const uint32_t *counts = a.counts + (uint64_t)blockIdx.x * a.n_chunks * kBins;
    uint32_t *hist = reinterpret_cast<uint32_t *>(sm.s.hist4);
    const uint32_t n = x.n, lo = a.sinks, span = n - a.recent - a.sinks;
    const uint32_t chunks = (uint32_t)cdiv(n, a.chunk_tokens);
    uint32_t want = x.keep - a.sinks - a.recent;

    auto clear = [&]() {
        for (int i = threadIdx.x; i < kCopyPitch * kCopies / 4; i += kSelect) sm.s.hist4[i] = uintx4{0, 0, 0, 0};
        __syncthreads();
    };
    for (uint32_t k = threadIdx.x; k < kMaxChunks; k += kSelect) sm.gt[k] = sm.eq[k] = 0;
    if (threadIdx.x == 0) sm.s.listed = 0;
    uint32_t bar = 0xFFFFFFFFu;
    if (want) {
        clear();
        {
            uintx2 h = {0, 0};
#pragma unroll 8
            for (uint32_t k = 0; k < chunks; k++) {
                const uintx2 y = *reinterpret_cast<const uintx2 *>(counts + (uint64_t)k * kBins + 2 * threadIdx.x);
                h[0] += y[0];
                h[1] += y[1];
            }
            hist[2 * threadIdx.x] = h[0];
            hist[2 * threadIdx.x + 1] = h[1];
        }
        __syncthreads();
        pick_digit(sm.s, want);
        uint32_t found = sm.s.pick[0];
        want = sm.s.pick[1];
        const bool fits = sm.s.pick[2] <= kList;
        // every chunk's masses of a larger first digit
        for (uint32_t k = wave; k < chunks; k += kSelectWaves) {
            uint32_t c = 0;
            for (uint32_t b = found + 1 + lane; b < kBins; b += 64) c += counts[(uint64_t)k * kBins + b];
            c = wave_sum(c);
            if (lane == 0) sm.gt[k] = c;
        }
        // f(token, key) for the masses of the first digit sought, all waves
        // side by side
        const uint32_t first = found;
        auto scan = [&](auto &&f) {
#pragma unroll 1
            for (uint32_t j = 0; j < n; j += kSelect * 2 * kAhead) {
                float v[2 * kAhead];
#pragma unroll
                for (int i = 0; i < 2 * kAhead; i++) {
                    const uint32_t at = j + i * kSelect + threadIdx.x;
                    v[i] = mass[at < n ? at : n - 1];
                }
#pragma unroll
                for (int i = 0; i < 2 * kAhead; i++) {
                    const uint32_t at = j + i * kSelect + threadIdx.x, key = mass_key(v[i]);
                    f(at, key, at - lo < span && key >> 21 == first);
                }
            }
        };
        if (fits)
            scan([&](uint32_t j, uint32_t key, bool on) {
                const uint64_t all = __ballot(on);
                if (!all) return;
                uint32_t to = 0;
                if (lane == 0) to = atomicAdd(&sm.s.listed, (uint32_t)__popcll(all));
                to = readlane32(to, 0) + (uint32_t)__popcll(all & lanemask_lt());
                if (on) {
                    sm.s.list[to] = key;
                    sm.token[to] = j;
                }
            });
        __syncthreads();
        auto each = [&](auto &&f) {
            if (fits)
                for (uint32_t i = threadIdx.x; i < sm.s.listed; i += kSelect) f(sm.token[i], sm.s.list[i]);
            else
                scan([&](uint32_t j, uint32_t key, bool on) {
                    if (on) f(j, key);
                });
        };
#pragma unroll 1
        for (int shift = 10; shift >= 0; shift -= 10) {
            // bits 20 .. 10, then 9 .. 0
            const uint32_t mask = shift ? 2047u : 1023u;
            const int above = shift ? 21 : 10;
            clear();
            each([&](uint32_t, uint32_t key) {
                if (key >> above == found) atomicAdd(&hist[(lane & (kCopies - 1)) * kCopyPitch + ((key >> shift) & mask)], 1u);
            });
            __syncthreads();
            pick_digit(sm.s, want);
            found = found << (shift ? 11 : 10) | sm.s.pick[0];
            want = sm.s.pick[1];
        }
        bar = found;
        each([&](uint32_t j, uint32_t key) {
            if (key >= bar) atomicAdd(key > bar ? &sm.gt[j / a.chunk_tokens] : &sm.eq[j / a.chunk_tokens], 1u);
        });
    }
    __syncthreads();
    // kept and equal tokens before each chunk (kMaxChunks = four waves' lanes)
    const uint32_t t = threadIdx.x;
    uint32_t eq = 0, gt = 0;
    if (t < chunks) {
        const uint32_t j0 = t * a.chunk_tokens, j1 = j0 + a.chunk_tokens < n ? j0 + a.chunk_tokens : n, hi = lo + span;
        eq = sm.eq[t];
        gt = sm.gt[t];
        if (j0 < lo) gt += (j1 < lo ? j1 : lo) - j0;                    // the first tokens
        if (j1 > hi) gt += j1 - (j0 > hi ? j0 : hi);                    // the last ones
    }
    __syncthreads();
    const uint32_t eq_incl = wave_incl_scan_dpp(eq);
    if (lane == 63) sm.s.wave_total[wave] = eq_incl;
    __syncthreads();
    uint32_t eq_before = eq_incl - eq;
    for (int w = 0; w < wave; w++) eq_before += sm.s.wave_total[w];
    __syncthreads();
    const uint32_t left = eq_before < want ? want - eq_before : 0;
    const uint32_t stay = gt + (eq < left ? eq : left), incl = wave_incl_scan_dpp(stay);
    if (lane == 63) sm.s.wave_total[wave] = incl;
    __syncthreads();
    uint32_t before = incl - stay;
    for (int w = 0; w < wave; w++) before += sm.s.wave_total[w];
    if (t < chunks) {
        uint32_t *to = a.starts + ((uint64_t)blockIdx.x * a.n_chunks + t) * 2;
        to[0] = before;
        to[1] = eq_before;
    }
    if (t == 0) {
        a.bars[2 * (uint64_t)blockIdx.x] = bar;
        a.bars[2 * (uint64_t)blockIdx.x + 1] = want;
    }
}

__global__ __launch_bounds__(kSelect) void walk_kernel(const EvictArgs a)
{
    __shared__ uint32_t gt_of[kSelectWaves], eq_of[kSelectWaves];
    const ChunkOf c = chunk_of(a);
    const Cut x = cut_of(a, c.row);
    const uint32_t j0 = c.chunk * a.chunk_tokens, j1 = j0 + a.chunk_tokens < x.n ? j0 + a.chunk_tokens : x.n;
    if (x.keep == x.n || j0 >= x.n) return;
    const int wave = threadIdx.x >> 6, lane = lane_id();
    const float *mass = a.mass + ((uint64_t)x.req * a.src.n_kv + c.head) * a.mass_len;
    uint32_t *kept = a.kept + c.pair * a.kept_len;
    float *kept_mass = a.kept_mass + c.pair * a.most_kept;
    const uint32_t bar = a.bars[2 * c.pair], want = a.bars[2 * c.pair + 1], lo = a.sinks, span = x.n - a.recent - a.sinks;
    uint32_t at = a.starts[(c.pair * a.n_chunks + c.chunk) * 2], eq_at = a.starts[(c.pair * a.n_chunks + c.chunk) * 2 + 1];
    // each wave owns a run of the chunk
    const uint32_t run = a.chunk_tokens / kSelectWaves, w0 = j0 + wave * run;
    auto walk = [&](auto &&f) {
#pragma unroll 1
        for (uint32_t j = w0; j < w0 + run && j < j1; j += 64 * kAhead) {
            float v[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; i++) {
                const uint32_t t = j + i * 64 + lane;
                v[i] = mass[t < x.n ? t : x.n - 1];
            }
#pragma unroll
            for (int i = 0; i < kAhead; i++) {
                const uint32_t t = j + i * 64 + lane, key = mass_key(v[i]);
                if (j + i * 64 >= w0 + run) break;
                const bool in = t < j1, competes = t - lo < span;
                f(t, v[i], in && (!competes || key > bar), in && competes && want && key == bar);
            }
        }
    };
    uint32_t n_gt = 0, n_eq = 0;
    walk([&](uint32_t, float, bool gt, bool eq) {
        n_gt += (uint32_t)__popcll(__ballot(gt));
        n_eq += (uint32_t)__popcll(__ballot(eq));
    });
    if (lane == 0) {
        gt_of[wave] = n_gt;
        eq_of[wave] = n_eq;
    }
    __syncthreads();
    for (int w = 0; w < wave; w++) {
        const uint32_t left = eq_at < want ? want - eq_at : 0;
        at += gt_of[w] + (eq_of[w] < left ? eq_of[w] : left);
        eq_at += eq_of[w];
    }
    walk([&](uint32_t j, float v, bool gt, bool eq) {
        bool stays = gt;
        if (const uint64_t eqs = __ballot(eq)) {
            stays = stays || (eq && eq_at + (uint32_t)__popcll(eqs & lanemask_lt()) < want);
            eq_at += (uint32_t)__popcll(eqs);
        }
        const uint64_t all = __ballot(stays);
        const uint32_t to = at + (uint32_t)__popcll(all & lanemask_lt());
        if (stays) {
            kept[to] = j;
            kept_mass[to] = v;
        }
        at += (uint32_t)__popcll(all);
    });
}

__global__ __launch_bounds__(kSelect) void select_kernel(const EvictArgs a)
{
    __shared__ Select sm;
    const uint32_t row = blockIdx.x / a.src.n_kv, head = blockIdx.x % a.src.n_kv;
    const Cut x = cut_of(a, row);
    if (threadIdx.x == 0 && head == 0) a.dst.len[row] = x.keep;
    if (x.keep == x.n) return;
    const uint64_t of = ((uint64_t)x.req * a.src.n_kv + head) * a.mass_len;
    uint32_t *kept = a.kept + ((uint64_t)row * a.src.n_kv + head) * a.kept_len;
    select_tokens(a, x, a.mass + of, a.mass_out + of, kept, sm);
}

// 16 bytes; whole lines go past the caches: nothing is read twice.
template <bool kShared>
__device__ __forceinline__ void put(uint8_t *to, const uint8_t *from)
{
    const uintx4 *f = reinterpret_cast<const uintx4 *>(from);
    uintx4 *t = reinterpret_cast<uintx4 *>(to);
    if constexpr (kShared)
        *t = *f;
    else
        __builtin_nontemporal_store(__builtin_nontemporal_load(f), t);
}

// 16 bytes of a key or value per thread and step; `groups` workgroups share a
// (row, head) in pieces of `tokens` kept tokens. kShared: a head's bytes end
// inside a cache line, so neighbouring heads share lines. They go through the
// caches, and the heads of one piece to one die (dies take workgroups in turn)
// (32 rows of 2,000 to 6,000 tokens, 8 heads, kShared / not: 80 dimensions in
// 16 bits 97 / 148 us, in 8 bits 76 / 118, 64 in 8 bits 56 / 64; 128 in 16
// bits 121 / 116). Taken from 64 pieces of all rows on, eight for each die (80
// dimensions in 16 bits, whole call, kShared / not: 16 rows of 2,000 tokens
// 34.6 / 38.5 us, 3 rows, 72 pieces, 17.5 / 19.2; below, 2 rows, 48 pieces,
// 16.6 / 17.9, one row, 24 pieces, 15.0 / 15.0).
template <bool kShared>
__global__ __launch_bounds__(256) void copy_kernel(const EvictArgs a, uint32_t groups, uint32_t tokens, uint32_t elem)
{
    const uint32_t n_kv = a.src.n_kv;
    uint32_t head, piece, row;
    if constexpr (kShared) {
        const uint32_t unit = blockIdx.x / 8 / n_kv * 8 + blockIdx.x % 8;
        head = blockIdx.x / 8 % n_kv;
        piece = unit % groups;
        row = unit / groups;
        if (row >= a.n_rows) return;
    } else {
        piece = blockIdx.x % groups;
        head = blockIdx.x / groups % n_kv;
        row = blockIdx.x / groups / n_kv;
    }
    const uint32_t pair = row * n_kv + head;
    const Cut x = cut_of(a, row);
    if (x.keep == x.n) return;
    const KvView &s = a.src, &d = a.dst;
    const uint32_t *kept = a.kept + (uint64_t)pair * a.kept_len;
    const uint32_t units = s.dim * elem / 16;
    for (uint32_t first = piece * tokens; first < x.keep; first += groups * tokens) {
        const uint32_t left = x.keep - first, count = left < tokens ? left : tokens;
        if (a.n_chunks && threadIdx.x < count) {
            // the chunks' walks may not write into masses that others still read
            const uint32_t to = first + threadIdx.x;
            a.mass_out[((uint64_t)x.req * s.n_kv + head) * a.mass_len + to] = a.kept_mass[(uint64_t)pair * a.most_kept + to];
        }
        for (uint32_t i = threadIdx.x; i < count * units; i += 256) {
            const uint32_t to = first + i / units, from = kept[to], u = i % units;
            if (from >= x.n) continue;     // an entry that no selection wrote (select_tokens)
            const uint32_t sp = s.table[(uint64_t)x.req * s.max_pages + from / s.page_size];
            const uint32_t dp = d.table[(uint64_t)row * d.max_pages + to / d.page_size];
            if (sp >= s.n_pages || dp >= d.n_pages) continue;
            const uint64_t sa = (sp * s.page_stride + (from % s.page_size) * s.token_stride + head * s.head_stride) * elem + u * 16;
            const uint64_t da = (dp * d.page_stride + (to % d.page_size) * d.token_stride + head * d.head_stride) * elem + u * 16;
            put<kShared>(d.k + da, s.k + sa);
            put<kShared>(d.v + da, s.v + sa);
        }
    }
}

void evict_plan(EvictArgs &a)
{
    uint64_t most = (uint64_t)a.dst.max_pages * a.dst.page_size;
    if (most > a.kept_len) most = a.kept_len;
    if (most > a.src.cap) most = a.src.cap;
    a.most_kept = (uint32_t)most;
    a.n_chunks = 0;
    a.chunk_tokens = 8192;
    if (a.src.cap > kLongTokens) {
        if (a.src.cap > kMaxChunks * a.chunk_tokens) a.chunk_tokens = (uint32_t)align_up(cdiv(a.src.cap, kMaxChunks), 1024);
        a.n_chunks = (uint32_t)cdiv(a.src.cap, a.chunk_tokens);
    }
}

static uint64_t chunks_of(const EvictArgs &a) { return (uint64_t)a.n_rows * a.src.n_kv * a.n_chunks; }

size_t evict_ws_bytes(const EvictArgs &a)
{
    if (!a.n_chunks) return 0;
    const uint64_t pairs = (uint64_t)a.n_rows * a.src.n_kv;
    return chunks_of(a) * kBins * 4 + align_up(chunks_of(a) * 8, 256) + align_up(pairs * 8, 256) + align_up(pairs * a.most_kept * 4, 256);
}

hipError_t evict_launch(EvictArgs a, void *ws, hipStream_t s)
{
    const uint32_t pairs = a.n_rows * a.src.n_kv;
    hipError_t e;
    if (a.n_chunks) {
        uint8_t *p = static_cast<uint8_t *>(ws);
        a.counts = reinterpret_cast<uint32_t *>(p);
        p += chunks_of(a) * kBins * 4;
        a.starts = reinterpret_cast<uint32_t *>(p);
        p += align_up(chunks_of(a) * 8, 256);
        a.bars = reinterpret_cast<uint32_t *>(p);
        p += align_up((uint64_t)pairs * 8, 256);
        a.kept_mass = reinterpret_cast<float *>(p);
        const uint32_t grid = pairs * a.n_chunks;
        count_kernel<<<grid, kSelect, 0, s>>>(a);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        threshold_kernel<<<pairs, kSelect, 0, s>>>(a);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        walk_kernel<<<grid, kSelect, 0, s>>>(a);
    } else {
        select_kernel<<<pairs, kSelect, 0, s>>>(a);
    }
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    // tokens of one workgroup of the copy: 8 KB of keys, two rounds of its threads
    const uint32_t elem = a.src.type == DS_E4M3 ? 1 : 2, bytes = a.src.dim * elem;
    const uint32_t tokens = bytes >= 256 ? 32 : bytes <= 32 ? 256 : 8192 / bytes;
    const uint32_t chunks = (uint32_t)cdiv(a.most_kept, tokens);
    if (!chunks) return hipSuccess;
    const uint32_t share = kCopyGroups / pairs ? kCopyGroups / pairs : 1, groups = chunks < share ? chunks : share;
    if (bytes % 128 && a.n_rows * groups >= 64)        // pieces for every die
        copy_kernel<true><<<(uint32_t)align_up(a.n_rows * groups, 8) * a.src.n_kv, 256, 0, s>>>(a, groups, tokens, elem);
    else
        copy_kernel<false><<<pairs * groups, 256, 0, s>>>(a, groups, tokens, elem);
    return hipGetLastError();
}

__global__ void evict_check_kernel(const EvictArgs a, uint32_t *flag)
{
    for (uint32_t i = blockIdx.x; i < a.n_rows; i += gridDim.x) {
        bool bad = false;
        const Cut x = cut_of(a, i, &bad);
        if (x.keep != x.n)
            for (uint32_t p = threadIdx.x; p < (uint32_t)cdiv(x.keep, a.dst.page_size); p += blockDim.x)
                bad = bad || a.dst.table[(uint64_t)i * a.dst.max_pages + p] >= a.dst.n_pages;
        if (bad) atomicOr(flag, 1u);
    }
}

hipError_t evict_check(const EvictArgs &a, uint32_t *flag, hipStream_t s)
{
    hipError_t e = cache_check(a.src, a.rows, a.n_rows, true, flag, s);
    if (e != hipSuccess) return e;
    evict_check_kernel<<<a.n_rows < 4096 ? a.n_rows : 4096, 256, 0, s>>>(a, flag);
    return hipGetLastError();
}

}  // namespace ds
