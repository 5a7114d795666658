// Attention over the paged cache: the split over the cache's length, the join
// of the splits, the weight per cached token, and the checks of the device
// data. The attention itself is in attend.h.
#include "attend.h"
#include "kernels.h"

namespace ds {

// Units of a launch, where the caches are long enough. More of them even out
// the end of a launch, each costs a start, and a partial result per query
// row: 32 rows of 8,192 tokens, 8 heads, units 1024 / 1536 / 2048: 256
// dimensions in 16 bits 348 / 358 / 362 us, 64 dimensions 119 / 113 / 108 us,
// 128 in 8 bits 118 / 117 / 113 us, 40 query rows 268 / 274 / 276 us; three
// rows of up to 131,072 tokens, 128 dimensions in 16 bits 264 / 251 / 255 us.
static uint32_t unit_goal(uint32_t key_bytes, uint32_t unit_tiles)
{
    return unit_tiles > 1 || key_bytes > 256 ? 1024 : key_bytes > 128 ? 1536 : 2048;
}
constexpr uint32_t kMassTokens = 1024;     // tokens of one workgroup of the weights' sum
constexpr uint32_t kMaxQueryRows = DS_MAX_QUERY_ROWS;

void decode_plan(DecodeArgs &a)
{
    const uint32_t query_rows = a.group * a.tokens, unit_rows = 16 * unit_tiles(a.c.dim, query_rows);
    a.n_tiles = (uint32_t)cdiv(query_rows, unit_rows);
    a.part_rows = a.n_tiles == 1 ? query_rows : unit_rows;
    const uint32_t key_bytes = a.c.dim * (a.c.type == DS_E4M3 ? 1 : 2);
    uint64_t blocks = cdiv(a.c.cap, kBlockTokens);
    if (a.window) {
        const uint64_t seen = cdiv(a.sinks, kBlockTokens) + cdiv((uint64_t)a.window + a.tokens + kBlockTokens - 2, kBlockTokens);
        blocks = blocks < seen ? blocks : seen;
    }
    a.score_len = (uint32_t)blocks * kBlockTokens;
    // two steps per wave; four where a step has two tiles of query rows and
    // only two workgroups fit a compute unit (16 rows of 1,024 visible tokens
    // and 40 query rows: 640 workgroups in two rounds 27 us, 384 in one 19 us)
    a.slot_blocks = unit_rows > 16 ? 16 : 8;
    // no row can be cut, or more rows than each workgroup looks through: one slot each
    a.slot_goal = blocks > a.slot_blocks && a.n_rows <= kBalancedRows ? (uint32_t)cdiv(unit_goal(key_bytes, unit_rows / 16), a.c.n_kv * a.n_tiles) : 0;
    a.n_slots = a.n_rows;
    if (a.slot_goal) {
        // ceil(total / most) <= total / most + 1 per row
        const uint64_t most = (uint64_t)a.n_rows * cdiv(blocks, a.slot_blocks);
        a.n_slots = (uint32_t)(a.slot_goal + a.n_rows < most ? a.slot_goal + a.n_rows : most);
    }
    // a die per slot where every die gets several (attend_kernel)
    a.spread = (key_bytes <= 128 || key_bytes % 128) && a.n_slots >= 64 ? kDieOfSlot : a.c.n_kv <= 8 ? kSlotsFirst : kHeadsFirst;
}

static uint64_t part_rows_of(const DecodeArgs &a) { return (uint64_t)a.n_slots * a.c.n_kv * a.n_tiles * a.part_rows; }

size_t decode_ws_bytes(const DecodeArgs &a, bool with_mass)
{
    size_t b = 0;
    if (a.slot_goal) b += align_up(part_rows_of(a) * padded_dim(a.c.dim) * 4, 256);
    if (a.slot_goal || with_mass) b += align_up(part_rows_of(a) * 8, 256) + align_up((uint64_t)a.n_rows * 8, 256);
    if (with_mass) b += align_up((uint64_t)a.n_rows * a.c.n_kv * a.group * a.tokens * a.score_len * 4, 256);
    return b;
}

// Partial result of query row r in slot `slot` of a head, in rows; the slots
// of a row lie n_kv * n_tiles * part_rows apart.
__device__ __forceinline__ uint64_t part_at(const DecodeArgs &a, uint32_t slot, uint32_t head, uint32_t r, uint32_t unit_rows)
{
    return (((uint64_t)slot * a.c.n_kv + head) * a.n_tiles + r / unit_rows) * a.part_rows + r % unit_rows;
}

// Maximum and sum over the slots of one query row, by kLanes adjacent lanes.
template <int kLanes>
__device__ inline floatx2 join_ml(const float *ml, uint64_t stride, uint32_t slots)
{
    const uint32_t t = threadIdx.x % kLanes;
    floatx2 x = {-__builtin_inff(), 0.0f};
    for (uint32_t s = t; s < slots; s += kLanes) {
        const floatx2 y = *reinterpret_cast<const floatx2 *>(ml + 2 * s * stride);
        const float top = finite_or_zero(fmaxf(x[0], y[0]));
        x = floatx2{fmaxf(x[0], y[0]), x[1] * __builtin_amdgcn_exp2f(x[0] - top) + y[1] * __builtin_amdgcn_exp2f(y[0] - top)};
    }
    float top = x[0];
#pragma unroll
    for (int d = kLanes / 2; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    float l = x[1] * __builtin_amdgcn_exp2f(x[0] - finite_or_zero(top));
#pragma unroll
    for (int d = kLanes / 2; d >= 1; d >>= 1) l += __shfl_xor(l, d, 64);
    return floatx2{top, l};
}

// The first n_rows * n_kv * query rows workgroups (none where no row is cut)
// join the slots of one query row each; the others sum the weights of
// kMassTokens tokens. Both are chains of a few loads from what other dies
// wrote, a microsecond each, so each chain is kept short and there are many.
template <typename T, int kDim>
__global__ __launch_bounds__(256) void join_kernel(const DecodeArgs a, uint32_t join_groups, uint32_t mass_groups,
                                                   uint32_t unit_rows)
{
    constexpr int kLanes = kDim / 4;                  // lanes of one partial row
    constexpr int kTeams = 256 / kLanes;
    const KvView &c = a.c;
    const uint32_t query_rows = a.group * a.tokens;
    const uint64_t stride = (uint64_t)c.n_kv * a.n_tiles * a.part_rows;
    if (blockIdx.x < join_groups) {
        __shared__ __align__(16) float sm_o[kTeams][kDim];
        const uint32_t r = blockIdx.x % query_rows, head = blockIdx.x / query_rows % c.n_kv;
        const uint32_t row = blockIdx.x / query_rows / c.n_kv;
        const uint32_t first = a.row_slots[2 * row], count = a.row_slots[2 * row + 1];
        if (count == 1) return;
        const uint64_t at = part_at(a, first, head, r, unit_rows);
        const uint32_t team = threadIdx.x / kLanes, d = threadIdx.x % kLanes * 4;
        const float *from = a.part_o + at * kDim + d, *m = a.part_ml + 2 * at;
        const floatx2 ml = join_ml<kLanes>(m, stride, count);
        const float base = finite_or_zero(ml[0]), inv = ml[1] == 0.0f ? 0.0f : 1.0f / ml[1];
        floatx4 o = {0, 0, 0, 0};
#pragma unroll 8
        for (uint32_t s = team; s < count; s += kTeams) {
            const floatx2 y = *reinterpret_cast<const floatx2 *>(m + 2 * s * stride);
            const float f = __builtin_amdgcn_exp2f(y[0] - base) * y[1] * inv;
            const floatx4 x = *reinterpret_cast<const floatx4 *>(from + s * stride * kDim);
#pragma unroll
            for (int e = 0; e < 4; e++) o[e] += f * x[e];
        }
        *reinterpret_cast<floatx4 *>(&sm_o[team][d]) = o;
        __syncthreads();
        if (team == 0 && d < c.dim) {
            for (int k = 1; k < kTeams; k++) {
                const floatx4 x = *reinterpret_cast<const floatx4 *>(&sm_o[k][d]);
#pragma unroll
                for (int e = 0; e < 4; e++) o[e] += x[e];
            }
            const float times = c.type == DS_E4M3 && c.v_scale ? c.v_scale[head] : 1.0f;
            const uint32_t tok = r / a.group, h = r % a.group;
            uint16_t *to = static_cast<uint16_t *>(a.out) +
                           (((uint64_t)row * a.tokens + tok) * c.n_kv * a.group + (uint64_t)head * a.group + h) * c.dim + d;
            *reinterpret_cast<uintx2 *>(to) = uintx2{T::pack(o[0] * times, o[1] * times), T::pack(o[2] * times, o[3] * times)};
        }
        return;
    }
    __shared__ float sm_m[kMaxQueryRows], sm_inv[kMaxQueryRows];
    const uint32_t id = blockIdx.x - join_groups;
    const uint32_t chunk = id % mass_groups, head = id / mass_groups % c.n_kv, row = id / mass_groups / c.n_kv;
    uint32_t req;
    const uint32_t n = length_of(a, row, req);
    const Span span = span_of(n, a.tokens, a.window, a.sinks);
    if (chunk * (kMassTokens / kBlockTokens) >= span.total) return;
    // the scores of the first query rows and what the masses are to be added
    // to are under way while the maxima and sums are joined
    constexpr uint32_t kAhead = 8;
    const uint32_t tok = chunk * kMassTokens + threadIdx.x * 4, v = tok / kBlockTokens;
    const bool on = v < span.total;
    const uint32_t b = v < span.sink_blocks ? v : span.first_block + (v - span.sink_blocks);
    const uint32_t j = b * kBlockTokens + tok % kBlockTokens;
    const float *from = a.scores + ((uint64_t)row * c.n_kv + head) * query_rows * a.score_len + tok;
    float *to = a.mass + ((uint64_t)req * c.n_kv + head) * a.mass_len + j;
    floatx4 ahead[kAhead], w = {0, 0, 0, 0};
#pragma unroll
    for (uint32_t r = 0; r < kAhead; r++)
        if (on && r < query_rows) ahead[r] = *reinterpret_cast<const floatx4 *>(from + (uint64_t)r * a.score_len);
    float old[4];
#pragma unroll
    for (int e = 0; e < 4; e++) old[e] = on && j + e + a.tokens < n ? to[e] : 0.0f;   // the newest tokens start from 0
    const uint32_t first = a.row_slots[2 * row], count = a.row_slots[2 * row + 1];
    for (uint32_t r = threadIdx.x / 16; r < query_rows; r += 16) {
        const floatx2 ml = join_ml<16>(a.part_ml + 2 * part_at(a, first, head, r, unit_rows), stride, count);
        if (threadIdx.x % 16 == 0) {
            sm_m[r] = finite_or_zero(ml[0]);
            sm_inv[r] = ml[1] == 0.0f ? 0.0f : 1.0f / ml[1];
        }
    }
    __syncthreads();
    if (!on) return;
    auto add = [&](uint32_t r, floatx4 s) {
#pragma unroll
        for (int e = 0; e < 4; e++) w[e] += __builtin_amdgcn_exp2f(s[e] - sm_m[r]) * sm_inv[r];
    };
#pragma unroll
    for (uint32_t r = 0; r < kAhead; r++)
        if (r < query_rows) add(r, ahead[r]);
#pragma unroll 4
    for (uint32_t r = kAhead; r < query_rows; r++) add(r, *reinterpret_cast<const floatx4 *>(from + (uint64_t)r * a.score_len));
#pragma unroll
    for (int e = 0; e < 4; e++)
        if (j + e < n) to[e] = old[e] + w[e];
}

template <typename T>
static hipError_t join(const DecodeArgs &a, hipStream_t s)
{
    const uint32_t query_rows = a.group * a.tokens, unit_rows = 16 * unit_tiles(a.c.dim, query_rows);
    const uint32_t groups = a.slot_goal ? a.n_rows * a.c.n_kv * query_rows : 0;
    const uint32_t mass_groups = a.mass ? (uint32_t)cdiv(a.score_len, kMassTokens) : 0;
    const uint32_t grid = groups + a.n_rows * a.c.n_kv * mass_groups;
    const uint32_t dim = padded_dim(a.c.dim);
    if (dim == 64)
        join_kernel<T, 64><<<grid, 256, 0, s>>>(a, groups, mass_groups, unit_rows);
    else if (dim == 128)
        join_kernel<T, 128><<<grid, 256, 0, s>>>(a, groups, mass_groups, unit_rows);
    else
        join_kernel<T, 256><<<grid, 256, 0, s>>>(a, groups, mass_groups, unit_rows);
    return hipGetLastError();
}

hipError_t decode_launch(DecodeArgs a, void *ws, hipStream_t s)
{
    a.part_o = a.part_ml = a.scores = nullptr;
    a.row_slots = nullptr;
    uint8_t *p = static_cast<uint8_t *>(ws);
    if (a.slot_goal) {
        a.part_o = reinterpret_cast<float *>(p);
        p += align_up(part_rows_of(a) * padded_dim(a.c.dim) * 4, 256);
    }
    if (a.slot_goal || a.mass) {
        a.part_ml = reinterpret_cast<float *>(p);
        p += align_up(part_rows_of(a) * 8, 256);
        a.row_slots = reinterpret_cast<uint32_t *>(p);
        p += align_up((uint64_t)a.n_rows * 8, 256);
    }
    if (a.mass) a.scores = reinterpret_cast<float *>(p);
    const bool bf16 = a.q_type == DS_BF16, e4m3 = a.c.type == DS_E4M3;
    hipError_t e = e4m3 ? (bf16 ? decode_attend_bf16_e4m3(a, s) : decode_attend_f16_e4m3(a, s))
                        : (bf16 ? decode_attend_bf16(a, s) : decode_attend_f16(a, s));
    if (e != hipSuccess || !a.part_ml) return e;
    return bf16 ? join<Bf16>(a, s) : join<F16>(a, s);
}

// Contract of the batch: requests in range (once each, where the call writes
// per request), lengths and pages in range.
__global__ void cache_check_kernel(const KvView c, const uint32_t *rows, uint32_t n_rows, bool once, uint32_t *flag)
{
    for (uint32_t i = blockIdx.x; i < n_rows; i += gridDim.x) {
        const uint32_t req = rows ? rows[i] : i;
        if (req >= c.n_requests) {
            if (threadIdx.x == 0) atomicOr(flag, 1u);
            continue;
        }
        const uint32_t n = c.len[req];
        bool bad = n > c.cap;
        const uint32_t pages = (uint32_t)cdiv(n < c.cap ? n : c.cap, c.page_size);
        for (uint32_t p = threadIdx.x; p < pages; p += blockDim.x)
            bad = bad || c.table[(uint64_t)req * c.max_pages + p] >= c.n_pages;
        if (once && rows)
            for (uint32_t k = threadIdx.x; k < i; k += blockDim.x) bad = bad || rows[k] == req;
        if (bad) atomicOr(flag, 1u);
    }
}

hipError_t cache_check(const KvView &c, const uint32_t *rows, uint32_t n_rows, bool once, uint32_t *flag, hipStream_t s)
{
    cache_check_kernel<<<n_rows < 4096 ? n_rows : 4096, 256, 0, s>>>(c, rows, n_rows, once, flag);
    return hipGetLastError();
}

hipError_t decode_check(const DecodeArgs &a, uint32_t *flag, hipStream_t s)
{
    return cache_check(a.c, a.rows, a.n_rows, a.mass != nullptr, flag, s);
}

}  // namespace ds
