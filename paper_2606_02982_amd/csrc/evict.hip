// Eviction from the paged cache by accumulated attention weight.
//
// Per (row, head) the kept set is a selection: the k-th largest of the masses
// that compete is found digit by digit (8 bits from the top, counting the
// values that agree with the digits found so far), then one walk in token
// order keeps what is larger, and of what is equal the earliest. The copy of
// the kept keys and values is a second launch over all tokens of all rows.
#include "common.h"
#include "serve.h"

namespace ds {

constexpr int kSelect = 1024;              // threads of one selection
constexpr int kSelectWaves = kSelect / 64;
constexpr uint32_t kCopyTokens = 64;       // tokens of one workgroup of the copy

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

__global__ __launch_bounds__(kSelect) void select_kernel(const EvictArgs a)
{
    __shared__ uint32_t hist[256], pick[2], gt_of[kSelectWaves], eq_of[kSelectWaves];
    const uint32_t row = blockIdx.x / a.src.n_kv, head = blockIdx.x % a.src.n_kv;
    const Cut x = cut_of(a, row);
    if (threadIdx.x == 0 && head == 0) a.dst.len[row] = x.keep;
    if (x.keep == x.n) return;
    const float *mass = a.mass + ((uint64_t)x.req * a.src.n_kv + head) * a.mass_len;
    uint32_t *kept = a.kept + ((uint64_t)row * a.src.n_kv + head) * a.kept_len;
    const uint32_t lo = a.sinks, hi = x.n - a.recent;          // the tokens that compete
    uint32_t want = x.keep - a.sinks - a.recent;               // how many of them stay
    const int wave = threadIdx.x >> 6;

    uint32_t bar = 0xFFFFFFFFu;            // the smallest kept key; of it the first `want` stay
    if (want) {
        uint32_t found = 0;                // the digits of bar so far
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (threadIdx.x < 256) hist[threadIdx.x] = 0;
            __syncthreads();
            for (uint32_t j = lo + threadIdx.x; j < hi; j += kSelect) {
                const uint32_t key = mass_key(mass[j]);
                if (shift == 24 || (key >> (shift + 8)) == (found >> (shift + 8))) atomicAdd(&hist[(key >> shift) & 255u], 1u);
            }
            __syncthreads();
            if (wave == 0) {
                // lane l holds digits 255 - 4 l .. 252 - 4 l: counts from the largest digit down
                uint32_t h[4], own = 0;
#pragma unroll
                for (int k = 0; k < 4; k++) own += h[k] = hist[255 - 4 * lane_id() - k];
                uint32_t before = wave_incl_scan_dpp(own) - own;
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    if (before < want && want <= before + h[k]) {
                        pick[0] = 255 - 4 * lane_id() - k;
                        pick[1] = want - before;
                    }
                    before += h[k];
                }
            }
            __syncthreads();
            found |= pick[0] << shift;
            want = pick[1];
            __syncthreads();
        }
        bar = found;
    }

    // kept tokens in their order: each wave walks a run of its own
    const uint32_t run = (uint32_t)align_up(cdiv(x.n, kSelectWaves), 64);
    const uint32_t j0 = wave * run < x.n ? wave * run : x.n, j1 = j0 + run < x.n ? j0 + run : x.n;
    uint32_t n_gt = 0, n_eq = 0;
    auto state = [&](uint32_t j, bool &gt, bool &eq) {
        const bool in = j < j1, sure = in && (j < lo || j >= hi);
        const uint32_t key = in && !sure ? mass_key(mass[j]) : 0u;
        gt = sure || (in && key > bar);
        eq = in && !sure && want && key == bar;
    };
    for (uint32_t j = j0; j < j1; j += 64) {
        bool gt, eq;
        state(j + lane_id(), gt, eq);
        n_gt += __popcll(__ballot(gt));
        n_eq += __popcll(__ballot(eq));
    }
    if (lane_id() == 0) {
        gt_of[wave] = n_gt;
        eq_of[wave] = n_eq;
    }
    __syncthreads();
    uint32_t at = 0, eq_at = 0;
    for (int w = 0; w < wave; w++) {
        const uint32_t left = eq_at < want ? want - eq_at : 0;
        at += gt_of[w] + (eq_of[w] < left ? eq_of[w] : left);
        eq_at += eq_of[w];
    }
    for (uint32_t j = j0; j < j1; j += 64) {
        bool gt, eq;
        state(j + lane_id(), gt, eq);
        const uint64_t eqs = __ballot(eq);
        const bool stays = gt || (eq && eq_at + __popcll(eqs & lanemask_lt()) < want);
        const uint64_t all = __ballot(stays);
        if (stays) kept[at + __popcll(all & lanemask_lt())] = j + lane_id();
        at += __popcll(all);
        eq_at += __popcll(eqs);
    }
    __syncthreads();
    // kept[i] >= i: reading a piece before writing it is enough where mass_out is mass
    float *mass_out = a.mass_out + ((uint64_t)x.req * a.src.n_kv + head) * a.mass_len;
    for (uint32_t i = 0; i < x.keep; i += kSelect) {
        const uint32_t k = i + threadIdx.x;
        const float val = k < x.keep ? mass[kept[k]] : 0.0f;
        __syncthreads();
        if (k < x.keep) mass_out[k] = val;
        __syncthreads();
    }
}

// 16 bytes of a key or value per thread and step.
__global__ __launch_bounds__(256) void copy_kernel(const EvictArgs a, uint32_t chunks, uint32_t elem)
{
    const uint32_t chunk = blockIdx.x % chunks, head = blockIdx.x / chunks % a.src.n_kv;
    const uint32_t row = blockIdx.x / chunks / a.src.n_kv;
    const Cut x = cut_of(a, row);
    if (x.keep == x.n || chunk * kCopyTokens >= x.keep) return;
    const KvView &s = a.src, &d = a.dst;
    const uint32_t *kept = a.kept + ((uint64_t)row * s.n_kv + head) * a.kept_len;
    const uint32_t left = x.keep - chunk * kCopyTokens, count = left < kCopyTokens ? left : kCopyTokens;
    const uint32_t units = s.dim * elem / 16;
    for (uint32_t i = threadIdx.x; i < count * units; i += 256) {
        const uint32_t to = chunk * kCopyTokens + i / units, from = kept[to], u = i % units;
        const uint32_t sp = s.table[(uint64_t)x.req * s.max_pages + from / s.page_size];
        const uint32_t dp = d.table[(uint64_t)row * d.max_pages + to / d.page_size];
        if (sp >= s.n_pages || dp >= d.n_pages) continue;
        const uint64_t sa = (sp * s.page_stride + (from % s.page_size) * s.token_stride + head * s.head_stride) * elem + u * 16;
        const uint64_t da = (dp * d.page_stride + (to % d.page_size) * d.token_stride + head * d.head_stride) * elem + u * 16;
        *reinterpret_cast<uint4 *>(d.k + da) = *reinterpret_cast<const uint4 *>(s.k + sa);
        *reinterpret_cast<uint4 *>(d.v + da) = *reinterpret_cast<const uint4 *>(s.v + sa);
    }
}

hipError_t evict_launch(const EvictArgs &a, hipStream_t s)
{
    select_kernel<<<a.n_rows * a.src.n_kv, kSelect, 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    uint64_t most = (uint64_t)a.dst.max_pages * a.dst.page_size;
    if (most > a.kept_len) most = a.kept_len;
    if (most > a.src.cap) most = a.src.cap;
    const uint32_t chunks = (uint32_t)cdiv(most, kCopyTokens);
    if (!chunks) return hipSuccess;
    copy_kernel<<<a.n_rows * a.src.n_kv * chunks, 256, 0, s>>>(a, chunks, a.src.type == DS_E4M3 ? 1 : 2);
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
