// Verification of drafted tokens and the draw that follows it.
//
// Which draft is the first rejected one needs two numbers per draft; every
// workgroup finds that by itself. The draw is the inverse of a distribution
// function over one row of the vocabulary: sums per chunk first, then the
// chunk that holds the drawn point is walked. All sums are in 64 bits: a step
// of the distribution function can be as small as the rounding of a 32-bit sum.
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include "common.h"
#include "serve.h"

namespace ds {

constexpr uint32_t kChunk = 4096;          // entries of one sum
constexpr int kThreads = 256;
constexpr int kEach = kChunk / kThreads;

// Sums of every (row, chunk), then the accepted drafts of every row.
static uint64_t sums_bytes(uint32_t n_rows, uint32_t vocab) { return align_up(n_rows * cdiv(vocab, kChunk) * 16, 256); }

size_t verify_ws_bytes(uint32_t n_rows, uint32_t vocab) { return sums_bytes(n_rows, vocab) + align_up((uint64_t)n_rows * 4, 256); }

__device__ __forceinline__ double value(float x) { return (double)x; }
__device__ __forceinline__ double value(__half x) { return (double)__half2float(x); }
__device__ __forceinline__ double value(__hip_bfloat16 x) { return (double)__bfloat162float(x); }

// 16 bytes of a row, which may begin at any entry.
template <typename E>
struct Pack {
    static constexpr uint32_t kN = 16 / sizeof(E);
    E x[kN];
    __device__ __forceinline__ void load(const E *p) { __builtin_memcpy(x, p, 16); }
};

// The drawn position of a row: a accepted drafts of m.
struct Verdict {
    uint32_t a, m;
};

template <typename E>
__device__ inline Verdict verdict(const VerifyArgs &v, uint32_t row)
{
    Verdict r;
    r.m = v.n_draft ? v.n_draft[row] : v.n_drafts;
    if (r.m > v.n_drafts) r.m = v.n_drafts;
    const uint32_t t = lane_id();
    bool ok = false;
    if (t < r.m) {
        const int32_t x = v.tokens[(uint64_t)row * v.n_drafts + t];
        if (x >= 0 && (uint32_t)x < v.vocab) {
            const double p = value(static_cast<const E *>(v.target)[row * v.t_row + t * v.t_pos + x]);
            const double q = v.draft ? value(static_cast<const E *>(v.draft)[row * v.d_row + t * v.d_pos + x]) : 1.0;
            ok = (double)v.u[(uint64_t)row * v.n_drafts + t] * q < p;
        }
    }
    r.a = (uint32_t)__builtin_ctzll(~__ballot(ok));      // at most 63 drafts: bit 63 is clear
    return r;
}

// The weights of the drawn position: w (the residual where a draft was
// rejected) and p.
template <typename E>
struct Weights {
    const E *p, *q;
    int32_t without;                       // the rejected token, if the drafts were not drawn
    bool residual;
    __device__ Weights(const VerifyArgs &v, uint32_t row, Verdict r)
    {
        residual = r.a < r.m;
        p = static_cast<const E *>(v.target) + row * v.t_row + r.a * v.t_pos;
        q = v.draft && residual ? static_cast<const E *>(v.draft) + row * v.d_row + r.a * v.d_pos : nullptr;
        without = !v.draft && residual ? v.tokens[(uint64_t)row * v.n_drafts + r.a] : -1;
    }
    __device__ __forceinline__ void of(uint32_t j, E pe, E qe, double &w, double &pp) const
    {
        const double x = value(pe);
        pp = x > 0.0 ? x : 0.0;
        w = pp;
        if (q) {
            const double y = x - value(qe);
            w = y > 0.0 ? y : 0.0;
        } else if ((int32_t)j == without) {
            w = 0.0;
        }
    }
    // f(k, w, p) for the entries first + 16 bytes' worth * step * i + k, in
    // order; 0 past the vocabulary.
    template <typename F>
    __device__ __forceinline__ void each(uint32_t first, uint32_t step, uint32_t vocab, F &&f) const
    {
        constexpr uint32_t kN = Pack<E>::kN, kPacks = kEach / kN;
        Pack<E> a[kPacks], b[kPacks];
#pragma unroll
        for (uint32_t i = 0; i < kPacks; i++) {
            const uint32_t j = first + i * step * kN;
            if (j + kN <= vocab) {
                a[i].load(p + j);
                if (q) b[i].load(q + j);
            } else {
#pragma unroll
                for (uint32_t k = 0; k < kN; k++) {
                    a[i].x[k] = j + k < vocab ? p[j + k] : E(0.0f);
                    b[i].x[k] = q && j + k < vocab ? q[j + k] : E(0.0f);
                }
            }
        }
#pragma unroll
        for (uint32_t i = 0; i < kPacks; i++)
#pragma unroll
            for (uint32_t k = 0; k < kN; k++) {
                double w, pp;
                of(first + i * step * kN + k, a[i].x[k], b[i].x[k], w, pp);
                f(i * kN + k, w, pp);
            }
    }
};

__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) x += __shfl_xor(x, d, 64);
    return x;
}

template <typename F>
__device__ __forceinline__ uint32_t wave_reduce(uint32_t x, F &&f)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) x = f(x, (uint32_t)__shfl_xor((int)x, d, 64));
    return x;
}

// Sum over the threads before this one; the sum of all in `all`.
__device__ inline double block_before(double x, double *lds, double &all)
{
    double incl = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const double y = __shfl_up(incl, d, 64);
        if (lane_id() >= d) incl += y;
    }
    const int wave = threadIdx.x >> 6;
    __syncthreads();                       // lds may be in use from a call before
    if (lane_id() == 63) lds[wave] = incl;
    __syncthreads();
    double off = 0.0;
    all = 0.0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; w++) {
        if (w < wave) off += lds[w];
        all += lds[w];
    }
    return off + (incl - x);
}

template <typename E>
__global__ __launch_bounds__(kThreads) void sums_kernel(const VerifyArgs v, uint32_t chunks)
{
    __shared__ double part[2][kThreads / 64];
    const uint32_t row = blockIdx.x / chunks, chunk = blockIdx.x % chunks;
    const Verdict r = verdict<E>(v, row);
    if (chunk == 0 && threadIdx.x == 0) v.accepted[row] = r.a;
    const Weights<E> weights(v, row, r);
    double sw = 0.0, sp = 0.0;
    weights.each(chunk * kChunk + threadIdx.x * Pack<E>::kN, kThreads, v.vocab, [&](uint32_t, double w, double p) {
        sw += w;
        sp += p;
    });
    sw = wave_sum(sw);
    sp = wave_sum(sp);
    if (lane_id() == 0) {
        part[0][threadIdx.x >> 6] = sw;
        part[1][threadIdx.x >> 6] = sp;
    }
    __syncthreads();
    if (threadIdx.x < 2) {
        double s = 0.0;
        for (int w = 0; w < kThreads / 64; w++) s += part[threadIdx.x][w];
        v.sums[((uint64_t)row * chunks + chunk) * 2 + threadIdx.x] = s;
    }
}

template <typename E>
__global__ __launch_bounds__(kThreads) void draw_kernel(const VerifyArgs v, uint32_t chunks)
{
    constexpr uint32_t kNone = 0xFFFFFFFFu;
    __shared__ double lds[kThreads / 64], sm_before;
    __shared__ uint32_t sm_chunk, sm_some, sm_found, sm_last;
    const uint32_t row = blockIdx.x, t = threadIdx.x;
    Verdict r;
    r.m = v.n_draft ? v.n_draft[row] : v.n_drafts;
    if (r.m > v.n_drafts) r.m = v.n_drafts;
    r.a = v.accepted[row];
    const Weights<E> weights(v, row, r);
    const double *sums = v.sums + (uint64_t)row * chunks * 2;
    if (t == 0) {
        sm_chunk = kNone;
        sm_found = kNone;
        sm_some = 0;
        sm_last = 0;
    }

    // the chunk in which the sum passes the target; if rounding leaves none,
    // the last with anything in it
    const uint32_t each = (chunks + kThreads - 1) / kThreads;
    const uint32_t k0 = t * each < chunks ? t * each : chunks, k1 = k0 + each < chunks ? k0 + each : chunks;
    double sw = 0.0, sp = 0.0, all_w, all_p;
    for (uint32_t k = k0; k < k1; k++) {
        sw += sums[2 * k];
        sp += sums[2 * k + 1];
    }
    const double before_w = block_before(sw, lds, all_w), before_p = block_before(sp, lds, all_p);
    const int use = all_w > 0.0 ? 0 : 1;   // no residual: the target itself
    const double target = (double)v.u_sample[row] * (use ? all_p : all_w);
    const double start = use ? before_p : before_w;
    double c0 = start;
    uint32_t some = 0, hit = kNone;
    for (uint32_t k = k0; k < k1; k++) {
        const double x = sums[2 * k + use];
        c0 += x;
        if (x > 0.0) {
            some = k + 1;
            if (c0 > target && hit == kNone) hit = k;
        }
    }
    some = wave_reduce(some, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
    hit = wave_reduce(hit, [](uint32_t x, uint32_t y) { return x < y ? x : y; });
    if (lane_id() == 0) {
        atomicMax(&sm_some, some);
        atomicMin(&sm_chunk, hit);
    }
    __syncthreads();
    const uint32_t chunk = sm_chunk != kNone ? sm_chunk : sm_some - 1;
    int32_t drawn = -1;
    if (chunk != kNone) {                  // the same for all threads
        if (chunk >= k0 && chunk < k1) {
            double b = start;
            for (uint32_t k = k0; k < chunk; k++) b += sums[2 * k + use];
            sm_before = b;
        }
        double own[kEach], s = 0.0, all;
        const uint32_t j0 = chunk * kChunk + t * kEach;
        weights.each(j0, 1, v.vocab, [&](uint32_t k, double w, double p) {
            own[k] = use ? p : w;
            s += own[k];
        });
        double c1 = block_before(s, lds, all);
        c1 += sm_before;
        hit = kNone;
        some = 0;                          // one atomic per wave: of many to one word each waits for the last
#pragma unroll
        for (int k = 0; k < kEach; k++) {
            c1 += own[k];
            if (own[k] > 0.0) {
                some = j0 + k;
                if (c1 > target && hit == kNone) hit = j0 + k;
            }
        }
        some = wave_reduce(some, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
        hit = wave_reduce(hit, [](uint32_t x, uint32_t y) { return x < y ? x : y; });
        if (lane_id() == 0) {
            atomicMax(&sm_last, some);
            atomicMin(&sm_found, hit);
        }
        __syncthreads();
        drawn = (int32_t)(sm_found != kNone ? sm_found : sm_last);
    }
    if (t <= v.n_drafts)
        v.out[(uint64_t)row * (v.n_drafts + 1) + t] = t < r.a    ? v.tokens[(uint64_t)row * v.n_drafts + t]
                                                      : t == r.a ? drawn
                                                                 : -1;
    if (t == 0) {
        const uint32_t emitted = r.a + (drawn >= 0 ? 1 : 0);
        v.n_emitted[row] = emitted;
        const uint32_t req = v.rows ? v.rows[row] : row;
        if (req < v.n_requests) {
            if (v.observed) atomicAdd(&v.observed[req], emitted);
            if (v.len) {
                const uint32_t n = v.len[req], off = r.m - r.a;
                v.len[req] = n > off ? n - off : 0;
            }
        }
    }
}

template <typename E>
static hipError_t launch(const VerifyArgs &v, hipStream_t s)
{
    const uint32_t chunks = (uint32_t)cdiv(v.vocab, kChunk);
    sums_kernel<E><<<v.n_rows * chunks, kThreads, 0, s>>>(v, chunks);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    draw_kernel<E><<<v.n_rows, kThreads, 0, s>>>(v, chunks);
    return hipGetLastError();
}

hipError_t verify_launch(VerifyArgs v, void *ws, hipStream_t s)
{
    v.sums = static_cast<double *>(ws);
    v.accepted = reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(ws) + sums_bytes(v.n_rows, v.vocab));
    return v.type == DS_F32 ? launch<float>(v, s) : v.type == DS_F16 ? launch<__half>(v, s) : launch<__hip_bfloat16>(v, s);
}

__global__ void verify_check_kernel(const VerifyArgs v, uint32_t *flag)
{
    for (uint32_t i = blockIdx.x; i < v.n_rows; i += gridDim.x) {
        bool bad = false;
        const uint32_t m = v.n_draft ? v.n_draft[i] : v.n_drafts;
        if (m > v.n_drafts) bad = true;
        if (threadIdx.x < m && threadIdx.x < v.n_drafts) {
            const int32_t x = v.tokens[(uint64_t)i * v.n_drafts + threadIdx.x];
            const float u = v.u[(uint64_t)i * v.n_drafts + threadIdx.x];
            bad = bad || x < 0 || (uint32_t)x >= v.vocab || !(u >= 0.0f && u < 1.0f);
        }
        const float u = v.u_sample[i];
        bad = bad || !(u >= 0.0f && u < 1.0f);
        const uint32_t req = v.rows ? v.rows[i] : i;
        if (v.observed || v.len) bad = bad || req >= v.n_requests;
        if (v.len && v.rows)
            for (uint32_t k = threadIdx.x; k < i; k += blockDim.x) bad = bad || v.rows[k] == req;
        if (bad) atomicOr(flag, 1u);
    }
}

hipError_t verify_check(const VerifyArgs &v, uint32_t *flag, hipStream_t s)
{
    verify_check_kernel<<<v.n_rows < 4096 ? v.n_rows : 4096, 256, 0, s>>>(v, flag);
    return hipGetLastError();
}

}  // namespace ds
