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

size_t verify_ws_bytes(uint32_t n_rows, uint32_t vocab) { return align_up(n_rows * cdiv(vocab, kChunk) * 16, 256); }

__device__ __forceinline__ double value(const float *p, uint64_t i) { return (double)p[i]; }
__device__ __forceinline__ double value(const __half *p, uint64_t i) { return (double)__half2float(p[i]); }
__device__ __forceinline__ double value(const __hip_bfloat16 *p, uint64_t i) { return (double)__bfloat162float(p[i]); }

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
            const double p = value(static_cast<const E *>(v.target), row * v.t_row + t * v.t_pos + x);
            const double q = v.draft ? value(static_cast<const E *>(v.draft), row * v.d_row + t * v.d_pos + x) : 1.0;
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
    __device__ __forceinline__ void at(uint32_t j, double &w, double &pp) const
    {
        const double x = value(p, j);
        pp = x > 0.0 ? x : 0.0;
        w = pp;
        if (q) {
            const double y = x - value(q, j);
            w = y > 0.0 ? y : 0.0;
        } else if ((int32_t)j == without) {
            w = 0.0;
        }
    }
};

__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) x += __shfl_xor(x, d, 64);
    return x;
}

template <typename E>
__global__ __launch_bounds__(kThreads) void sums_kernel(const VerifyArgs v, uint32_t chunks)
{
    __shared__ double part[2][kThreads / 64];
    const uint32_t row = blockIdx.x / chunks, chunk = blockIdx.x % chunks;
    const Verdict r = verdict<E>(v, row);
    const Weights<E> weights(v, row, r);
    double sw = 0.0, sp = 0.0;
    for (uint32_t k = threadIdx.x; k < kChunk; k += kThreads) {
        const uint32_t j = chunk * kChunk + k;
        if (j < v.vocab) {
            double w, p;
            weights.at(j, w, p);
            sw += w;
            sp += p;
        }
    }
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
    __shared__ double tot[kThreads];
    __shared__ uint32_t found, last;
    __shared__ double before;
    const uint32_t row = blockIdx.x, t = threadIdx.x;
    const Verdict r = verdict<E>(v, row);
    const Weights<E> weights(v, row, r);
    const double *sums = v.sums + (uint64_t)row * chunks * 2;
    __shared__ int use;
    __shared__ double target;
    __shared__ uint32_t at_chunk;
    if (t == 0) {
        double sw = 0.0, sp = 0.0;
        for (uint32_t c = 0; c < chunks; c++) {
            sw += sums[2 * c];
            sp += sums[2 * c + 1];
        }
        use = sw > 0.0 ? 0 : 1;            // no residual: the target itself
        const double s = use ? sp : sw;
        target = (double)v.u_sample[row] * s;
        // the chunk in which the sum passes the target; if rounding leaves
        // none, the last with anything in it
        double c0 = 0.0;
        at_chunk = 0xFFFFFFFFu;
        before = 0.0;
        for (uint32_t c = 0; c < chunks; c++) {
            const double x = sums[2 * c + use];
            if (x > 0.0) {
                at_chunk = c;
                before = c0;
            }
            c0 += x;
            if (c0 > target) break;
        }
        found = 0xFFFFFFFFu;
        last = 0;
    }
    __syncthreads();
    int32_t drawn = -1;
    if (at_chunk != 0xFFFFFFFFu) {
        double own[kEach], s = 0.0;
        const uint32_t j0 = at_chunk * kChunk + t * kEach;
#pragma unroll
        for (int k = 0; k < kEach; k++) {
            double w = 0.0, p = 0.0;
            if (j0 + k < v.vocab) weights.at(j0 + k, w, p);
            own[k] = use ? p : w;
            s += own[k];
        }
        tot[t] = s;
        __syncthreads();
        double c0 = before;
        for (uint32_t k = 0; k < t; k++) c0 += tot[k];
#pragma unroll
        for (int k = 0; k < kEach; k++) {
            c0 += own[k];
            if (own[k] > 0.0) {
                atomicMax(&last, j0 + k);
                if (c0 > target) atomicMin(&found, j0 + k);
            }
        }
        __syncthreads();
        drawn = (int32_t)(found != 0xFFFFFFFFu ? found : last);
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
