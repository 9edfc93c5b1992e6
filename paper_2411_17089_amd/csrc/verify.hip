// Verification of drafted tokens against the target's probabilities, from given random numbers (formulas at kvpr_verify_drafts).
//
// One workgroup per request: the softmax of a row of either model as (largest logit, sum of exponentials), row after row until a
// draft is rejected, then the token from what is left by the inverse of the summed shares.
// Shares and their sums are held in 64 bits: a uniform number falls between two of some 10^5 borders, and sums in 32 bits would
// move those by more than a few per mille of the distance of the closer ones.
#include "paged.h"
#include <math.h>

namespace kvpr {
namespace {

constexpr int THREADS = 1024, WAVES = THREADS / 64;

// a logit that takes part; NaN counts as -inf
__device__ __forceinline__ float logit(float v) { return v == v ? v : -INFINITY; }

// exp((v - top) / T), 1 at the top itself (also an infinite one)
__device__ __forceinline__ double weight(float v, float top, double inv_t) {
    return v == top ? 1.0 : exp(((double)v - (double)top) * inv_t);
}

struct Top { float v; int i; };
__device__ __forceinline__ void take(Top& a, float v, int i) {
    if (v > a.v || (v == a.v && i < a.i)) a = Top{v, i};
}

__device__ __forceinline__ double block_sum(double v, double* part) {
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
    for (int w = 0; w < WAVES; ++w) s += part[w];
    return s;
}

__device__ __forceinline__ Top block_top(Top t, Top* part) {
    for (int o = 32; o > 0; o >>= 1) take(t, __shfl_xor(t.v, o), __shfl_xor(t.i, o));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = t;
    __syncthreads();
    t = part[0];
    for (int w = 1; w < WAVES; ++w) take(t, part[w].v, part[w].i);
    return t;
}

template <class T>
__global__ __launch_bounds__(THREADS) void verify_kernel(const T* __restrict__ target, int64_t ld_target, const T* __restrict__ draft, int64_t ld_draft,
                                                         const int32_t* __restrict__ tokens, const int32_t* __restrict__ row_start, int rows, int vocab,
                                                         const float* __restrict__ temperature, const float* __restrict__ u_accept,
                                                         const float* __restrict__ u_sample, const int32_t* len_in, int32_t* len_out,
                                                         int32_t* __restrict__ kept, int32_t* __restrict__ out) {
    __shared__ double sums[WAVES];
    __shared__ Top tops[WAVES];
    const int tid = threadIdx.x, r = blockIdx.x;
    const int first = max(row_start[r], 0), end = min(row_start[r + 1], rows);
    const float t = temperature[r];
    const bool greedy = !(t > 0.f);
    const double inv_t = greedy ? 1.0 : 1.0 / (double)t;
    auto stats = [&](const T* row, Top& top, double& sum) {
        top = Top{-INFINITY, 0x7fffffff};
        for (int i = tid; i < vocab; i += THREADS) take(top, logit((float)row[i]), i);
        top = block_top(top, tops);
        double s = 0.0;
        if (!greedy)
            for (int i = tid; i < vocab; i += THREADS) s += weight(logit((float)row[i]), top.v, inv_t);
        sum = block_sum(s, sums);
    };
    if (first >= end) {
        if (tid == 0) {
            kept[r] = 0;
            if (len_out) len_out[r] = len_in[r];
        }
        return;
    }
    int row = first, next = -1;
    for (;; ++row) {
        const bool drafted = row + 1 < end;
        const int token = drafted ? tokens[row + 1] : -1;
        const T* pr = target + row * ld_target;
        const T* qr = drafted && draft ? draft + (row + 1) * ld_draft : nullptr;
        Top pt, qt{-INFINITY, 0x7fffffff};
        double ps, qs = 1.0;
        stats(pr, pt, ps);
        if (pt.v == -INFINITY) break;                       // no distribution: nothing accepted, no token
        if (greedy) {
            if (drafted && token == pt.i) continue;
            next = pt.i;
            break;
        }
        if (qr) stats(qr, qt, qs);
        const bool q_empty = qr && qt.v == -INFINITY;
        const bool valid = drafted && token >= 0 && token < vocab;
        if (valid) {
            const double p = weight(logit((float)pr[token]), pt.v, inv_t) / ps;
            const double q = !qr ? 1.0 : q_empty ? 0.0 : weight(logit((float)qr[token]), qt.v, inv_t) / qs;
            if ((double)u_accept[row + 1] * q < p) continue;
        }
        // the token from max(p - q, 0), from p where that leaves nothing
        auto rest = [&](int i, bool minus) {
            const double p = weight(logit((float)pr[i]), pt.v, inv_t) / ps;
            if (!minus) return p;
            const double q = !qr ? (double)(i == token) : q_empty ? 0.0 : weight(logit((float)qr[i]), qt.v, inv_t) / qs;
            return fmax(p - q, 0.0);
        };
        const int each = (vocab + THREADS - 1) / THREADS, i0 = min(tid * each, vocab), i1 = min(i0 + each, vocab);
        bool minus = valid;
        double mine = 0.0, total;
        for (;;) {
            mine = 0.0;
            for (int i = i0; i < i1; ++i) mine += rest(i, minus);
            total = block_sum(mine, sums);
            if (total > 0.0 || !minus) break;
            minus = false;
        }
        double upto = mine;                                   // inclusive prefix over the workgroup
        for (int o = 1; o < 64; o <<= 1) {
            const double u = __shfl_up(upto, o);
            if ((tid & 63) >= o) upto += u;
        }
        __syncthreads();
        if ((tid & 63) == 63) sums[tid >> 6] = upto;
        __syncthreads();
        for (int w = 0; w < (tid >> 6); ++w) upto += sums[w];
        const double goal = (double)u_sample[r] * total;
        __shared__ int pick, last;
        if (tid == 0) { pick = 0x7fffffff; last = -1; }
        __syncthreads();
        double s = upto - mine;
        int li = -1;
        for (int i = i0; i < i1; ++i) {
            const double w = rest(i, minus);
            s += w;
            if (w > 0.0) {
                li = i;
                if (s > goal) { atomicMin(&pick, i); break; }
            }
        }
        if (li >= 0) atomicMax(&last, li);
        __syncthreads();
        next = pick < vocab ? pick : last;
        break;
    }
    for (int i = first + tid; i < end; i += THREADS) out[i] = i < row ? tokens[i + 1] : i == row ? next : -1;
    if (tid == 0) {
        kept[r] = row - first + 1;
        if (len_out) len_out[r] = len_in[r] + row - first + 1;
    }
}

}  // namespace

size_t verify_workspace_bytes(int, int, int) { return 16; }

int launch_verify(const Verify& v, void*, hipStream_t st) {
    if (v.f16)
        hipLaunchKernelGGL(verify_kernel<_Float16>, dim3((unsigned)v.n), dim3(THREADS), 0, st, (const _Float16*)v.target, v.ld_target, (const _Float16*)v.draft,
                           v.ld_draft, v.tokens, v.row_start, v.rows, v.vocab, v.temperature, v.u_accept, v.u_sample, v.len_in, v.len_out, v.kept, v.out);
    else
        hipLaunchKernelGGL(verify_kernel<float>, dim3((unsigned)v.n), dim3(THREADS), 0, st, (const float*)v.target, v.ld_target, (const float*)v.draft,
                           v.ld_draft, v.tokens, v.row_start, v.rows, v.vocab, v.temperature, v.u_accept, v.u_sample, v.len_in, v.len_out, v.kept, v.out);
    KVPR_HIP(hipGetLastError());
    return KVPR_OK;
}

}  // namespace kvpr
