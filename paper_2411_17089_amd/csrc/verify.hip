// Verification of drafted tokens against the target's probabilities, from given random numbers (formulas at kvpr_verify_drafts).
//
// Three launches over chunks of the vocabulary, since the order of a request's steps leaves one workgroup per request otherwise
// (five rows of 50272: 226 us in one workgroup):
//   verify_stats   every row of both models at once: of a chunk the largest logit, its index and the sum of exponentials;
//   verify_masses  a request's rows joined from their chunks, the run of drafts that stand, and of each chunk of the row behind
//                  them the sum of max(p - q, 0);
//   verify_pick    the chunk in which the random number falls, then the token in it.
// The first reads everything once and is bound by that; the others read one row of each model again, from the caches.
// Shares and their sums are held in 64 bits: a uniform number falls between two of some 10^5 borders, and sums in 32 bits would
// move those by more than a few per mille of the distance of the closer ones.  Partial sums are added in an order that depends on the sizes
// alone.
#include "paged.h"
#include <math.h>
#include <algorithm>

namespace kvpr {
namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;

// a logit that takes part; NaN counts as -inf
__device__ __forceinline__ float logit(float v) { return v == v ? v : -INFINITY; }

// exp(x) for x <= 0, to 2^-46: x = k ln 2 + r, the Taylor polynomial of degree 11 in |r| <= 0.347 (the rest of the series is below
// 0.347^12 / 12! = 7e-15), ldexp.  A third of the instructions of the library function.
__device__ __forceinline__ double exp_of(double x) {
    x = fmax(x, -800.0);                                   // 0 from -745 on
    const double k = rint(x * 1.4426950408889634);
    const double r = fma(k, -1.9082149292705877e-10, fma(k, -0.6931471803691238, x));
    double p = 1.0 / 39916800.0;
    p = fma(p, r, 1.0 / 3628800.0);
    p = fma(p, r, 1.0 / 362880.0);
    p = fma(p, r, 1.0 / 40320.0);
    p = fma(p, r, 1.0 / 5040.0);
    p = fma(p, r, 1.0 / 720.0);
    p = fma(p, r, 1.0 / 120.0);
    p = fma(p, r, 1.0 / 24.0);
    p = fma(p, r, 1.0 / 6.0);
    p = fma(p, r, 0.5);
    p = fma(p, r, 1.0);
    p = fma(p, r, 1.0);
    return __builtin_ldexp(p, (int)k);
}

// exp((v - top) / T), 1 at the top itself (also an infinite one)
__device__ __forceinline__ double weight(float v, float top, double inv_t) {
    return exp_of(v == top ? 0.0 : ((double)v - (double)top) * inv_t);
}

struct Top { float v; int i; };
__device__ __forceinline__ void take(Top& a, float v, int i) {
    if (v > a.v || (v == a.v && i < a.i)) a = Top{v, i};
}
__device__ __forceinline__ Top wave_top(Top t) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) take(t, __shfl_xor(t.v, o), __shfl_xor(t.i, o));
    return t;
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
__device__ __forceinline__ double block_sum(double v, double* part) {
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s += part[w];
    return s;
}

// of a chunk of a row; top = -inf: nothing takes part
struct Stat {
    float top;
    int at;
    double sum;             // of exp((logit - top) / T); not set for greedy requests
};
// what verify_masses found out about a request
struct Decision {
    int row, token;         // the row that the next token comes from; greedy: the token
    int minus;              // draft row to be taken off (row + 1), or -1
    int pad;
    Stat target, draft;
};

struct VerifyArgs {
    Verify v;
    int chunk, chunks;
    Stat* stats;            // [2][rows][chunks]
    Decision* decisions;    // [n]
    double2* masses;        // [n][chunks] of (max(p - q, 0), p)
};

__device__ __forceinline__ double inverse(float t) { return t > 0.f ? 1.0 / (double)fminf(t, 0x1.fffffep127f) : 0.0; }       // 0: greedy

template <class T> struct Eight;
// 8 logits; rows start anywhere, the hardware takes such loads
template <> struct Eight<float> {
    typedef float half_of __attribute__((ext_vector_type(4), aligned(4)));
    half_of a, b;
    __device__ void load(const float* p) {
        a = __builtin_nontemporal_load(reinterpret_cast<const half_of*>(p));
        b = __builtin_nontemporal_load(reinterpret_cast<const half_of*>(p) + 1);
    }
    __device__ float at(int i) const { return i < 4 ? a[i & 3] : b[i & 3]; }
};
template <> struct Eight<_Float16> {
    typedef _Float16 eight __attribute__((ext_vector_type(8), aligned(2)));
    eight a;
    __device__ void load(const _Float16* p) { a = __builtin_nontemporal_load(reinterpret_cast<const eight*>(p)); }
    __device__ float at(int i) const { return (float)a[i]; }
};

// E elements a thread, in pieces of 8
template <class T, int E>
__global__ __launch_bounds__(THREADS) void verify_stats(const VerifyArgs a) {
    const Verify& v = a.v;
    __shared__ double sums[WAVES];
    __shared__ Top tops[WAVES];
    __shared__ int counts[WAVES];
    const int tid = threadIdx.x, row = blockIdx.x / a.chunks, chunk = blockIdx.x - row * a.chunks, side = blockIdx.y;
    // the request that the row belongs to: the last that starts at or before it
    int count = 0;
    for (int r = 1 + tid; r < v.n; r += THREADS) count += v.row_start[r] <= row;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) count += __shfl_xor(count, o);
    if ((tid & 63) == 0) counts[tid >> 6] = count;
    // the row is asked for meanwhile
    const T* from = (side ? (const T*)v.draft + row * v.ld_draft : (const T*)v.target + row * v.ld_target) + (int64_t)chunk * a.chunk;
    const int n = min(a.chunk, v.vocab - chunk * a.chunk);
    Eight<T> x[E / 8];
#pragma unroll
    for (int j = 0; j < E / 8; ++j) {
        const int i = (j * THREADS + tid) * 8;
        if (i + 8 <= n) x[j].load(from + i);
    }
    __syncthreads();
    int owner = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) owner += counts[w];
    const int first = v.row_start[owner];
    if (row >= v.row_start[owner + 1] || row < first || (side && row == first)) return;
    const double inv_t = inverse(v.temperature[owner]);
    // the elements that are no whole piece of 8: at most 7, one a thread
    const int tail = n & ~7;
    const float last = tail + tid < n ? logit((float)from[tail + tid]) : -INFINITY;
    Top top{last, tail + tid};
#pragma unroll
    for (int j = 0; j < E / 8; ++j) {
        const int i = (j * THREADS + tid) * 8;
        if (i + 8 > n) break;
#pragma unroll
        for (int e = 0; e < 8; ++e) take(top, logit(x[j].at(e)), i + e);
    }
    top = wave_top(top);
    if ((tid & 63) == 0) tops[tid >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) take(top, tops[w].v, tops[w].i);
    double sum = 0.0;
    if (inv_t > 0.0 && top.v > -INFINITY) {
        if (tail + tid < n) sum = weight(last, top.v, inv_t);
#pragma unroll
        for (int j = 0; j < E / 8; ++j) {
            if ((j * THREADS + tid) * 8 + 8 > n) break;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += weight(logit(x[j].at(e)), top.v, inv_t);
        }
        sum = block_sum(sum, sums);
    }
    if (tid == 0) a.stats[((int64_t)side * v.rows + row) * a.chunks + chunk] = Stat{top.v, chunk * a.chunk + top.i, sum};
}

// a row's chunks joined by one wave
__device__ __forceinline__ Stat row_stat(const VerifyArgs& a, int side, int row, double inv_t) {
    const int lane = threadIdx.x & 63;
    const Stat* from = a.stats + ((int64_t)side * a.v.rows + row) * a.chunks;
    Top top{-INFINITY, 0x7fffffff};
    Stat mine{-INFINITY, 0, 0.0};
    for (int c = lane; c < a.chunks; c += 64) {
        mine = from[c];
        if (mine.top > -INFINITY) take(top, mine.top, mine.at);
    }
    top = wave_top(top);
    double sum = 0.0;
    if (inv_t > 0.0 && top.v > -INFINITY) {
        for (int c = lane; c < a.chunks; c += 64) {
            if (a.chunks > 64) mine = from[c];
            if (mine.top > -INFINITY) sum += mine.sum * weight(mine.top, top.v, inv_t);
        }
        sum = wave_sum(sum);
    }
    return Stat{top.v, top.i, sum};
}

// the shares of one token in either model
template <class T>
struct Shares {
    const T *target, *draft;
    Stat t, d;
    double inv_t;
    int drafted;            // the draft itself, where it comes without probabilities
    bool minus;
    __device__ double p(int i) const { return weight(logit((float)target[i]), t.top, inv_t) / t.sum; }
    __device__ double q(int i) const {
        return !draft ? (double)(i == drafted) : d.top == -INFINITY ? 0.0 : weight(logit((float)draft[i]), d.top, inv_t) / d.sum;
    }
    __device__ double rest(int i, double p_) const { return minus ? fmax(p_ - q(i), 0.0) : p_; }
};
template <class T>
__device__ __forceinline__ Shares<T> shares_of(const VerifyArgs& a, const Decision& d, double inv_t) {
    Shares<T> s;
    s.target = (const T*)a.v.target + d.row * a.v.ld_target;
    s.minus = d.minus >= 0;
    s.draft = s.minus && a.v.draft ? (const T*)a.v.draft + d.minus * a.v.ld_draft : nullptr;
    s.t = d.target;
    s.d = d.draft;
    s.inv_t = inv_t;
    s.drafted = s.minus ? a.v.tokens[d.minus] : -1;
    return s;
}

template <class T>
__global__ __launch_bounds__(THREADS) void verify_masses(const VerifyArgs a) {
    const Verify& v = a.v;
    __shared__ int stop;
    __shared__ double sums[WAVES];
    __shared__ Decision decided;
    const int tid = threadIdx.x, wave = tid >> 6, chunk = blockIdx.x, r = blockIdx.y;
    const int first = max(v.row_start[r], 0), end = min(v.row_start[r + 1], v.rows);
    if (first >= end) return;
    const double inv_t = inverse(v.temperature[r]);
    const bool greedy = inv_t == 0.0;
    // a wave per row, four rows at a time, up to the first draft that does not stand
    int at = first;
    for (;; at += WAVES) {
        if (tid == 0) stop = end;
        __syncthreads();
        const int row = at + wave;
        Decision d;
        bool stands = true;
        if (row < end) {
            const bool drafted = row + 1 < end;
            const int token = drafted ? v.tokens[row + 1] : -1;
            const bool valid = token >= 0 && token < v.vocab;
            d.row = row;
            d.minus = valid && !greedy ? row + 1 : -1;
            d.target = row_stat(a, 0, row, inv_t);
            d.draft = valid && v.draft && !greedy ? row_stat(a, 1, row + 1, inv_t) : Stat{-INFINITY, 0, 0.0};
            const bool empty = d.target.top == -INFINITY;
            d.token = empty ? -1 : d.target.at;
            if (greedy) {
                stands = drafted && !empty && token == d.target.at;
            } else if (valid && !empty) {
                const Shares<T> s = shares_of<T>(a, d, inv_t);
                stands = (double)v.u_accept[row + 1] * s.q(token) < s.p(token);
            } else {
                stands = false;                           // also the last row of a request, which has no draft behind it
            }
            if (!stands && (tid & 63) == 0) atomicMin(&stop, row);
        }
        __syncthreads();
        if (row < end && row == stop && (tid & 63) == 0) decided = d;
        __syncthreads();
        if (stop < end) break;
        __syncthreads();
    }
    const Decision d = decided;
    if (chunk == 0 && tid == 0) a.decisions[r] = d;
    if (greedy || d.target.top == -INFINITY) return;
    const Shares<T> s = shares_of<T>(a, d, inv_t);
    const int i0 = chunk * a.chunk, i1 = min(i0 + a.chunk, v.vocab);
    double rest = 0.0, all = 0.0;
    for (int i = i0 + tid; i < i1; i += THREADS) {
        const double p = s.p(i);
        all += p;
        rest += s.rest(i, p);
    }
    rest = block_sum(rest, sums);
    all = block_sum(all, sums);
    if (tid == 0) a.masses[(int64_t)r * a.chunks + chunk] = make_double2(rest, all);
}

// sum over the threads before this one; total: over all
__device__ __forceinline__ double sum_before(double v, double* part, double& total) {
    double s = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const double u = __shfl_up(s, o);
        if ((threadIdx.x & 63) >= o) s += u;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 63) part[threadIdx.x >> 6] = s;
    __syncthreads();
    double before = 0.0;
    total = 0.0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w < (int)(threadIdx.x >> 6)) before += part[w];
        total += part[w];
    }
    return before + s - v;
}

template <class T>
__global__ __launch_bounds__(THREADS) void verify_pick(const VerifyArgs a) {
    const Verify& v = a.v;
    __shared__ double sums[WAVES], base;
    __shared__ int found, last;
    const int tid = threadIdx.x, r = blockIdx.x;
    const int first = max(v.row_start[r], 0), end = min(v.row_start[r + 1], v.rows);
    if (first >= end) {
        if (tid == 0) {
            v.kept[r] = 0;
            if (v.len_out) v.len_out[r] = v.len_in[r];
        }
        return;
    }
    const double inv_t = inverse(v.temperature[r]);
    const Decision d = a.decisions[r];
    int next = d.token;
    if (inv_t > 0.0 && d.target.top > -INFINITY) {
        Shares<T> s = shares_of<T>(a, d, inv_t);
        const double2* masses = a.masses + (int64_t)r * a.chunks;
        // p where p - q leaves nothing
        double sum = 0.0;
        for (int c = tid; c < a.chunks; c += THREADS) sum += masses[c].x;
        if (!(block_sum(sum, sums) > 0.0)) s.minus = false;
        // chunks, a run of them per thread
        const int each = (a.chunks + THREADS - 1) / THREADS, c0 = min(tid * each, a.chunks), c1 = min(c0 + each, a.chunks);
        auto mass = [&](int c) { return s.minus ? masses[c].x : masses[c].y; };
        double mine = 0.0, total;
        for (int c = c0; c < c1; ++c) mine += mass(c);
        double before = sum_before(mine, sums, total);
        const double goal = (double)v.u_sample[r] * total;
        if (tid == 0) { found = a.chunks; last = -1; }
        __syncthreads();
        {
            double upto = before;
            for (int c = c0; c < c1; ++c) {
                upto += mass(c);
                if (mass(c) > 0.0) {
                    atomicMax(&last, c);
                    if (upto > goal) {
                        atomicMin(&found, c);
                        break;
                    }
                }
            }
        }
        __syncthreads();
        const int chunk = found < a.chunks ? found : last;
        // the sum in front of the chunk, as its thread has it
        if (chunk >= c0 && chunk < c1) {
            double upto = before;
            for (int c = c0; c < chunk; ++c) upto += mass(c);
            base = upto;
        }
        __syncthreads();
        if (tid == 0) { found = v.vocab; last = -1; }
        __syncthreads();
        // the chunk's tokens, a run of them per thread
        const int width = (a.chunk + THREADS - 1) / THREADS;
        const int i0 = min(chunk * a.chunk + tid * width, v.vocab), i1 = min(min(i0 + width, (chunk + 1) * a.chunk), v.vocab);
        double here = 0.0, unused;
        for (int i = i0; i < i1; ++i) here += s.rest(i, s.p(i));
        double upto = base + sum_before(here, sums, unused);
        // only threads whose run may pass the goal look again, a little more of them than by the sums, which are not exact
        if (here > 0.0 && upto + here + 1e-9 * total > goal) {
            for (int i = i0; i < i1; ++i) {
                const double w = s.rest(i, s.p(i));
                upto += w;
                if (w > 0.0 && upto > goal) {
                    atomicMin(&found, i);
                    break;
                }
            }
        }
        __syncthreads();
        if (found == v.vocab && here > 0.0) {              // the goal is the whole sum but for its rounding: the last token with a share
            for (int i = i1 - 1; i >= i0; --i)
                if (s.rest(i, s.p(i)) > 0.0) {
                    atomicMax(&last, i);
                    break;
                }
        }
        __syncthreads();
        next = found < v.vocab ? found : last;
    }
    for (int i = first + tid; i < end; i += THREADS) v.out[i] = i < d.row ? v.tokens[i + 1] : i == d.row ? next : -1;
    if (tid == 0) {
        const int gained = d.row - first + 1;
        v.kept[r] = gained;
        if (v.len_out) v.len_out[r] = v.len_in[r] + gained;
    }
}

struct Layout {
    int chunk, chunks;
    size_t stats, decisions, masses;
};
// Chunks of 8192 logits, of 4096 or 2048 where that leaves fewer than 1024 workgroups.
Layout layout_of(int n, int rows, int vocab) {
    Layout l;
    l.chunk = 8192;
    while (l.chunk > 2048 && 2 * (int64_t)rows * ((vocab + l.chunk - 1) / l.chunk) < 1024) l.chunk /= 2;
    l.chunks = (vocab + l.chunk - 1) / l.chunk;
    l.stats = 2 * (size_t)rows * l.chunks * sizeof(Stat);
    l.decisions = (size_t)n * sizeof(Decision);
    l.masses = (size_t)n * l.chunks * sizeof(double2);
    return l;
}

template <class T>
int launch(const Verify& v, void* ws, hipStream_t st) {
    const Layout l = layout_of(v.n, v.rows, v.vocab);
    VerifyArgs a;
    a.v = v;
    a.chunk = l.chunk;
    a.chunks = l.chunks;
    a.stats = (Stat*)ws;
    a.decisions = (Decision*)((char*)ws + l.stats);
    a.masses = (double2*)((char*)ws + l.stats + l.decisions);
    if (v.rows > 0) {
        auto stats = l.chunk == 8192 ? verify_stats<T, 32> : l.chunk == 4096 ? verify_stats<T, 16> : verify_stats<T, 8>;
        hipLaunchKernelGGL(stats, dim3((unsigned)(v.rows * l.chunks), v.draft ? 2 : 1), dim3(THREADS), 0, st, a);
        KVPR_HIP(hipGetLastError());
        hipLaunchKernelGGL(verify_masses<T>, dim3((unsigned)l.chunks, (unsigned)v.n), dim3(THREADS), 0, st, a);
        KVPR_HIP(hipGetLastError());
    }
    hipLaunchKernelGGL(verify_pick<T>, dim3((unsigned)v.n), dim3(THREADS), 0, st, a);
    KVPR_HIP(hipGetLastError());
    return KVPR_OK;
}

}  // namespace

size_t verify_workspace_bytes(int n, int rows, int vocab) {
    const Layout l = layout_of(n, rows, vocab);
    return l.stats + l.decisions + l.masses;
}

int launch_verify(const Verify& v, void* ws, hipStream_t st) { return v.f16 ? launch<_Float16>(v, ws, st) : launch<float>(v, ws, st); }

}  // namespace kvpr
