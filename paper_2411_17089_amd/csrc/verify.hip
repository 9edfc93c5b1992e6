// Verification of drafted tokens against the target's probabilities, from given random numbers (formulas at kvpr_verify_drafts; kvpr_verify_step is the
// same behind a plan that may have refused requests, and with prompt chunks).
//
// Three launches over chunks of the vocabulary, since the order of a request's steps leaves one workgroup per request otherwise
// (five rows of 50272: 226 us in one workgroup):
//   verify_stats   every row of both models at once: of a chunk the largest logit, its index and the sum of exponentials;
//   verify_decide  a request's rows joined from their chunks, and the run of drafts that stand;
//   verify_draw    of each chunk of the row behind them the sum of max(p - q, 0); the last workgroup of a request then finds the chunk in
//                  which the random number falls, and the token in it.
// The first reads everything once and is bound by its vector instructions, 38 a logit: at 4 cycles each and 2.4 GHz 31 of 34 us for 240 rows of 131071 in
// float32 (whose bytes are 26), 13 of 19 for 400 rows of 32000 in float16.  The last reads one row of each model again, from the caches, and
// is a chain of waits - loads, acknowledged stores, barriers - in which its waves spend 60 to 70 % of their time.
// Shares, good to some 10^-12, and their sums are held in 64 bits: a uniform number falls between two of some 10^5 borders, and sums in 32 bits would
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

// 2^t for -1100 <= t <= 0, subnormal numbers among them: t = k + f with |f| <= 1/2 (adding 1.5 2^52 leaves k in the low word), the polynomial of degree 8 that meets 2^f
// in the 9 Chebyshev points of that interval (off by 1.1 10^-12 at most, in turns above and below), ldexp: 14 of the 38 vector instructions a
// logit, which bound the reading of many logits.  The library's exp and the steps around it are 40 by themselves.
__device__ __forceinline__ double exp2_of(double t) {
    const double big = 6755399441055744.0, kd = t + big, f = t - (kd - big);
    double p = 1.325497460306718e-06;
    p = fma(p, f, 1.531007807039615e-05);
    p = fma(p, f, 0.00015403457039410448);
    p = fma(p, f, 0.0013333450573018062);
    p = fma(p, f, 0.009618129157656703);
    p = fma(p, f, 0.055504109412010456);
    p = fma(p, f, 0.24022650695821055);
    p = fma(p, f, 0.6931471805459343);
    p = fma(p, f, 0.9999999999999997);
    return __builtin_ldexp(p, __double2loint(kd));
}

// exp((v - top) / T) of one row; with an infinite top 1 where the logit is infinite too and 0 elsewhere
struct Weight {
    float top, low;                 // low: logits so far down, and NaN, have weight 0 (below 2^-1075)
    double c;
    __device__ Weight(float top_, double inv_t) : top(top_) {
        c = inv_t * 1.4426950408889634;
        low = top == INFINITY ? 0x1.fffffep127f : (float)((double)top - 1076.0 / c);
        if (low == top) low = nextafterf(top, -INFINITY);       // 1076 / c less than half a step of the type
    }
    __device__ double operator()(float v) const {
        const double w = top == INFINITY ? 1.0 : exp2_of(((double)v - (double)top) * c);
        return v > low ? w : 0.0;
    }
};

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
    int at;                 // index of it, for greedy requests
    double sum;             // of exp((logit - top) / T), for the others
};
// what verify_decide found out about a request whose next token is drawn
struct Decision {
    int first, end, row;    // its rows, and the one that the next token comes from; row = -1: nothing is left to do
    int drafted;            // the draft that did not stand, to be taken off, or -1
    float target_top, draft_top;
    float goal;             // u_sample
    unsigned arrived;       // workgroups of verify_draw that are done
    double inv_t, p_norm, q_norm;       // 1 / sums; q_norm = 0: the draft row has no distribution
};

struct VerifyArgs {
    Verify v;
    int chunk, chunks;
    Stat* stats;            // [2][rows][chunks]
    Decision* decisions;    // [n]
    int picks;              // chunks of PICK
    double* masses;         // [n][picks] of max(p - q, 0)
};

__device__ __forceinline__ double inverse(float t) { return t > 0.f ? 1.0 / (double)fminf(t, 1e30f) : 0.0; }       // 0: greedy

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

// the last certain row of a request with rows first .. end - 1: those in front of it are followed by a token that needs no verification
__device__ __forceinline__ int last_certain(const Verify& v, int r, int first, int end) {
    return v.certain ? first + min(max(v.certain[r], 1), end - first) - 1 : first;
}

// E elements a thread, in pieces of 8
template <class T, int E>
__global__ __launch_bounds__(THREADS) void verify_stats(const VerifyArgs a) {
    const Verify& v = a.v;
    __shared__ double sums[WAVES];
    __shared__ float tops[WAVES];
    __shared__ int counts[WAVES];
    const int tid = threadIdx.x, row = blockIdx.x / a.chunks, chunk = blockIdx.x - row * a.chunks, side = blockIdx.y;
    // the request that the row belongs to: the last that starts at or before it
    int count = 0;
    for (int r = 1 + tid; r < v.n; r += THREADS) count += v.row_start[r] <= row;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) count += __shfl_xor(count, o);
    if ((tid & 63) == 0) counts[tid >> 6] = count;
    const T* from = (side ? (const T*)v.draft + row * v.ld_draft : (const T*)v.target + row * v.ld_target) + (int64_t)chunk * a.chunk;
    const int n = min(a.chunk, v.vocab - chunk * a.chunk);
    Eight<T> x[E / 8];
    auto ask = [&] {
#pragma unroll
        for (int j = 0; j < E / 8; ++j) {
            const int i = (j * THREADS + tid) * 8;
            if (i + 8 <= n) x[j].load(from + i);
        }
    };
    // a row of the target is asked for meanwhile; one of the draft only once it is known to be a draft's: the others need not be there.  With
    // prompts most rows of the target are not needed either
    const bool early = !side && !v.certain;
    if (early) ask();
    __syncthreads();
    int owner = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) owner += counts[w];
    const int first = v.row_start[owner];
    const int end = min(v.row_start[owner + 1], v.rows);
    if (row >= end || row < first || (v.seq_len && v.seq_len[owner] <= 0)) return;
    const int from_row = last_certain(v, owner, max(first, 0), end);
    if (row < from_row || (side && row == from_row)) return;
    if (!early) ask();
    const double inv_t = inverse(v.temperature[owner]);
    // the elements that are no whole piece of 8: at most 7, one a thread
    const int tail = n & ~7;
    const float last = tail + tid < n ? logit((float)from[tail + tid]) : -INFINITY;
    float best = last;
#pragma unroll
    for (int j = 0; j < E / 8; ++j)
        if ((j * THREADS + tid) * 8 + 8 <= n)
#pragma unroll
            for (int e = 0; e < 8; ++e) best = fmaxf(best, x[j].at(e));            // the number, of a NaN and a number
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) best = fmaxf(best, __shfl_xor(best, o));
    if ((tid & 63) == 0) tops[tid >> 6] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) best = fmaxf(best, tops[w]);
    double sum = 0.0;
    int at = 0x7fffffff;
    if (inv_t > 0.0) {
        if (best > -INFINITY) {
            const Weight weight(best, inv_t);
            sum = weight(last);
#pragma unroll
            for (int j = 0; j < E / 8; ++j) {
                if ((j * THREADS + tid) * 8 + 8 > n) break;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += weight(x[j].at(e));
            }
            sum = block_sum(sum, sums);
        }
    } else {
        // greedy: where it is
        if (last == best) at = tail + tid;
#pragma unroll
        for (int j = E / 8 - 1; j >= 0; --j) {
            const int i = (j * THREADS + tid) * 8;
            if (i + 8 <= n)
#pragma unroll
                for (int e = 7; e >= 0; --e) at = x[j].at(e) == best ? i + e : at;
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) at = min(at, __shfl_xor(at, o));
        if ((tid & 63) == 0) counts[tid >> 6] = at;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) at = min(at, counts[w]);
        at += chunk * a.chunk;
    }
    if (tid == 0) a.stats[((int64_t)side * v.rows + row) * a.chunks + chunk] = Stat{best, at, sum};
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
        const Weight weight(top.v, inv_t);
        for (int c = lane; c < a.chunks; c += 64) {
            if (a.chunks > 64) mine = from[c];
            sum += mine.sum * weight(mine.top);
        }
        sum = wave_sum(sum);
    }
    return Stat{top.v, top.i, sum};
}

// the shares of tokens in either model
template <class T>
struct Shares {
    const T *target, *draft;
    Weight p_weight, q_weight;
    double p_norm, q_norm;
    int drafted;
    __device__ Shares(const VerifyArgs& a, const Decision& d)
        : p_weight(d.target_top, d.inv_t), q_weight(d.draft_top > -INFINITY ? d.draft_top : 0.f, d.inv_t) {
        target = (const T*)a.v.target + d.row * a.v.ld_target;
        drafted = d.drafted;
        draft = drafted >= 0 && a.v.draft ? (const T*)a.v.draft + (d.row + 1) * a.v.ld_draft : nullptr;
        p_norm = d.p_norm;
        q_norm = d.q_norm;
    }
    __device__ double p(float v) const { return p_weight(v) * p_norm; }
    __device__ double q(float v, int i) const { return draft ? q_weight(v) * q_norm : (double)(i == drafted); }
};
// max(p - q, 0), or p behind the last draft, of a thread's 8 tokens of one chunk of PICK; gives the first of them
constexpr int PICK = THREADS * 8;
template <class T>
__device__ __forceinline__ int shares_of_chunk(const Shares<T>& s, int chunk, int vocab, double (&rest)[8]) {
    const int i = chunk * PICK + threadIdx.x * 8;
    float x[8], y[8];
    if (i + 8 <= vocab) {
        Eight<T> e;
        e.load(s.target + i);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = e.at(j);
        if (s.draft) {
            e.load(s.draft + i);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = e.at(j);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[j] = i + j < vocab ? (float)s.target[i + j] : -INFINITY;
            y[j] = s.draft && i + j < vocab ? (float)s.draft[i + j] : -INFINITY;
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        rest[j] = s.p(x[j]);
        if (s.drafted >= 0) rest[j] = fmax(rest[j] - s.q(s.draft ? y[j] : 0.f, i + j), 0.0);
    }
    return i;
}

// One workgroup per request: its rows from the last certain one on joined, a wave per row and eight rows at a time, up to the first draft that does not stand
// (five rows of 50272: 5.4 us, with four at a time 6.7; 64 requests of 32000: 6.2 and 9.1).
constexpr int DECIDE_WAVES = 8;
template <class T>
__global__ __launch_bounds__(DECIDE_WAVES * 64) void verify_decide(const VerifyArgs a) {
    const Verify& v = a.v;
    __shared__ int stop, best;
    const int tid = threadIdx.x, wave = tid >> 6, r = blockIdx.x;
    const int first = max(v.row_start[r], 0), end = min(v.row_start[r + 1], v.rows);
    const double inv_t = inverse(v.temperature[r]);
    const bool greedy = inv_t == 0.0;
    // no rows, or refused by the plan: its rows have no slots, so no attention and no logits stand behind them
    if (first >= end || (v.seq_len && v.seq_len[r] <= 0)) {
        if (tid == 0) {
            v.kept[r] = 0;
            if (v.len_out) v.len_out[r] = v.len_in[r];
            a.decisions[r].row = -1;
        }
        for (int i = first + tid; i < end; i += DECIDE_WAVES * 64) v.out[i] = -1;
        return;
    }
    for (int at = last_certain(v, r, first, end);; at += DECIDE_WAVES) {
        if (tid == 0) stop = end;
        __syncthreads();
        const int row = at + wave;
        Decision d{};
        bool stands = true, empty = false;
        int token = -1, top_at = -1;
        if (row < end) {
            token = row + 1 < end ? v.tokens[row + 1] : -1;
            const bool valid = token >= 0 && token < v.vocab;
            const Stat t = row_stat(a, 0, row, inv_t);
            const Stat q = valid && v.draft && !greedy ? row_stat(a, 1, row + 1, inv_t) : Stat{-INFINITY, 0, 0.0};
            empty = t.top == -INFINITY;
            top_at = empty ? -1 : t.at;
            d = Decision{first, end, row, valid ? token : -1, t.top, q.top, v.u_sample[r], 0u, inv_t, 1.0 / t.sum, q.top > -INFINITY ? 1.0 / q.sum : 0.0};
            if (greedy) {
                stands = row + 1 < end && !empty && token == t.at;
            } else if (valid && !empty) {
                const Shares<T> s(a, d);
                stands = (double)v.u_accept[row + 1] * s.q(s.draft ? (float)s.draft[token] : 0.f, token) < s.p((float)s.target[token]);
            } else {
                stands = false;                           // also the last row of a request, which has no draft behind it
            }
            if (!stands && (tid & 63) == 0) atomicMin(&stop, row);
        }
        __syncthreads();
        if (row < end && row == stop && (tid & 63) == 0) {
            best = top_at;
            const int gained = row - first + 1;
            v.kept[r] = gained;
            if (v.len_out) v.len_out[r] = v.len_in[r] + gained;
            if (greedy || empty) d.row = -1;
            a.decisions[r] = d;
        }
        __syncthreads();
        if (stop < end) break;
        __syncthreads();
    }
    // the tokens; one that is drawn is put in its place by verify_draw
    for (int i = first + tid; i < end; i += DECIDE_WAVES * 64) v.out[i] = i < stop ? v.tokens[i + 1] : i == stop ? best : -1;
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

// What goes from workgroup to workgroup of one launch is stored and loaded past the L2 of either's XCD.
__device__ __forceinline__ void put(double* p, double v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ double get(const double* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// The mass of every chunk of the row that the next token comes from; the workgroup of a request that is done last finds the chunk in which the
// random number falls, and the token in it.
template <class T>
__global__ __launch_bounds__(THREADS) void verify_draw(const VerifyArgs a) {
    const Verify& v = a.v;
    __shared__ double sums[WAVES], base;
    __shared__ int found, last;
    const int tid = threadIdx.x, r = blockIdx.y;
    const Decision d = a.decisions[r];
    if (d.row < 0) return;
    Shares<T> s(a, d);
    double* masses = a.masses + (int64_t)r * a.picks;
    double rest[8], mine = 0.0, total;
    shares_of_chunk(s, blockIdx.x, v.vocab, rest);
#pragma unroll
    for (int j = 0; j < 8; ++j) mine += rest[j];
    mine = wave_sum(mine);
    if ((tid & 63) == 0) sums[tid >> 6] = mine;
    __syncthreads();
    if (tid == 0) {
        put(masses + blockIdx.x, (sums[0] + sums[1]) + (sums[2] + sums[3]));
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
        __builtin_amdgcn_s_waitcnt(0x0F70);              // vmcnt(0): the store has been acknowledged before the arrival is counted
        last = (int)__hip_atomic_fetch_add(&a.decisions[r].arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (last != a.picks - 1) return;
    // chunks, a run of them per thread
    const int each = (a.picks + THREADS - 1) / THREADS, c0 = min(tid * each, a.picks), c1 = min(c0 + each, a.picks);
    mine = 0.0;
    for (int c = c0; c < c1; ++c) mine += get(masses + c);
    double before = sum_before(mine, sums, total);
    if (!(total > 0.0)) {
        // p - q leaves nothing: p itself, whose chunks are summed here, as this is not met but for equal distributions
        s.drafted = -1;
        s.draft = nullptr;
        for (int c = 0; c < a.picks; ++c) {
            shares_of_chunk(s, c, v.vocab, rest);
            double here = 0.0;
#pragma unroll
            for (int j = 0; j < 8; ++j) here += rest[j];
            here = block_sum(here, sums);
            if (c >= c0 && c < c1) {
                put(masses + c, here);
                mine += here;
            }
        }
        before = sum_before(mine, sums, total);
    }
    const double goal = (double)d.goal * total;
    if (tid == 0) { found = 0x7fffffff; last = -1; }
    __syncthreads();
    double upto = before;
    if (mine > 0.0) {
        // the thread's first chunk that passes the goal, or its last one with a share
        int here = -1, passes = 0x7fffffff;
        for (int c = c0; c < c1; ++c) {
            const double m = each == 1 ? mine : get(masses + c);
            upto += m;
            if (m > 0.0) {
                here = c;
                if (upto > goal) {
                    passes = c;
                    break;
                }
            }
        }
        if (passes < 0x7fffffff) atomicMin(&found, passes);
        atomicMax(&last, here);
    }
    __syncthreads();
    const int chunk = found < a.picks ? found : last;
    if (chunk >= c0 && chunk < c1) {                       // the sum in front of the chunk, as its thread has it
        upto = before;
        for (int c = c0; c < chunk; ++c) upto += get(masses + c);
        base = upto;
    }
    __syncthreads();
    if (tid == 0) { found = 0x7fffffff; last = -1; }
    const int i = shares_of_chunk(s, chunk, v.vocab, rest);
    double here = 0.0;
#pragma unroll
    for (int j = 0; j < 8; ++j) here += rest[j];
    upto = sum_before(here, sums, total) + base;
    int holds = 0x7fffffff, positive = -1;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        upto += rest[j];
        if (rest[j] > 0.0) {
            positive = i + j;
            if (upto > goal) holds = min(holds, i + j);
        }
    }
    if (holds < 0x7fffffff) atomicMin(&found, holds);
    if (positive >= 0) atomicMax(&last, positive);          // where the goal is the whole sum but for its rounding: the last token with a share
    __syncthreads();
    if (tid == 0) v.out[d.row] = found < 0x7fffffff ? found : last;
}

struct Layout {
    int chunk, chunks;
    int picks;
    size_t stats, decisions, masses;
};
// Chunks of the first launch: 8192 logits, 4096 or 2048 where that leaves fewer than 1024 workgroups.
Layout layout_of(int n, int rows, int vocab) {
    Layout l;
    l.chunk = 8192;
    while (l.chunk > 2048 && 2 * (int64_t)rows * ((vocab + l.chunk - 1) / l.chunk) < 1024) l.chunk /= 2;
    l.chunks = (vocab + l.chunk - 1) / l.chunk;
    l.stats = 2 * (size_t)rows * l.chunks * sizeof(Stat);
    l.decisions = (size_t)n * sizeof(Decision);
    l.picks = (vocab + PICK - 1) / PICK;
    l.masses = (size_t)n * l.picks * sizeof(double);
    return l;
}

template <class T>
int launch(const Verify& v, void* ws, hipStream_t st) {
    const Layout l = layout_of(v.n, v.rows, v.vocab);
    VerifyArgs a;
    a.v = v;
    a.chunk = l.chunk;
    a.chunks = l.chunks;
    a.picks = l.picks;
    a.stats = (Stat*)ws;
    a.decisions = (Decision*)((char*)ws + l.stats);
    a.masses = (double*)((char*)ws + l.stats + l.decisions);
    if (v.rows > 0) {
        auto stats = l.chunk == 8192 ? verify_stats<T, 32> : l.chunk == 4096 ? verify_stats<T, 16> : verify_stats<T, 8>;
        hipLaunchKernelGGL(stats, dim3((unsigned)(v.rows * l.chunks), v.draft ? 2 : 1), dim3(THREADS), 0, st, a);
        KVPR_HIP(hipGetLastError());
    }
    hipLaunchKernelGGL(verify_decide<T>, dim3((unsigned)v.n), dim3(DECIDE_WAVES * 64), 0, st, a);
    KVPR_HIP(hipGetLastError());
    if (v.rows > 0) {
        hipLaunchKernelGGL(verify_draw<T>, dim3((unsigned)l.picks, (unsigned)v.n), dim3(THREADS), 0, st, a);
        KVPR_HIP(hipGetLastError());
    }
    return KVPR_OK;
}

}  // namespace

size_t verify_workspace_bytes(int n, int rows, int vocab) {
    const Layout l = layout_of(n, rows, vocab);
    return l.stats + l.decisions + l.masses;
}

int launch_verify(const Verify& v, void* ws, hipStream_t st) { return v.f16 ? launch<_Float16>(v, ws, st) : launch<float>(v, ws, st); }

}  // namespace kvpr
