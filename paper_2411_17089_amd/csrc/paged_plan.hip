// The plan of one step of a ragged batch, on the GPU: pages given back and taken, row offsets, slots and positions of the new
// tokens, all from the requests' lengths (formulas at kvpr_paged_plan).
//
// The work is a chain of latencies, not of bytes: three prefix sums over the requests (pages given back, pages taken, rows) in one
// pass of one workgroup, then the pages, a thread each whatever request they belong to (a thread per request walked up to 128 pages
// one by one), then the new tokens, a thread each: by the same workgroup, or, where they are many, by a launch of their own.
// 8 requests 4.6 us; 512 requests, 31500 new tokens 8.3 and 4.4 us, 88 by one workgroup with searches in global memory.
#include "paged.h"

namespace kvpr {
namespace {

constexpr int ROWS_HERE = 2048;         // new tokens up to which the first launch places them itself

struct Three { int64_t v[3]; };

// inclusive prefix sums over the lanes of a wave
__device__ __forceinline__ Three wave_scan(Three s) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1)
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const int64_t u = __shfl_up(s.v[i], o);
            if ((int)(threadIdx.x & 63) >= o) s.v[i] += u;
        }
    return s;
}

// exclusive prefix sums over the workgroup of three numbers a thread; total: the sums of all.  part: WAVES + 1 of LDS
template <int WAVES>
__device__ __forceinline__ Three block_scan(const Three& x, Three* part, Three& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Three s = wave_scan(x);
    __syncthreads();
    if (lane == 63) part[wave] = s;
    __syncthreads();
    if (wave == 0) {
        Three w = lane < WAVES ? part[lane] : Three{{0, 0, 0}};
        const Three own = w;
        w = wave_scan(w);
        if (lane == WAVES - 1) part[WAVES] = w;
#pragma unroll
        for (int i = 0; i < 3; ++i) w.v[i] -= own.v[i];
        if (lane < WAVES) part[lane] = w;
    }
    __syncthreads();
    total = part[WAVES];
#pragma unroll
    for (int i = 0; i < 3; ++i) s.v[i] += part[wave].v[i] - x.v[i];
    return s;
}

__device__ __forceinline__ int32_t low32(int64_t v) { return (int32_t)(v < 0x7fffffff ? v : 0x7fffffff); }

// the last i in [0, n) with from[i] <= x; from[0] <= x
__device__ __forceinline__ int last_upto(const int32_t* from, int n, int x) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (from[mid] <= x) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// row t of the step; row_start: n + 1 numbers, read from where they are near
__device__ __forceinline__ void place_row(const PagedShape& s, const PagedPlan& p, const int32_t* row_start, int t) {
    int32_t slot = -1, position = 0;
    if (t < row_start[p.n]) {
        const int r = last_upto(row_start, p.n, t);
        position = low32((int64_t)max(p.base_len[r], 0) + t - row_start[r]);
        if (position < p.seq_len[r]) {
            const int32_t id = p.table[(int64_t)r * s.width + (position >> s.page_log2)];
            if (id >= 0 && id < s.n_pages) slot = id * s.page + (position & (s.page - 1));
        }
    }
    p.slots[t] = slot;
    p.positions[t] = position;
}

// For at most THREADS requests (ONCE) each thread reads its own once and the others' pages from LDS.
template <int THREADS, bool ONCE>
__global__ __launch_bounds__(THREADS) void paged_plan_kernel(PagedShape s, PagedPlan p) {
    constexpr int WAVES = THREADS / 64, MOST = ONCE ? THREADS : kMaxRequests;
    __shared__ Three part[WAVES + 1];
    __shared__ int32_t given_at[MOST + 1], taken_at[MOST + 1];      // sums before a request
    __shared__ int32_t held_of[ONCE ? THREADS : 1], need_of[ONCE ? THREADS : 1];
    __shared__ int granted_pages, refused;
    const int tid = threadIdx.x, page = s.page;
    struct Request { int held; int64_t need, want, fresh; };
    auto request = [&](int r) {
        Request q;
        q.fresh = max(p.new_len[r], 0);
        q.held = min(max(p.held_in[r], 0), s.width);
        q.want = (int64_t)max(p.base_len[r], 0) + q.fresh;
        q.need = (q.want + page - 1) >> s.page_log2;
        return q;
    };
    Request mine{0, 0, 0, 0};
    if (ONCE && tid < p.n) mine = request(tid);
    auto own = [&](int r) { return ONCE ? mine : request(r); };     // of a thread's own r
    auto takes = [&](const Request& q) { return q.need <= s.width && q.need > q.held ? q.need - q.held : (int64_t)0; };
    const int count = min(max(*p.count_in, 0), s.n_pages);
    Three sum{{0, 0, 0}};                               // pages given back, pages taken, rows
    for (int r0 = 0; r0 < p.n; r0 += THREADS) {
        const int r = r0 + tid;
        Three x{{0, 0, 0}}, total;
        if (r < p.n) {
            const Request q = own(r);
            if (ONCE) { held_of[r] = q.held; need_of[r] = low32(q.need); }
            x = Three{{max((int64_t)q.held - q.need, (int64_t)0), takes(q), q.fresh}};
        }
        const Three before = block_scan<WAVES>(x, part, total);
        if (r < p.n) {
            given_at[r] = low32(sum.v[0] + before.v[0]);
            taken_at[r] = low32(sum.v[1] + before.v[1]);
            p.row_start[r] = low32(sum.v[2] + before.v[2]);
        }
#pragma unroll
        for (int i = 0; i < 3; ++i) sum.v[i] += total.v[i];
    }
    if (tid == 0) {
        given_at[p.n] = low32(sum.v[0]);
        taken_at[p.n] = low32(sum.v[1]);
        p.row_start[p.n] = low32(sum.v[2]);
        granted_pages = refused = 0;
    }
    __syncthreads();
    // pages given back go onto the stack
    const int given = min(given_at[p.n], s.n_pages - count), avail = count + given;
    for (int k = tid; k < given; k += THREADS) {
        const int r = last_upto(given_at, p.n, k);
        const int64_t need = ONCE ? need_of[r] : request(r).need;
        p.free_pages[count + k] = p.table[(int64_t)r * s.width + need + (k - given_at[r])];
    }
    __syncthreads();
    // pages come off it; the requests that find theirs are those whose sum stays within it
    for (int k = tid; k < min(taken_at[p.n], avail); k += THREADS) {
        const int r = last_upto(taken_at, p.n, k);
        if (taken_at[r + 1] > avail) continue;
        p.table[(int64_t)r * s.width + (ONCE ? held_of[r] : request(r).held) + (k - taken_at[r])] = p.free_pages[avail - 1 - k];
    }
    __syncthreads();                                    // held_out may be held_in
    int most = 0, none = 0;
    for (int r = tid; r < p.n; r += THREADS) {
        const Request q = own(r);
        const bool granted = q.need <= s.width && (takes(q) == 0 || taken_at[r + 1] <= avail);
        if (takes(q) > 0 && granted) most = max(most, taken_at[r + 1]);
        none += !granted;
        p.seq_len[r] = granted ? (int32_t)q.want : 0;
        p.held_out[r] = granted ? (int32_t)q.need : q.held;
    }
    if (most) atomicMax(&granted_pages, most);
    if (none) atomicAdd(&refused, none);
    __syncthreads();
    if (tid == 0) {
        *p.count_out = avail - granted_pages;
        *p.refused = refused;
    }
    if (p.max_rows > ROWS_HERE) return;
    for (int r = tid; r <= p.n; r += THREADS) given_at[r] = p.row_start[r];
    __syncthreads();
    for (int t = tid; t < p.max_rows; t += THREADS) place_row(s, p, given_at, t);
}

__global__ __launch_bounds__(256) void paged_rows_kernel(PagedShape s, PagedPlan p) {
    const int t = blockIdx.x * 256 + threadIdx.x;
    if (t < p.max_rows) place_row(s, p, p.row_start, t);
}

}  // namespace

int launch_paged_plan(const PagedShape& s, const PagedPlan& p, hipStream_t st) {
    if (p.n <= 256) hipLaunchKernelGGL((paged_plan_kernel<256, true>), dim3(1), dim3(256), 0, st, s, p);
    else if (p.n <= 1024) hipLaunchKernelGGL((paged_plan_kernel<1024, true>), dim3(1), dim3(1024), 0, st, s, p);
    else hipLaunchKernelGGL((paged_plan_kernel<1024, false>), dim3(1), dim3(1024), 0, st, s, p);
    KVPR_HIP(hipGetLastError());
    if (p.max_rows > ROWS_HERE) {
        hipLaunchKernelGGL(paged_rows_kernel, dim3((unsigned)((p.max_rows + 255) / 256)), dim3(256), 0, st, s, p);
        KVPR_HIP(hipGetLastError());
    }
    return KVPR_OK;
}

}  // namespace kvpr
