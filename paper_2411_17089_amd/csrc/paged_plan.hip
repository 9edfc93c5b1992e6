// The plan of one step of a ragged batch, on the GPU: pages given back and taken, row offsets, slots and positions of the new
// tokens, all from the requests' lengths (formulas at kvpr_paged_plan).
//
// One workgroup: three prefix sums over the requests (pages given back, pages taken, rows), then the new tokens.
#include "paged.h"

namespace kvpr {
namespace {

constexpr int THREADS = 1024, WAVES = THREADS / 64;

// exclusive prefix sum over the workgroup; total: the sum of all.  part: WAVES numbers of LDS
template <class T>
__device__ __forceinline__ T block_scan(T v, T* part, T& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    T s = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const T u = __shfl_up(s, o);
        if (lane >= o) s += u;
    }
    __syncthreads();
    if (lane == 63) part[wave] = s;
    __syncthreads();
    T before = 0;
    total = 0;
    for (int w = 0; w < WAVES; ++w) {
        if (w < wave) before += part[w];
        total += part[w];
    }
    return before + s - v;
}

__device__ __forceinline__ int32_t low32(int64_t v) { return (int32_t)(v < 0x7fffffff ? v : 0x7fffffff); }

__global__ __launch_bounds__(THREADS) void paged_plan_kernel(PagedShape s, PagedPlan p) {
    __shared__ int64_t part[WAVES];
    const int tid = threadIdx.x, page = s.page;
    struct Request { int held; int64_t need, want, base, fresh; };
    auto request = [&](int r) {
        Request q{0, 0, 0, 0, 0};
        if (r >= p.n) return q;
        q.base = max(p.base_len[r], 0);
        q.fresh = max(p.new_len[r], 0);
        q.held = min(max(p.held_in[r], 0), s.width);
        q.want = q.base + q.fresh;
        q.need = (q.want + page - 1) >> s.page_log2;
        return q;
    };
    const int count = min(max(*p.count_in, 0), s.n_pages);
    // pages given back
    int64_t given = 0, total;
    for (int r0 = 0; r0 < p.n; r0 += THREADS) {
        const int r = r0 + tid;
        const Request q = request(r);
        const int64_t gives = max((int64_t)q.held - q.need, (int64_t)0);
        const int64_t at = count + given + block_scan(gives, part, total);
        for (int64_t i = 0; i < gives && at + i < s.n_pages; ++i) p.free_pages[at + i] = p.table[(int64_t)r * s.width + q.need + i];
        given += total;
    }
    __syncthreads();
    const int64_t avail = min((int64_t)count + given, (int64_t)s.n_pages);
    // pages taken, rows
    int64_t taken = 0, rows = 0, granted_pages = 0, refused = 0;
    for (int r0 = 0; r0 < p.n; r0 += THREADS) {
        const int r = r0 + tid;
        const Request q = request(r);
        const bool fits = q.need <= s.width;
        const int64_t takes = fits ? max(q.need - q.held, (int64_t)0) : 0;
        const int64_t before = taken + block_scan(takes, part, total);
        taken += total;
        const bool granted = fits && (takes == 0 || before + takes <= avail);
        if (r < p.n) {
            if (granted)
                for (int64_t i = 0; i < takes; ++i) p.table[(int64_t)r * s.width + q.held + i] = p.free_pages[avail - 1 - before - i];
            p.seq_len[r] = granted ? (int32_t)q.want : 0;
            p.held_out[r] = granted ? (int32_t)q.need : q.held;
        }
        const int64_t start = rows + block_scan(q.fresh, part, total);
        rows += total;
        if (r < p.n) p.row_start[r] = low32(start);
        block_scan((int64_t)(granted ? takes : 0), part, total);
        granted_pages += total;
        block_scan((int64_t)(r < p.n && !granted), part, total);
        refused += total;
    }
    if (tid == 0) {
        p.row_start[p.n] = low32(rows);
        *p.count_out = (int32_t)(avail - granted_pages);
        *p.refused = (int32_t)refused;
    }
    __threadfence_block();
    __syncthreads();
    // new tokens: the request of a row is the last one that starts at or before it
    for (int t = tid; t < p.max_rows; t += THREADS) {
        int32_t slot = -1, position = 0;
        if (t < rows) {
            int lo = 0, hi = p.n - 1;
            while (lo < hi) {
                const int mid = (lo + hi + 1) / 2;
                if (p.row_start[mid] <= t) lo = mid; else hi = mid - 1;
            }
            position = low32((int64_t)max(p.base_len[lo], 0) + t - p.row_start[lo]);
            if (position < p.seq_len[lo]) {
                const int32_t id = p.table[(int64_t)lo * s.width + (position >> s.page_log2)];
                if (id >= 0 && id < s.n_pages) slot = id * page + (position & (page - 1));
            }
        }
        p.slots[t] = slot;
        p.positions[t] = position;
    }
}

}  // namespace

int launch_paged_plan(const PagedShape& s, const PagedPlan& p, hipStream_t st) {
    hipLaunchKernelGGL(paged_plan_kernel, dim3(1), dim3(THREADS), 0, st, s, p);
    KVPR_HIP(hipGetLastError());
    return KVPR_OK;
}

}  // namespace kvpr
