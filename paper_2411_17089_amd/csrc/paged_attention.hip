// Attention of a ragged batch's new tokens over a paged 4-bit cache (formulas at kvpr_paged_attention).
//
// One wave per (query head, new token): 64 positions at a time, a lane scores one position, then owns d / 64 columns of the sum.
#include "paged.h"
#include <math.h>

namespace kvpr {
namespace {

template <int D, class Q>
__global__ __launch_bounds__(64) void paged_attention_kernel(PagedShape s, const Q* __restrict__ q, int64_t ldq, const uint8_t* __restrict__ pages,
                                                             const int32_t* __restrict__ table, const int32_t* __restrict__ row_start,
                                                             const int32_t* __restrict__ seq_len, int rows, _Float16* __restrict__ z,
                                                             int64_t ldz, float scale_log2) {
    constexpr int E = D / 64;
    const int lane = threadIdx.x, head = blockIdx.x, r = blockIdx.y, kv_head = head / (s.heads / s.kv_heads);
    const int first = row_start[r], m = row_start[r + 1] - first;
    const int len = min(max(seq_len[r], 0), s.width * s.page);
    __shared__ float qs[D], ps[64];
    for (int i = blockIdx.z; i < m; i += gridDim.z) {
        const int row = first + i;
        if (row < 0 || row >= rows) break;
        const int seen = min(len, seq_len[r] - m + i + 1);
        __syncthreads();
        for (int e = 0; e < E; ++e) qs[lane + 64 * e] = (float)q[row * ldq + (int64_t)head * D + lane + 64 * e];
        __syncthreads();
        float m_run = -0x1p126f, l_run = 0.f, acc[E] = {};     // finite, so that no difference of maxima is NaN
        for (int t0 = 0; t0 < seen; t0 += 64) {
            auto block_of = [&](int t) -> const uint8_t* {
                const int id = table[(int64_t)r * s.width + (t >> s.page_log2)];
                return id >= 0 && id < s.n_pages ? pages + id * s.page_bytes() + kv_head * s.block_bytes() : nullptr;
            };
            const int t = t0 + lane;
            float score = -INFINITY;
            const uint8_t* block = t < seen ? block_of(t) : nullptr;
            if (block) {
                const int u = t & (s.page - 1);
                score = 0.f;
                for (int g = 0; g < E; ++g) {
                    const _Float16* meta = reinterpret_cast<const _Float16*>(block + s.page * D + (u * E + g) * 4);
                    float dot = 0.f, sum = 0.f;
                    for (int k = 0; k < 32; ++k) {
                        const int byte = block[u * (D / 2) + key_place<D>(32 * g + k)];
                        const float a = qs[64 * g + 2 * k], b = qs[64 * g + 2 * k + 1];
                        dot += a * (float)(byte & 15) + b * (float)(byte >> 4);
                        sum += a + b;
                    }
                    score += dot * (float)meta[0] + sum * (float)meta[1];
                }
                score *= scale_log2;
            }
            float m_new = score;
            for (int o = 32; o > 0; o >>= 1) m_new = fmaxf(m_new, __shfl_xor(m_new, o));
            m_new = fmaxf(m_new, m_run);
            const float p = exp2f(score - m_new), keep = exp2f(m_run - m_new);
            float p_sum = p;
            for (int o = 32; o > 0; o >>= 1) p_sum += __shfl_xor(p_sum, o);
            l_run = l_run * keep + p_sum;
            m_run = m_new;
            ps[lane] = p;
            __syncthreads();
            for (int e = 0; e < E; ++e) acc[e] *= keep;
            for (int j = 0; j < 64 && t0 + j < seen; ++j) {
                const uint8_t* from = block_of(t0 + j);
                if (!from) continue;
                const int u = (t0 + j) & (s.page - 1);
                for (int e = 0; e < E; ++e) {
                    const int k = 32 * e + lane / 2;
                    const int byte = from[s.page * (D / 2) + (u >> 2) * (2 * D) + value_place<D>(k) * 4 + (u & 3)];
                    const _Float16* meta = reinterpret_cast<const _Float16*>(from + s.page * D + s.page * (D / 16) + (u * E + e) * 4);
                    const int code = lane & 1 ? byte >> 4 : byte & 15;
                    acc[e] += ps[j] * ((float)code * (float)meta[0] + (float)meta[1]);
                }
            }
            __syncthreads();
        }
        for (int e = 0; e < E; ++e)
            z[row * ldz + (int64_t)head * D + lane + 64 * e] = (_Float16)(l_run == 0.f ? 0.f : acc[e] / l_run);
    }
}

}  // namespace

size_t paged_attention_workspace_bytes(const PagedShape&, int, int, int, int) { return 16; }

int launch_paged_attention(const PagedShape& s, const PagedAttention& a, void*, size_t, hipStream_t st) {
    const float scale_log2 = (float)(1.4426950408889634 / sqrt((double)s.d));
    const dim3 grid((unsigned)s.heads, (unsigned)a.n, (unsigned)(a.max_new < 1024 ? a.max_new : 1024));
#define KVPR_LAUNCH(D_, Q_)                                                                                                                   \
    hipLaunchKernelGGL((paged_attention_kernel<D_, Q_>), grid, dim3(64), 0, st, s, (const Q_*)a.q, a.ldq, (const uint8_t*)a.pages, a.table,   \
                       a.row_start, a.seq_len, a.rows, (_Float16*)a.z, a.ldz, scale_log2)
    if (s.d == 128) {
        if (a.q_f32) KVPR_LAUNCH(128, float); else KVPR_LAUNCH(128, _Float16);
    } else {
        if (a.q_f32) KVPR_LAUNCH(64, float); else KVPR_LAUNCH(64, _Float16);
    }
#undef KVPR_LAUNCH
    KVPR_HIP(hipGetLastError());
    return KVPR_OK;
}

}  // namespace kvpr
