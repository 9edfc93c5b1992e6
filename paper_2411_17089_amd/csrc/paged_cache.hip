// New tokens' rows into the pages of the 4-bit cache, and slots of it back to float16.
//
// Append: a row is [q | k | v] of one token.  q and k are rotated by the token's position (kvpr_rope_table's angles; element i of a
// head with element i + d / 2), q goes out as float16, k and v are packed by the codec of the compressed store into the token's
// slot.  The rotation is evaluated in 64 bits and rounded to float16 once: a code depends on the float16 value, so an ulp
// would now and then move a value by a whole step of the codec.
#include "int4_codec.h"
#include "paged.h"

namespace kvpr {
namespace {

// float64 -> float16 in one rounding: the float32 between is made odd in its last bit where it is inexact, and an odd one is
// neither a float16 nor the middle between two
__device__ __forceinline__ _Float16 to_half(double x) {
    float f = (float)x;
    const double rest = x - (double)f;
    int bits = __float_as_int(f);
    if (rest != 0.0 && !(bits & 1)) bits += (rest > 0.0) == (f > 0.f) ? 1 : -1;
    return (_Float16)__int_as_float(bits);
}

// One wave per head of a token: lane i holds element i and, for d = 128, element i + 64 too.
template <int D>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedShape s, const _Float16* __restrict__ qkv, int64_t ld,
                                                           const int32_t* __restrict__ slots, const int32_t* __restrict__ positions,
                                                           const float2* __restrict__ rope, int n_pos, _Float16* __restrict__ q_out,
                                                           int64_t ldq, uint8_t* __restrict__ pages) {
    constexpr int E = D / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = blockIdx.x;
    const int slot = slots[row];
    const int position = rope ? positions[row] : 0;
    if (rope && (position < 0 || position >= n_pos)) return;
    const bool kept = slot >= 0 && slot < s.n_pages * s.page;
    const int page = kept ? slot >> s.page_log2 : 0, t = kept ? slot & (s.page - 1) : 0;
    for (int head = (q_out ? 0 : s.heads) + wave; head < s.heads + 2 * s.kv_heads; head += 4) {
        const bool is_q = head < s.heads, is_k = !is_q && head < s.heads + s.kv_heads;
        const _Float16* src = qkv + (int64_t)row * ld + (int64_t)head * D;
        _Float16 x[E];
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = src[lane + 64 * e];
        if (rope && (is_q || is_k)) {
            const int i = lane & (D / 2 - 1);
            const float2 cs = rope[(int64_t)position * (D / 2) + i];
            if constexpr (D == 128) {
                const double a = (double)(float)x[0], b = (double)(float)x[1];
                x[0] = to_half(a * cs.x - b * cs.y);
                x[1] = to_half(b * cs.x + a * cs.y);
            } else {
                const float other = __shfl_xor((float)x[0], 32);
                const double a = (double)(float)x[0], b = (double)other;
                x[0] = to_half(lane < 32 ? a * cs.x - b * cs.y : a * cs.x + b * cs.y);
            }
        }
        if (is_q) {
#pragma unroll
            for (int e = 0; e < E; ++e) q_out[(int64_t)row * ldq + (int64_t)head * D + lane + 64 * e] = x[e];
            continue;
        }
        if (!kept) continue;
        uint8_t* block = pages + (int64_t)page * s.page_bytes() + (int64_t)(is_k ? head - s.heads : head - s.heads - s.kv_heads) * s.block_bytes();
#pragma unroll
        for (int e = 0; e < E; ++e) {
            float mn = (float)x[e], mx = mn;
            for (int o = 32; o > 0; o >>= 1) {
                mn = fminf(mn, __shfl_xor(mn, o));
                mx = fmaxf(mx, __shfl_xor(mx, o));
            }
            const _Float16 scale16 = int4_scale(mn, mx);
            const float scale = (float)scale16;
            const int code = scale > 0.f ? (int)int4_code((float)x[e], scale, mn, __builtin_amdgcn_rcpf(scale)) : 0;
            const int pair = code | __shfl_xor(code, 1) << 4;
            const int k = 32 * e + lane / 2;
            if (!(lane & 1))
                block[is_k ? t * (D / 2) + key_place<D>(k) : s.page * (D / 2) + (t >> 2) * (2 * D) + value_place<D>(k) * 4 + (t & 3)] = (uint8_t)pair;
            if (lane == 0) {
                _Float16* meta = reinterpret_cast<_Float16*>(block + s.page * D + (is_k ? 0 : s.page * (D / 16)) + (t * (D / 64) + e) * 4);
                meta[0] = scale16;
                meta[1] = (_Float16)mn;
            }
        }
    }
}

// One thread per byte of codes: two columns of one head of one row.
template <int D>
__global__ __launch_bounds__(256) void paged_read_kernel(PagedShape s, const uint8_t* __restrict__ pages, const int32_t* __restrict__ slots,
                                                         _Float16* __restrict__ kv, int64_t ld) {
    const int row = blockIdx.x, slot = slots[row];
    if (slot < 0 || slot >= s.n_pages * s.page) return;
    const int page = slot >> s.page_log2, t = slot & (s.page - 1);
    const int per_side = s.kv_heads * (D / 2);
    for (int i = threadIdx.x; i < 2 * per_side; i += 256) {
        const bool is_k = i < per_side;
        const int j = is_k ? i : i - per_side, head = j / (D / 2), k = j % (D / 2);
        const uint8_t* block = pages + (int64_t)page * s.page_bytes() + (int64_t)head * s.block_bytes();
        const int byte = block[is_k ? t * (D / 2) + key_place<D>(k) : s.page * (D / 2) + (t >> 2) * (2 * D) + value_place<D>(k) * 4 + (t & 3)];
        const _Float16* meta = reinterpret_cast<const _Float16*>(block + s.page * D + (is_k ? 0 : s.page * (D / 16)) + (t * (D / 64) + k / 32) * 4);
        const float scale = (float)meta[0], mn = (float)meta[1];
        _Float16* out = kv + (int64_t)row * ld + 2 * i;
        out[0] = (_Float16)((float)(byte & 15) * scale + mn);
        out[1] = (_Float16)((float)(byte >> 4) * scale + mn);
    }
}

}  // namespace

int launch_paged_append(const PagedShape& s, const void* qkv, int64_t ld, const int32_t* slots, const int32_t* positions, int rows,
                        const void* rope, int n_pos, void* q_out, int64_t ldq, void* pages, hipStream_t st) {
    auto kern = s.d == 128 ? paged_append_kernel<128> : paged_append_kernel<64>;
    hipLaunchKernelGGL(kern, dim3((unsigned)rows), dim3(256), 0, st, s, (const _Float16*)qkv, ld, slots, positions, (const float2*)rope,
                       n_pos, (_Float16*)q_out, ldq, (uint8_t*)pages);
    KVPR_HIP(hipGetLastError());
    return KVPR_OK;
}

int launch_paged_read(const PagedShape& s, const void* pages, const int32_t* slots, int rows, void* kv, int64_t ld, hipStream_t st) {
    auto kern = s.d == 128 ? paged_read_kernel<128> : paged_read_kernel<64>;
    hipLaunchKernelGGL(kern, dim3((unsigned)rows), dim3(256), 0, st, s, (const uint8_t*)pages, slots, (_Float16*)kv, ld);
    KVPR_HIP(hipGetLastError());
    return KVPR_OK;
}

}  // namespace kvpr
