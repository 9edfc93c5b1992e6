// New tokens' rows into the pages of the 4-bit cache, and slots of it back to float16.
//
// Append: a row is [q | k | v] of one token.  q and k are rotated by the token's position (kvpr_rope_table's angles; element i of a
// head with element i + d / 2), q goes out as float16, k and v are packed by the codec of the compressed store into the token's
// slot.  The rotation is evaluated in 64 bits and rounded to float16 once: a code depends on the float16 value, so an ulp
// would now and then move a value by a whole step of the codec.
//
// Both kernels stream.  A lane has 8 columns of a head (16 bytes in, one word of codes out), a wave four rows of one head (d = 128) or
// two (d = 64): the codes of a row's keys are 64 bytes in a row, those of four rows 256.  Values lie with the bytes of four positions side by
// side.  Where four rows are the four positions of such a quad (a prompt's rows are), the wave that has the first of them turns
// their bytes over between its lanes and stores whole words; other rows store bytes.
#include "int4_codec.h"
#include "paged.h"
#include <algorithm>

namespace kvpr {
namespace {

// float64 -> float16 in one rounding: the float32 between is made odd in its last bit where it is inexact, and an odd one is
// neither a float16 nor the middle between two.  Zeros (of less than half the smallest float32) and infinities (whose rest is NaN) stay
__device__ __forceinline__ _Float16 to_half(double x) {
    float f = (float)x;
    const double rest = x - (double)f;
    int bits = __float_as_int(f);
    if (fabs(rest) > 0.0 && f != 0.f && !(bits & 1)) bits += (rest > 0.0) == (f > 0.f) ? 1 : -1;
    return (_Float16)__int_as_float(bits);
}

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef uint32_t word2 __attribute__((ext_vector_type(2)));
constexpr int WAVES = 4;

// 8 columns rotated: lane j's element e goes with that of the lane half a head further
template <int D>
__device__ __forceinline__ half8 rotate(half8 x, const float2* __restrict__ rope, int64_t position, int j) {
    constexpr int LANES = D / 8;
    union { half8 h; int w[4]; } mine, other;
    mine.h = x;
#pragma unroll
    for (int i = 0; i < 4; ++i) other.w[i] = __shfl_xor(mine.w[i], LANES / 2);
    const float4* cs = reinterpret_cast<const float4*>(rope + position * (D / 2) + (j & (LANES / 2 - 1)) * 8);
    const double side = j < LANES / 2 ? -1.0 : 1.0;
    half8 out;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 t = cs[i];
        out[2 * i] = to_half(fma(side * (double)(float)other.h[2 * i], (double)t.y, (double)(float)x[2 * i] * (double)t.x));
        out[2 * i + 1] = to_half(fma(side * (double)(float)other.h[2 * i + 1], (double)t.w, (double)(float)x[2 * i + 1] * (double)t.z));
    }
    return out;
}

template <int CTRL>
__device__ __forceinline__ float across(float v) {       // the value of another lane of the same row of 16
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}

struct Packed { uint32_t codes, pair; };
// codes of a lane's 8 columns, and the (scale, minimum) of the group of 64, which 8 lanes share
__device__ __forceinline__ Packed pack(half8 x) {
    float mn = (float)x[0], mx = mn;
#pragma unroll
    for (int i = 1; i < 8; ++i) {
        mn = fminf(mn, (float)x[i]);
        mx = fmaxf(mx, (float)x[i]);
    }
    mn = fminf(mn, across<0xB1>(mn)); mx = fmaxf(mx, across<0xB1>(mx));          // quad_perm [1,0,3,2], [2,3,0,1], row_half_mirror
    mn = fminf(mn, across<0x4E>(mn)); mx = fmaxf(mx, across<0x4E>(mx));
    mn = fminf(mn, across<0x141>(mn)); mx = fmaxf(mx, across<0x141>(mx));
    const _Float16 scale16 = int4_scale(mn, mx);
    const float scale = (float)scale16, r = __builtin_amdgcn_rcpf(scale);
    float part[2];                                       // four codes each as one number below 2^16
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float c[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = int4_code((float)x[4 * i + e], scale, mn, r);
        part[i] = fmaf(fmaf(c[3], 16.f, c[2]), 256.f, fmaf(c[1], 16.f, c[0]));
    }
    union { _Float16 h[2]; uint32_t u; } pair;
    pair.h[0] = scale16;
    pair.h[1] = (_Float16)mn;
    return Packed{scale > 0.f ? (uint32_t)part[0] | (uint32_t)part[1] << 16 : 0u, pair.u};
}

// Byte i of the words of the four lanes l, l ^ 16, l ^ 32, l ^ 48 (in the order of lane >> 4) for lane >> 4 == i.
__device__ __forceinline__ uint32_t turn_over(uint32_t v) {
    const auto half = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    const auto a = __builtin_amdgcn_permlane16_swap(half[0], half[0], false, false), b = __builtin_amdgcn_permlane16_swap(half[1], half[1], false, false);
    const uint32_t i = (threadIdx.x & 63) >> 4, pick = i | (4 + i) << 8 | 0x0C0C0000u;      // 0x0C: a zero byte
    return __builtin_amdgcn_perm(a[1], a[0], pick) | __builtin_amdgcn_perm(b[1], b[0], pick) << 16;
}

template <int D, int HEADS>             // heads that a wave has, one behind the other
__global__ __launch_bounds__(WAVES * 64) void paged_append_kernel(PagedShape s, const _Float16* __restrict__ qkv, int64_t ld,
                                                                  const int32_t* __restrict__ slots, const int32_t* __restrict__ positions, int rows,
                                                                  const float2* __restrict__ rope, int n_pos, _Float16* __restrict__ q_out,
                                                                  int64_t ldq, uint8_t* __restrict__ pages) {
    constexpr int LANES = D / 8, SIDE = 16 / LANES, NG = D / 64;       // lanes of a head, heads side by side
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane >> 4, j = lane & (LANES - 1);
    // the waves of a workgroup have neighbouring rows of the same heads: pairs of 16 positions are one line of memory (with the waves on
    // other heads, and the neighbouring rows on another XCD, 8191 rows of 14336 columns took 101 us)
    const int row0 = (blockIdx.x * WAVES + wave) * 4, row = row0 + sub;
    const int pool = s.n_pages * s.page;
    if (row0 >= rows) return;
    // the slot of a row as far as it is kept
    auto slot_of = [&](int r) {
        if (r < 0 || r >= rows) return -1;
        const int slot = slots[r];
        if (slot < 0 || slot >= pool) return -1;
        if (rope && (positions[r] < 0 || positions[r] >= n_pos)) return -1;
        return slot;
    };
    // slots of rows row0 - 3 .. row0 + 6, a lane each; of a row r: is it one of four rows that are a quad of positions?
    const int near = slot_of(lane < 10 ? row0 - 3 + lane : -1);
    auto quad_of = [&](int r) {          // first row of the quad, or -1
        const int slot = __shfl(near, r - row0 + 3), first = r - (slot & 3);
        bool whole = slot >= 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) whole &= __shfl(near, min(max(first + i - row0 + 3, 0), 9)) == (slot & ~3) + i;
        return whole ? first : -1;
    };
    const int slot = __shfl(near, sub + 3), quad = quad_of(row);
    // the quad that starts here: at most one
    const bool starts = quad == row && row < row0 + 4;
    const uint64_t who = __ballot(starts);
    const int lead = who ? row0 + (__builtin_ctzll(who) >> 4) : -1;     // its first row
    const bool alone = slot >= 0 && quad < 0;
    const int lead_slot = lead >= 0 ? __shfl(near, lead - row0 + 3) : 0;
    const bool there = row < rows, turned = there && (!rope || (positions[row] >= 0 && positions[row] < n_pos));
    const int64_t position = rope && turned ? positions[row] : 0;
    const int q_heads = q_out ? s.heads : 0, units = (q_heads + 2 * s.kv_heads + SIDE - 1) / SIDE;
    const int unit0 = blockIdx.y * HEADS;
    // what a lane has of a unit
    struct Part { bool exists, is_q, is_k; int head; int64_t column; };
    auto part_of = [&](int unit) {
        Part p;
        const int h = unit * SIDE + (SIDE > 1 ? (lane >> 3) & 1 : 0);
        p.exists = unit < units && h < q_heads + 2 * s.kv_heads;
        p.is_q = h < q_heads;
        p.is_k = !p.is_q && h < q_heads + s.kv_heads;
        p.head = h - (p.is_q ? 0 : p.is_k ? q_heads : q_heads + s.kv_heads);
        p.column = (int64_t)(p.is_q ? p.head : p.is_k ? s.heads + p.head : s.heads + s.kv_heads + p.head) * D + j * 8;
        return p;
    };
    auto load = [&](const Part& p, int r, bool ok) {
        return ok && p.exists ? __builtin_nontemporal_load(reinterpret_cast<const half8*>(qkv + r * ld + p.column)) : half8{};
    };
    // of values the rows of the quad that starts here, whose last ones may be the next wave's
    auto load_unit = [&](const Part& p) {
        const bool quad_row = !p.is_q && !p.is_k && lead >= 0;
        return load(p, quad_row ? lead + sub : row, quad_row || there);
    };
    // AHEAD units' columns are on their way together (one ahead: 8191 rows of 14336 columns 106 us, bound by the bytes in flight)
    constexpr int AHEAD = HEADS < 4 ? HEADS : 4;
    half8 ahead[AHEAD];
    for (int unit = unit0; unit < min(unit0 + HEADS, units); unit += AHEAD) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) ahead[i] = load_unit(part_of(unit + i));
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const Part part = part_of(unit + i);
            half8 here = ahead[i];
            const bool exists = part.exists, is_q = part.is_q, is_k = part.is_k;
            const int head = part.head;
            if (is_q || is_k) {
                if (rope) here = rotate<D>(here, rope, position, j);
                if (is_q) {
                    if (turned) *reinterpret_cast<half8*>(q_out + row * ldq + (int64_t)head * D + j * 8) = here;
                    continue;
                }
                const Packed p = pack(here);
                if (slot < 0 || !exists) continue;
                const int t = slot & (s.page - 1);
                uint8_t* block = pages + (int64_t)(slot >> s.page_log2) * s.page_bytes() + (int64_t)head * s.block_bytes();
                *reinterpret_cast<uint32_t*>(block + t * (D / 2) + key_place<D>(4 * j)) = p.codes;
                if ((j & 7) == 0) *reinterpret_cast<uint32_t*>(block + s.page * D + (t * NG + (j >> 3)) * 4) = p.pair;
                continue;
            }
            // values: the quad that starts here, then rows that are in none
            if (lead >= 0) {
                const Packed p = pack(here);
                const uint32_t word = turn_over(p.codes);
                const int t = (lead_slot & (s.page - 1)) + sub;
                uint8_t* block = pages + (int64_t)(lead_slot >> s.page_log2) * s.page_bytes() + (int64_t)head * s.block_bytes();
                if (exists) {
                    *reinterpret_cast<uint32_t*>(block + s.page * (D / 2) + (t >> 2) * (2 * D) + value_place<D>(4 * j + sub) * 4) = word;
                    if ((j & 7) == 0) *reinterpret_cast<uint32_t*>(block + s.page * D + s.page * (NG * 4) + (t * NG + (j >> 3)) * 4) = p.pair;
                }
            }
            if (__any(alone)) {
                const Packed p = pack(lead >= 0 ? load(part, row, alone) : here);
                if (alone && exists) {
                    const int t = slot & (s.page - 1);
                    uint8_t* block = pages + (int64_t)(slot >> s.page_log2) * s.page_bytes() + (int64_t)head * s.block_bytes();
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        block[s.page * (D / 2) + (t >> 2) * (2 * D) + value_place<D>(4 * j + i) * 4 + (t & 3)] = (uint8_t)(p.codes >> (8 * i));
                    if ((j & 7) == 0) *reinterpret_cast<uint32_t*>(block + s.page * D + s.page * (NG * 4) + (t * NG + (j >> 3)) * 4) = p.pair;
                }
            }
        }
    }
}

// A lane has 8 columns of a head; of values it reads the four words that hold its bytes beside those of the neighbouring positions, which as
// a rule other rows of the wave need.
template <int D, int U>                 // heads that a lane has
__global__ __launch_bounds__(WAVES * 64) void paged_read_kernel(PagedShape s, const uint8_t* __restrict__ pages, const int32_t* __restrict__ slots,
                                                                int rows, _Float16* __restrict__ kv, int64_t ld) {
    constexpr int LANES = D / 8, SIDE = 16 / LANES, NG = D / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane >> 4, j = lane & (LANES - 1);
    const int row = blockIdx.x * 4 + sub;
    const int slot = row < rows ? slots[row] : -1;
    if (slot < 0 || slot >= s.n_pages * s.page) return;
    const int t = slot & (s.page - 1);
    const uint8_t* page = pages + (int64_t)(slot >> s.page_log2) * s.page_bytes();
    uint32_t codes[U], pairs[U];
    half8* to[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int h = ((blockIdx.y * WAVES + wave) * U + u) * SIDE + (SIDE > 1 ? (lane >> 3) & 1 : 0);
        to[u] = nullptr;
        if (h >= 2 * s.kv_heads) break;
        const bool is_k = h < s.kv_heads;
        const uint8_t* block = page + (int64_t)(is_k ? h : h - s.kv_heads) * s.block_bytes();
        if (is_k) {
            codes[u] = *reinterpret_cast<const uint32_t*>(block + t * (D / 2) + key_place<D>(4 * j));
        } else {
            // bytes 4 j, 4 j + 1 lie in neighbouring words, and so do 4 j + 2, 4 j + 3
            const uint8_t* words = block + s.page * (D / 2) + (t >> 2) * (2 * D);
            const word2 a = *reinterpret_cast<const word2*>(words + value_place<D>(4 * j) * 4), b = *reinterpret_cast<const word2*>(words + value_place<D>(4 * j + 2) * 4);
            const int by = 8 * (t & 3);
            codes[u] = (a[0] >> by & 255u) | (a[1] >> by & 255u) << 8 | (b[0] >> by & 255u) << 16 | (b[1] >> by & 255u) << 24;
        }
        pairs[u] = *reinterpret_cast<const uint32_t*>(block + s.page * D + (is_k ? 0 : s.page * (NG * 4)) + (t * NG + (j >> 3)) * 4);
        to[u] = reinterpret_cast<half8*>(kv + row * ld + (int64_t)h * D + j * 8);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (!to[u]) break;
        union { uint32_t u; _Float16 h[2]; } pair;
        pair.u = pairs[u];
        half8 out;
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] = (_Float16)((float)(codes[u] >> (4 * i) & 15u) * (float)pair.h[0] + (float)pair.h[1]);
        __builtin_nontemporal_store(out, to[u]);
    }
}

}  // namespace

// Rows of one launch: a dimension of a grid holds less than 2^32 threads, which 2^28 rows of an append and 2^26 of a read would pass (unreported: the read
// left nearly all rows as they were).  A multiple of the rows of a workgroup; a quad of positions that lies across the border is stored byte by byte.
constexpr int MOST_AT_ONCE = 1 << 24;

static int append_rows(const PagedShape& s, const void* qkv, int64_t ld, const int32_t* slots, const int32_t* positions, int rows,
                       const void* rope, int n_pos, void* q_out, int64_t ldq, void* pages, hipStream_t st) {
    const int units = (((q_out ? s.heads : 0) + 2 * s.kv_heads) * s.d + 127) / 128;      // of a wave: one head, two of 64 columns
    const int64_t quads = ((int64_t)rows + 3) / 4;
    // Eight heads a wave, whose slots and angles are then looked up once; one where that would leave the GPU's 1024 SIMDs without two waves each
    const bool many = quads * units >= 8 * 2048;
    auto launch = [&](auto kern, int heads) -> int {
        const dim3 grid((unsigned)((quads + WAVES - 1) / WAVES), (unsigned)((units + heads - 1) / heads));
        hipLaunchKernelGGL(kern, grid, dim3(WAVES * 64), 0, st, s, (const _Float16*)qkv, ld, slots, positions, rows, (const float2*)rope, n_pos,
                           (_Float16*)q_out, ldq, (uint8_t*)pages);
        KVPR_HIP(hipGetLastError());
        return KVPR_OK;
    };
    if (s.d == 128) return many ? launch(paged_append_kernel<128, 8>, 8) : launch(paged_append_kernel<128, 1>, 1);
    return many ? launch(paged_append_kernel<64, 8>, 8) : launch(paged_append_kernel<64, 1>, 1);
}

int launch_paged_append(const PagedShape& s, const void* qkv, int64_t ld, const int32_t* slots, const int32_t* positions, int rows,
                        const void* rope, int n_pos, void* q_out, int64_t ldq, void* pages, hipStream_t st) {
    for (int64_t r = 0; r < rows; r += MOST_AT_ONCE) {
        const int rc = append_rows(s, (const _Float16*)qkv + r * ld, ld, slots + r, positions ? positions + r : nullptr, (int)std::min<int64_t>(rows - r, MOST_AT_ONCE),
                                   rope, n_pos, q_out ? (_Float16*)q_out + r * ldq : nullptr, ldq, pages, st);
        if (rc) return rc;
    }
    return KVPR_OK;
}

static int read_rows(const PagedShape& s, const void* pages, const int32_t* slots, int rows, void* kv, int64_t ld, hipStream_t st) {
    const int units = (2 * s.kv_heads * s.d + 127) / 128;
    const int64_t quads = ((int64_t)rows + 3) / 4;
    const int each = quads * units >= 8 * 2048 ? 4 : 1;      // as above
    const dim3 grid((unsigned)quads, (unsigned)((units + each * WAVES - 1) / (each * WAVES)));
    auto kern = s.d == 128 ? (each == 4 ? paged_read_kernel<128, 4> : paged_read_kernel<128, 1>) : each == 4 ? paged_read_kernel<64, 4> : paged_read_kernel<64, 1>;
    hipLaunchKernelGGL(kern, grid, dim3(WAVES * 64), 0, st, s, (const uint8_t*)pages, slots, rows, (_Float16*)kv, ld);
    KVPR_HIP(hipGetLastError());
    return KVPR_OK;
}

int launch_paged_read(const PagedShape& s, const void* pages, const int32_t* slots, int rows, void* kv, int64_t ld, hipStream_t st) {
    for (int64_t r = 0; r < rows; r += MOST_AT_ONCE)
        if (const int rc = read_rows(s, pages, slots + r, (int)std::min<int64_t>(rows - r, MOST_AT_ONCE), (_Float16*)kv + r * ld, ld, st)) return rc;
    return KVPR_OK;
}

}  // namespace kvpr
