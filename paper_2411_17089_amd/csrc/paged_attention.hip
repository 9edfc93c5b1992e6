// Attention of a ragged batch's new tokens over a paged 4-bit cache (formulas at kvpr_paged_attention).
//
// The rows that share a key/value head - the new tokens times the query heads of its group - are the columns of the matrix
// products, 16 a tile: scores^T = K q^T with the positions as rows of K, then z^T = V^T p^T.  A lane then holds four positions'
// scores of one row (D fragment: column = lane & 15, rows 4 (lane >> 4) + 0..3), which are just the k values that it has to bring to the
// second product, so that the weights never leave its registers.  32 positions a turn and wave:
//   - a key lane (position lane & 15, g = lane >> 4) has one 16-byte load (d = 128) with its words of all steps, a value lane one
//     with four positions of the columns that it sums: the order of the bytes in a page is made for this (paged.h);
//   - a key's code as bits 0 - 3 (4 - 7) of a half is the subnormal number code 2^-24 (2^-20), which the matrix instruction takes
//     exactly: unpacking is a mask.  The factor 16 of the odd columns is taken out of q; the affine map is taken out of the
//     sum, k . q = scale (code . q) + minimum sum(q), per group of 64 columns, in float32;
//   - values are unpacked to float16, as kvpr_dequant_int4 gives them: (1024 + code) - 1024 exactly, then one fused
//     multiplication and addition.  That rounding is the library's definition of a stored value (whatever reads the cache sees the same
//     numbers), and the matrix instruction's operand; against values that are not rounded it makes the error 2.8 10^-4 of the result's size where
//     the result's own rounding gives 2.1;
//   - q is scaled by a power of two per row to a largest element of 2^10 .. 2^11; float32 q is brought as the sum of two
//     float16 numbers (the rest below 2^-22 of the largest element);
//   - weights are 2^(score - ref), brought to the product as the sum of two float16 numbers (one alone made the result's error 1.6
//     times that of its own rounding), summed in float32.  ref is the largest score less 6 when it was
//     last set and is set again only when a weight would pass 2^15: no reduction over lanes in the usual turn, and
//     weights keep all bits down to 2^-20 of the largest, some to 2^-30.
// What bounds it: long caches with one row a request the reading (32 x 1000 positions of 32 heads 36 - 39 us, 3.8 - 4.1 TB/s of packed rows); more
// rows a head the vector instructions between the products (unpacking 160 a turn and wave, 100 more for each tile of rows).
// Work: a unit is (request, key/value head, tile of rows).  Few rows: the workgroup's waves share a tile and take turns of 32 positions in
// turn, their sums meet in LDS; many rows: each wave has rows of its own.  The lengths are known on the device only.  Where the
// host's bounds let them differ much, every workgroup adds up the requests' work by itself and takes an equal run of it, whatever units
// that covers; what belongs to a unit of several workgroups meets in the workspace and is joined by a second launch.  (One workgroup
// per unit and chunk of 2048 positions: 64 requests of 1 to 8192 positions 79 us, most of it starts of workgroups with little or
// nothing to do; by runs 52.)  Elsewhere a workgroup has a unit, and there is no second launch.
#include "paged.h"
#include <math.h>
#include <algorithm>

namespace kvpr {
namespace {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t word2 __attribute__((ext_vector_type(2)));
typedef uint32_t word4 __attribute__((ext_vector_type(4)));

constexpr float LOWEST = -0x1p126f;     // where a reference starts: finite, so that no difference of two is NaN
constexpr int TURN = 32;                // positions a wave takes at once

// v of lanes l, l ^ 16, l ^ 32, l ^ 48 reduced; every lane gets the result
template <class F>
__device__ __forceinline__ float across_rows(float v, F f) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float max_of(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float sum_of(float a, float b) { return a + b; }

// what a wave writes to LDS, its lanes read in program order
__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

union Half8 {
    half8 v;
    uint32_t w[4];
    half2v h[4];
};

constexpr int NW = 4;                   // waves of a workgroup

struct AttentionArgs {
    PagedShape s;
    const void* q;
    const uint8_t* pages;
    const int32_t *table, *row_start, *seq_len;
    _Float16* z;
    float* part;                        // partial sums [workgroup][2][slot_rows][d + 2]: the sums, then (reference, sum of weights)
    struct Open* open;                  // [workgroup]
    int64_t ldq, ldz;
    int n, rows, group, slot_rows;
    float scale_log2;
};
// the unit that a workgroup began and left to those behind it, rows row0 .. end - 1 (fewer than slot_rows where the waves share them while
// other requests' units have more); pieces = 0: none
struct Open { int pieces, first, row0, end, kv_head; };
constexpr int FEW = 64;                 // rows up to which a workgroup's waves share them
constexpr int START = 3;                // what a unit costs beside its turns, in turns: lengths, queries, first operands, the join of the waves

// Lengths and page numbers are read through the constant address space, that is by scalar loads: as vector loads each of them waited
// for all operands on their way.  Nothing writes them while the kernel runs.
typedef const __attribute__((address_space(4))) int32_t* ScalarInts;
__device__ __forceinline__ ScalarInts scalar(const int32_t* p) { return (ScalarInts)(uintptr_t)p; }

// one request's work
struct Request {
    int first, m, len, span;
    int real;                           // rows per key/value head that there are
    bool own_rows;                      // each wave has rows of its own
    int tile_rows, step;                // rows of a unit, positions of a turn
    int tiles;
    int turns;                          // of a unit
    int cost;                           // of a unit, in turns: START for its beginning and end, then its turns
    int64_t units, work;
};
template <int MT, bool OWN>
__device__ __forceinline__ Request request(const AttentionArgs& a, int r) {
    Request q;
    q.first = scalar(a.row_start)[r];
    q.m = scalar(a.row_start)[r + 1] - q.first;
    q.len = scalar(a.seq_len)[r];
    q.span = min(max(q.len, 0), a.s.width * a.s.page);
    const int there = q.first < 0 ? 0 : max(min(q.m, a.rows - q.first), 0);
    q.real = there * a.group;
    q.own_rows = OWN && q.real > FEW;
    q.tile_rows = MT * 16 * (q.own_rows ? NW : 1);
    q.step = q.own_rows ? TURN : NW * TURN;
    q.tiles = (int)((unsigned)(q.real + q.tile_rows - 1) / (unsigned)q.tile_rows);
    q.turns = max((q.span + q.step - 1) / q.step, 1);
    q.units = (int64_t)q.tiles * a.s.kv_heads;
    q.cost = q.turns + START;
    q.work = q.units * q.cost;
    return q;
}

// exclusive sum of v over the 256 threads of the workgroup
__device__ __forceinline__ int64_t sum_before(int64_t v, int64_t* lds, int64_t& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t s = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t u = __shfl_up(s, o);
        if (lane >= o) s += u;
    }
    if (lane == 63) lds[wave] = s;
    __syncthreads();
    int64_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        before += w < wave ? lds[w] : 0;
        total += lds[w];
    }
    return before + s - v;
}

// request().work from vector loads
template <int MT, bool OWN>
__device__ __forceinline__ int64_t work_of(const AttentionArgs& a, int r) {
    const int first = a.row_start[r], m = a.row_start[r + 1] - first, span = min(max(a.seq_len[r], 0), a.s.width * a.s.page);
    const int real = (first < 0 ? 0 : max(min(m, a.rows - first), 0)) * a.group;
    const bool own_rows = OWN && real > FEW;
    const int tile_rows = MT * 16 * (own_rows ? NW : 1), step = own_rows ? TURN : NW * TURN;
    return (int64_t)((unsigned)(real + tile_rows - 1) / (unsigned)tile_rows) * a.s.kv_heads * (max((span + step - 1) / step, 1) + START);
}

// workgroup b of `groups` has the turns [total b / groups, total (b + 1) / groups): the one that has turn x
__device__ __forceinline__ int64_t group_of(int64_t x, int64_t groups, int64_t total) { return ((x + 1) * groups - 1) / total; }

// One turn's operands as they are loaded: the codes, and of the (scale, minimum) pairs of the 32 positions' keys and values, 512
// bytes, one lane's share.  The pairs go through LDS, where every lane reads those of its four positions: sixteen lanes
// need the same ones, and loading them so from the pages took 8 of 12 loads and 64 of 96 registers for two turns.
template <int D>
struct Turn {
    static constexpr int NG = D / 64, W = D / 32;
    uint32_t k[2][W], v[2][W], pairs[2];
};
// (scale, minimum) of four positions and NG groups
template <int D>
struct Pairs {
    static constexpr int NG = D / 64;
    word4 w[NG];
    __device__ half2v at(int pos, int gr) const {
        half2v h;
        const uint32_t v = w[(pos * NG + gr) >> 2][(pos * NG + gr) & 3];
        __builtin_memcpy(&h, &v, 4);
        return h;
    }
    __device__ void clear(int pos, int gr) { w[(pos * NG + gr) >> 2][(pos * NG + gr) & 3] = 0u; }
};

template <int D, int MT, bool F32, bool OWN, bool DIRECT>
__global__ __launch_bounds__(NW * 64, MT == 1 ? 3 : 2) void paged_attention_kernel(const AttentionArgs a) {
    constexpr int NG = D / 64, W = D / 32, NT = 2 * W;   // groups, words of codes a lane has per 16 positions, tiles of 16 columns
    __shared__ float part[NW][4][NT][64];
    __shared__ half8 q_lds[OWN ? NW : 1][F32 ? MT : 1][W][64];          // of float32 q, what float16 leaves
    __shared__ uint32_t pair_lds[NW][64 * NG];
    __shared__ float2 ml[NW][16];
    __shared__ int64_t sums[NW], found[2];
    const PagedShape& s = a.s;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m16 = lane & 15, g = lane >> 4;

    // ---- this workgroup's run of work ----
    int64_t total = 0, groups = 0, at = 0, end_of_run = 0, offset = 0, b = 0;       // offset: of `at` within the work of request r
    int r = blockIdx.y;
    if constexpr (!DIRECT) {
        const int64_t groups_max = gridDim.x;
        // consecutive runs to the same XCD (workgroups go round the 8 of them), so that the row tiles of a head meet in one L2
        b = groups_max % 8 ? blockIdx.x : (blockIdx.x & 7) * (groups_max / 8) + (blockIdx.x >> 3);
        const int each = (a.n + NW * 64 - 1) / (NW * 64), r0 = min((int)threadIdx.x * each, a.n), r1 = min(r0 + each, a.n);
        int64_t mine = 0;
        for (int i = r0; i < r1; ++i) mine += work_of<MT, OWN>(a, i);
        int64_t before = sum_before(mine, sums, total);
        groups = min(groups_max, total);
        if (threadIdx.x == 0) a.open[b].pieces = 0;
        if (b >= groups) return;
        at = total * b / groups;
        end_of_run = total * (b + 1) / groups;
        if (at >= before && at < before + mine) {
            for (int i = r0;; ++i) {
                const int64_t w = work_of<MT, OWN>(a, i);
                if (at < before + w) {
                    found[0] = i;
                    found[1] = at - before;
                    break;
                }
                before += w;
            }
        }
        __syncthreads();
        r = __builtin_amdgcn_readfirstlane((int)found[0]);
        offset = (int64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)found[1]) | (int64_t)__builtin_amdgcn_readfirstlane((int)(found[1] >> 32)) << 32;
    }
    const int64_t page_bytes = s.page_bytes();

    Request rq = request<MT, OWN>(a, r);
    if constexpr (DIRECT) {
        offset = blockIdx.x;                                // counts units here
        end_of_run = rq.units;
    }
    while (DIRECT ? offset < end_of_run : at < end_of_run) {
        int64_t unit = offset;
        int turn0 = 0, turn1 = rq.turns;
        if constexpr (DIRECT) {
            offset += gridDim.x;
        } else {
            if (offset >= rq.work) {
                offset -= rq.work;
                rq = request<MT, OWN>(a, ++r);
                continue;
            }
            unit = offset / rq.cost;
            const int from = (int)(offset - unit * rq.cost), to = (int)min((int64_t)rq.cost, from + (end_of_run - at));
            at += to - from;
            offset += to - from;
            turn0 = max(from - START, 0);
            turn1 = to - START;
            if (turn1 <= turn0) continue;                   // the beginning of a unit whose turns are the next workgroup's
        }
        const int kv_head = (int)(unit / rq.tiles);
        const int row0 = (int)(unit - (int64_t)kv_head * rq.tiles) * rq.tile_rows;
        const bool own_rows = OWN && rq.own_rows;
        const int c0 = turn0 * rq.step, c1 = min(rq.span, turn1 * rq.step);
        const ScalarInts ids = scalar(a.table) + (int64_t)r * s.width;
        const uint8_t* head_base = a.pages + (int64_t)kv_head * s.block_bytes();
        const int region = own_rows ? wave : 0, wave_row0 = row0 + region * (MT * 16), live_rows = min(rq.real - wave_row0, MT * 16);
        // positions that every / any row of the wave sees: those of its first and its last row
        const int see0 = rq.len - rq.m + 1, all_see = min(rq.span, see0 + wave_row0 / a.group),
                  any_see = live_rows > 0 ? min(rq.span, see0 + (wave_row0 + live_rows - 1) / a.group) : 0;
        const int end = min(c1, any_see), step = rq.step;
        int t0 = c0 + (own_rows ? 0 : wave * TURN);

        const int k_lane = m16 * (D / 2) + g * (D / 8), v_lane = s.page * (D / 2) + g * (2 * D) + m16 * (D / 8),
                  p_lane = s.page * D + (NG == 2 ? (lane & 32 ? s.page * 8 : 0) + (lane & 31) * 4 : (lane & 16 ? s.page * 4 : 0) + m16 * 4);
        auto id_of = [&](int t) { return ids[min(t, end - 1) >> s.page_log2]; };     // those behind the end are not used
        auto load = [&](Turn<D>& x, int t0, const int (&id)[2]) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                // a half of a turn that lies outside the pool reads its first page and is masked; one behind the end reads what is there
                const int tp = (t0 + 16 * u) & (s.page - 1);
                const uint8_t* b = head_base + (int64_t)((unsigned)id[u] < (unsigned)s.n_pages ? id[u] : 0) * page_bytes;
                const __amdgpu_buffer_rsrc_t block = __builtin_amdgcn_make_buffer_rsrc((void*)b, 0, (int)s.block_bytes(), 0x00027000);
                if constexpr (D == 128) {
                    const word4 kw = __builtin_amdgcn_raw_buffer_load_b128(block, k_lane, tp * (D / 2), 0),
                                vw = __builtin_amdgcn_raw_buffer_load_b128(block, v_lane, tp * (D / 2), 0);
#pragma unroll
                    for (int i = 0; i < W; ++i) { x.k[u][i] = kw[i]; x.v[u][i] = vw[i]; }
                } else {
                    const word2 kw = __builtin_amdgcn_raw_buffer_load_b64(block, k_lane, tp * (D / 2), 0),
                                vw = __builtin_amdgcn_raw_buffer_load_b64(block, v_lane, tp * (D / 2), 0);
#pragma unroll
                    for (int i = 0; i < W; ++i) { x.k[u][i] = kw[i]; x.v[u][i] = vw[i]; }
                }
                x.pairs[u] = __builtin_amdgcn_raw_buffer_load_b32(block, p_lane, tp * (NG * 4), 0);
            }
        };
        // two turns' operands in registers: one at work, one on its way; page numbers one turn further ahead
        Turn<D> xa, xb;
        int ia[2], ib[2];
        const bool any_turn = t0 < end;
        if (any_turn) {
            ia[0] = id_of(t0); ia[1] = id_of(t0 + 16); ib[0] = id_of(t0 + step); ib[1] = id_of(t0 + step + 16);
            load(xa, t0, ia);
        }
        // ---- rows: where they are, how far they see, q ----
        // row, head and whether there is one; worked out again at the end rather than kept
        auto place = [&](int mt, int& token, int& head) {
            const int rr = wave_row0 + mt * 16 + m16, there = min(rr, rq.real - 1), i = there / a.group;
            token = rq.first + i;
            head = kv_head * a.group + there - i * a.group;
            return rr < rq.real;
        };
        int seen[MT];
        bool real[MT];
        Half8 q[MT][W];
        float qs[MT][NG], score_unit[MT], to_log2[MT];      // unit of the scores, and that of the weights: smaller where scores are very large
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            int token, head;
            real[mt] = place(mt, token, head);
            seen[mt] = real[mt] ? min(rq.span, see0 + token - rq.first) : 0;
            const int64_t at = real[mt] ? token * a.ldq + (int64_t)head * D : 0;
            float x[W][8], big = 0.f;
#pragma unroll
            for (int st = 0; st < W; ++st) {
                const int col = (st * 4 + g) * 8;
                if constexpr (F32) {
                    const float4v* p = reinterpret_cast<const float4v*>((const float*)a.q + at + col);
                    const float4v u = p[0], w = p[1];
#pragma unroll
                    for (int e = 0; e < 4; ++e) { x[st][e] = u[e]; x[st][4 + e] = w[e]; }
                } else {
                    const half8 u = *reinterpret_cast<const half8*>((const _Float16*)a.q + at + col);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[st][e] = (float)u[e];
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) big = fmaxf(big, fabsf(x[st][e]));
            }
            big = across_rows(big, max_of);
            // exponent of the largest element (of 0 whatever); infinite and NaN rows become NaN
            const int ex = max((int)(__float_as_uint(big) >> 23) - 127, -100);
            const float up = __uint_as_float((uint32_t)(127 + 10 - ex) << 23);
            // beyond 2^85 the unit stays, so that no score overflows: any two that float32 tells apart are 2^30 and more apart there anyway
            score_unit[mt] = to_log2[mt] = a.scale_log2 * __uint_as_float((uint32_t)(127 + 24 - 10 + min(ex, 85)) << 23);
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) {
                float t = 0.f;
#pragma unroll
                for (int st = 2 * gr; st < 2 * gr + 2; ++st)
#pragma unroll
                    for (int e = 0; e < 8; ++e) t += x[st][e] * up;
                qs[mt][gr] = across_rows(t, sum_of) * 0x1p-24f;
            }
#pragma unroll
            for (int st = 0; st < W; ++st) {
                constexpr int order[8] = {0, 4, 1, 5, 2, 6, 3, 7};      // columns as the masks below leave them
                Half8 rest;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float y = x[st][order[e]] * up * ((e & 2) ? 0.0625f : 1.f);
                    const _Float16 hi = (_Float16)y;
                    q[mt][st].v[e] = hi;
                    if constexpr (F32) rest.v[e] = (_Float16)(y - (float)hi);
                }
                // the waves that share rows write the same
                if constexpr (F32) q_lds[region][mt][st][lane] = rest.v;
            }
        }

        float ref[MT], off[MT], l[MT];                      // off: the score that ref was set from
        float4v acc[MT][NT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            ref[mt] = off[mt] = LOWEST;
            l[mt] = 0.f;
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[mt][t] = float4v{0.f, 0.f, 0.f, 0.f};
        }

        // in a register, so that masking and setting the upper bits are one instruction (with two literals they are two)
        uint32_t magic = 0x64006400u;
        asm("" : "+v"(magic));
        auto compute = [&](const Turn<D>& x, int t0, const int (&id)[2]) __attribute__((always_inline)) {
            const bool masked = t0 + TURN > min(all_see, c1) || (unsigned)id[0] >= (unsigned)s.n_pages || (unsigned)id[1] >= (unsigned)s.n_pages;
            uint32_t* mine = pair_lds[wave];
#pragma unroll
            for (int u = 0; u < 2; ++u) mine[u * 32 * NG + (NG == 2 ? lane : lane & 31)] = x.pairs[u];
            wave_fence();
            auto pairs_of = [&](int u, int values) {
                Pairs<D> r;
                const word4* from = reinterpret_cast<const word4*>(mine + ((u * 2 + values) * 16 + g * 4) * NG);
#pragma unroll
                for (int i = 0; i < NG; ++i) r.w[i] = from[i];
                return r;
            };
            // ---- scores, in units of 2^to_log2 ----
            float sc[MT][2][4];
            float4v c[2][MT][NG];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int gr = 0; gr < NG; ++gr) c[u][mt][gr] = float4v{0.f, 0.f, 0.f, 0.f};
            auto score = [&](int u, int st, const half8 (&ql)[MT]) {
                Half8 kf;
                const uint32_t w = x.k[u][st], w8 = w >> 8;
                kf.w[0] = w & 0x000F000Fu; kf.w[1] = w & 0x00F000F0u; kf.w[2] = w8 & 0x000F000Fu; kf.w[3] = w8 & 0x00F000F0u;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    c[u][mt][st / 2] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf.v, q[mt][st].v, c[u][mt][st / 2], 0, 0, 0);
                    if constexpr (F32) c[u][mt][st / 2] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf.v, ql[mt], c[u][mt][st / 2], 0, 0, 0);
                }
            };
            half8 ql[MT];
            if constexpr (F32) {
                // both halves of the turn with one read of a step's rest
#pragma unroll
                for (int st = 0; st < W; ++st) {
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) ql[mt] = q_lds[region][mt][st][lane];
                    score(0, st, ql);
                    score(1, st, ql);
                }
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if constexpr (!F32)
#pragma unroll
                    for (int st = 0; st < W; ++st) score(u, st, ql);
                const Pairs<D> km = pairs_of(u, 0);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        float t = 0.f;
#pragma unroll
                        for (int gr = 0; gr < NG; ++gr) {
                            const half2v sm = km.at(p, gr);
                            t = fmaf((float)sm[0], c[u][mt][gr][p], fmaf((float)sm[1], qs[mt][gr], t));
                        }
                        sc[mt][u][p] = t;
                    }
            }
            Pairs<D> vm[2] = {pairs_of(0, 1), pairs_of(1, 1)};
            wave_fence();
            if (masked) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int all = (unsigned)id[u] < (unsigned)s.n_pages ? end : 0;
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        const int t = t0 + 16 * u + 4 * g + p;
                        float poison = 0.f;                             // NaN for values that are not finite, or whose largest passes float16 where not all rows see it
#pragma unroll
                        for (int gr = 0; gr < NG; ++gr) {
                            const half2v sm = vm[u].at(p, gr);
                            poison += (float)sm[0] * 0.f + (float)sm[1] * 0.f;
                            if (t >= all_see) poison += (float)(_Float16)fmaf((float)sm[0], 15.f, (float)sm[1]) * 0.f;
                        }
                        // positions that a row does not see must not reach its sum, not even as 0 times NaN
                        const bool out = t >= all || poison != 0.f;
#pragma unroll
                        for (int gr = 0; gr < NG; ++gr)
                            if (out) vm[u].clear(p, gr);
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            const bool sees = t < min(all, seen[mt]);
                            if (!sees) sc[mt][u][p] = -INFINITY;
                            l[mt] += sees ? poison : 0.f;              // the row is NaN
                        }
                    }
                }
            }
            // ---- weights, as the sum of two float16 numbers ----
            Half8 pw[MT], pl[MT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                float top = sc[mt][0][0];
#pragma unroll
                for (int j = 1; j < 8; ++j) top = fmaxf(top, sc[mt][j >> 2][j & 3]);
                if (__any(fmaf(top, to_log2[mt], -ref[mt]) > 15.f)) {
                    // Weights are exact to ref as it is rounded, which beyond 2^27 would carry them out of float16.  Scores of 2^26 and more are
                    // known to no better than 16 anyway, so their row's differences are counted in units of a power of two that brings them to 2^25 .. 2^26
                    const float was = off[mt];
                    off[mt] = fmaxf(was, across_rows(top, max_of));
                    const int over = max((int)(__float_as_uint(fabsf(off[mt] * score_unit[mt])) >> 23) - (127 + 25), 0);
                    const bool fine = over == 0 && to_log2[mt] == score_unit[mt];
                    to_log2[mt] = score_unit[mt] * __uint_as_float((uint32_t)(127 - over) << 23);
                    const float now = off[mt] == LOWEST ? LOWEST : off[mt] * to_log2[mt] - 6.f;
                    const float keep = exp2f(fine ? ref[mt] - now : (was - off[mt]) * score_unit[mt]);
                    ref[mt] = now;
                    l[mt] *= keep;
#pragma unroll
                    for (int t = 0; t < NT; ++t) acc[mt][t] *= keep;
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    float p[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        p[j] = __builtin_amdgcn_exp2f(fmaf(sc[mt][u][j], to_log2[mt], -ref[mt]));
                        l[mt] += p[j];
                    }
                    // order of the positions as the masks below leave them
#pragma unroll
                    for (int o = 0; o < 2; ++o) {
                        const half2v hi = __builtin_convertvector((float2v{p[o], p[o + 2]}), half2v);
                        pw[mt].h[2 * u + o] = hi;
                        pl[mt].h[2 * u + o] = __builtin_convertvector((float2v{fmaf((float)hi[0], -1.f, p[o]), fmaf((float)hi[1], -1.f, p[o + 2])}), half2v);
                    }
                }
            }
            // ---- values ----
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) {
                half2v sc2[2][2], mn2[2][2];                            // [half of the turn][positions 0, 2 | 1, 3]
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int o = 0; o < 2; ++o) {
                        const half2v lo = vm[u].at(o, gr), hi = vm[u].at(o + 2, gr);
                        sc2[u][o] = half2v{lo[0], hi[0]};
                        mn2[u][o] = half2v{lo[1], hi[1]};
                    }
#pragma unroll
                for (int i = 2 * gr; i < 2 * gr + 2; ++i)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        Half8 vf;
#pragma unroll
                        for (int u = 0; u < 2; ++u)
#pragma unroll
                            for (int o = 0; o < 2; ++o) {
                                // 1024 + code, or 1024 + 16 code where the code stays in the upper bits: both come out exactly
                                const uint32_t biased = (x.v[u][i] >> (8 * o) & (h ? 0x00F000F0u : 0x000F000Fu)) | magic;
                                half2v c;
                                __builtin_memcpy(&c, &biased, 4);
                                c = h ? __builtin_elementwise_fma(c, half2v{(_Float16)0.0625f, (_Float16)0.0625f}, half2v{(_Float16)-64.f, (_Float16)-64.f})
                                      : c - half2v{(_Float16)1024.f, (_Float16)1024.f};
                                vf.h[2 * u + o] = __builtin_elementwise_fma(c, sc2[u][o], mn2[u][o]);
                            }
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            acc[mt][2 * i + h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf.v, pw[mt].v, acc[mt][2 * i + h], 0, 0, 0);
                            acc[mt][2 * i + h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf.v, pl[mt].v, acc[mt][2 * i + h], 0, 0, 0);
                        }
                    }
            }
        };

        if (any_turn) {
            // loads behind the end (of pages that are there: id_of stays below it) keep the number of loads on their way the same on every path,
            // so that a turn waits for its own only
            while (true) {
                load(xb, t0 + step, ib);
                const int ic[2] = {id_of(t0 + 2 * step), id_of(t0 + 2 * step + 16)};
                compute(xa, t0, ia);
                t0 += step;
                if (t0 >= end) break;
                load(xa, t0 + step, ic);
                const int id[2] = {id_of(t0 + 2 * step), id_of(t0 + 2 * step + 16)};
                compute(xb, t0, ib);
                t0 += step;
                if (t0 >= end) break;
                ia[0] = ic[0]; ia[1] = ic[1];
                ib[0] = id[0]; ib[1] = id[1];
            }
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) l[mt] = across_rows(l[mt], sum_of);
        const bool all_here = DIRECT || (turn0 == 0 && turn1 == rq.turns);
        if (!all_here && turn0 == 0 && threadIdx.x == 0)    // the rest of the turns end in the workgroup that has the last of them
            a.open[b] = Open{(int)(group_of(at + (rq.turns - turn1) - 1, groups, total) - b) + 1, rq.first, row0, min(rq.real, row0 + rq.tile_rows), kv_head};
        float* slot = a.part + ((b * 2 + (turn0 == 0)) * a.slot_rows + region * (MT * 16)) * (D + 2);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            if (mt * 16 >= live_rows) break;
            int token, head;
            const bool real = place(mt, token, head);
            float lsum = l[mt], top = to_log2[mt] == score_unit[mt] || off[mt] == LOWEST ? ref[mt] : off[mt] * score_unit[mt] - 6.f;
            // columns 64 gr + 16 g + 4 p .. + 3 of one row from acc over (w, h)
            auto put = [&](int p, int gr, const float (&what)[4]) {
                if (!real) return;
                const int col = 64 * gr + (4 * g + p) * 4;
                if (all_here) {
                    const float inv = 1.f / lsum;
                    half4 out;
#pragma unroll
                    for (int e = 0; e < 4; ++e) out[e] = (_Float16)(lsum == 0.f ? 0.f : what[e] * inv);
                    *reinterpret_cast<half4*>(a.z + token * a.ldz + (int64_t)head * D + col) = out;
                } else {
                    float* to = slot + (mt * 16 + m16) * (D + 2);
                    *reinterpret_cast<float2*>(to + col) = make_float2(what[0], what[1]);
                    *reinterpret_cast<float2*>(to + col + 2) = make_float2(what[2], what[3]);
                    if (col == 0) *reinterpret_cast<float2*>(to + D) = make_float2(top, lsum);
                }
            };
            if (own_rows) {
#pragma unroll
                for (int p = 0; p < 4; ++p)
#pragma unroll
                    for (int gr = 0; gr < NG; ++gr) {
                        const float what[4] = {acc[mt][4 * gr][p], acc[mt][4 * gr + 1][p], acc[mt][4 * gr + 2][p], acc[mt][4 * gr + 3][p]};
                        put(p, gr, what);
                    }
            } else {
                // the waves' sums meet in LDS, a tile of rows at a time; wave w then has the columns of p = w
                if (mt) __syncthreads();
                if (g == 0) ml[wave][m16] = make_float2(top, lsum);
                __syncthreads();
                float all_top = LOWEST;
                lsum = 0.f;
#pragma unroll
                for (int w = 0; w < NW; ++w) all_top = fmaxf(all_top, ml[w][m16].x);
#pragma unroll
                for (int w = 0; w < NW; ++w) lsum += ml[w][m16].y * exp2f(ml[w][m16].x - all_top);
                const float mine = exp2f(top - all_top);
                top = all_top;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int p = 0; p < 4; ++p) part[wave][p][t][lane] = acc[mt][t][p] * mine;
                __syncthreads();
#pragma unroll
                for (int gr = 0; gr < NG; ++gr) {
                    float what[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int w = 0; w < NW; ++w)
#pragma unroll
                        for (int e = 0; e < 4; ++e) what[e] += part[w][wave][4 * gr + e][lane];
                    put(wave, gr, what);
                }
            }
        }
        __syncthreads();
    }
}

// Joins the units of several workgroups: a wave has one row of the unit that workgroup x of the first launch left open, and asks for 16 of
// its pieces at once, since what counts is the wait for them: 8 us for 64 units of 8 to 16 pieces and for 500 of 2 (four rows a wave
// and four pieces at once 14 and 8, workgroups of 16 waves 11 and 11).
template <int D>
__global__ __launch_bounds__(NW * 64) void paged_attention_join(const AttentionArgs a) {
    constexpr int E = D / 64, U = 16;
    const int lane = threadIdx.x & 63, row = blockIdx.y * NW + (threadIdx.x >> 6);
    const Open o = a.open[blockIdx.x];
    const int rr = o.row0 + row;
    if (o.pieces == 0 || rr >= o.end) return;
    const int64_t stride = 2 * (int64_t)a.slot_rows * (D + 2);
    const float* from = a.part + blockIdx.x * stride + (int64_t)row * (D + 2);          // slot 1 of the first, slot 0 of those behind it
    float top = LOWEST, l = 0.f, sum[E] = {};
    for (int c0 = 0; c0 < o.pieces; c0 += U) {
        float2 ml[U];
        float x[U][E];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = min(c0 + u, o.pieces - 1);
            const float* p = from + c * stride + (c == 0 ? (int64_t)a.slot_rows * (D + 2) : 0);
            ml[u] = *reinterpret_cast<const float2*>(p + D);
            __builtin_memcpy(x[u], p + lane * E, 4 * E);
        }
        float now = top;
#pragma unroll
        for (int u = 0; u < U; ++u) now = fmaxf(now, ml[u].x);
        const float keep = exp2f(top - now);
        top = now;
        l *= keep;
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] *= keep;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float w = c0 + u < o.pieces ? exp2f(ml[u].x - top) : 0.f;
            l = fmaf(ml[u].y, w, l);
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e] = fmaf(x[u][e], w, sum[e]);
        }
    }
    const int64_t token = o.first + rr / a.group, head = o.kv_head * a.group + rr % a.group;
    _Float16* z = a.z + token * a.ldz + head * D + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) z[e] = (_Float16)(l == 0.f ? 0.f : sum[e] / l);
}

// how a launch is cut, from what the host knows
struct Cut {
    int mt;                             // tiles of 16 rows a wave
    bool many_rows, direct;
    int groups, slot_rows;
};

Cut cut_of(const PagedShape& s, int n, int rows, int max_new, int max_len) {
    Cut c;
    const int64_t r = (int64_t)std::min(max_new, std::max(rows, 1)) * (s.heads / s.kv_heads);
    c.mt = r <= 16 ? 1 : 2;
    c.many_rows = r > FEW;
    c.slot_rows = c.mt * 16 * (c.many_rows ? NW : 1);
    const int resident = 256 * (c.mt == 1 ? 3 : 2);                        // workgroups that the GPU holds at once
    const int64_t units = s.kv_heads * ((r + c.slot_rows - 1) / c.slot_rows), all = units * std::min<int64_t>(n, std::max(rows, 1));
    const int64_t len = std::min<int64_t>(max_len, (int64_t)s.width * s.page), step = c.many_rows ? TURN : NW * TURN;
    // A unit each for a workgroup, or equal runs of the work: runs cost a second launch and the sums in front of the first, 9 us in all, and
    // units that differ in length keep the GPU waiting for the longest.  us by units / by runs: 32 x 1000 positions, 32 heads 36 / 45; 64 x 1 to
    // 8192, 8 heads 104 / 52; 4 x 25000, 8 heads 276 / 64; two chunks of 1000 rows 215 / 270.  So units where they fill half of the GPU and none
    // is longer than 16 turns, or where their rows are many, and where a unit has one turn.  The borders lie between these four.  max_new does not tell
    // two chunks from one chunk beside many single rows, which are units too and then unequal ones: 2 chunks of 1000 and 30 rows over 20000 to 32000
    // positions 960, where the chunks alone take 235 and the rows alone 179; with max_new given as 1, by runs of 16 rows, 480.
    c.direct = len <= step || (c.many_rows ? all >= resident / 2 : all >= resident / 2 && len <= 2048);
    if (c.direct) {
        c.groups = (int)std::min<int64_t>(units, 1 << 16);
    } else {
        c.groups = (int)std::min<int64_t>(resident, all * ((len + step - 1) / step));
        if (c.groups > 8) c.groups = (c.groups + 7) / 8 * 8;
    }
    return c;
}

}  // namespace

size_t paged_attention_workspace_bytes(const PagedShape& s, int n, int rows, int max_new, int max_len) {
    const Cut c = cut_of(s, n, rows, max_new, max_len);
    return c.direct ? 16 : (size_t)c.groups * (2 * (size_t)c.slot_rows * (s.d + 2) * 4 + sizeof(Open));
}

int launch_paged_attention(const PagedShape& s, const PagedAttention& x, void* ws, size_t, hipStream_t st) {
    const Cut c = cut_of(s, x.n, x.rows, x.max_new, x.max_len);
    AttentionArgs a;
    a.s = s;
    a.q = x.q;
    a.pages = (const uint8_t*)x.pages;
    a.table = x.table; a.row_start = x.row_start; a.seq_len = x.seq_len;
    a.z = (_Float16*)x.z;
    a.part = (float*)ws;
    a.open = (Open*)(a.part + (size_t)c.groups * 2 * c.slot_rows * (s.d + 2));
    a.ldq = x.ldq; a.ldz = x.ldz;
    a.n = x.n; a.rows = x.rows; a.group = s.heads / s.kv_heads; a.slot_rows = c.slot_rows;
    a.scale_log2 = (float)(1.4426950408889634 / sqrt((double)s.d));
    const dim3 grid((unsigned)c.groups, c.direct ? (unsigned)x.n : 1), joined((unsigned)c.groups, (unsigned)(c.slot_rows / NW));
    auto launch = [&](auto kern) -> int {
        hipLaunchKernelGGL(kern, grid, dim3(NW * 64), 0, st, a);
        KVPR_HIP(hipGetLastError());
        if (c.direct) return KVPR_OK;
        if (s.d == 128) hipLaunchKernelGGL(paged_attention_join<128>, joined, dim3(NW * 64), 0, st, a);
        else hipLaunchKernelGGL(paged_attention_join<64>, joined, dim3(NW * 64), 0, st, a);
        KVPR_HIP(hipGetLastError());
        return KVPR_OK;
    };
#define KVPR_CASE(D_, F32_, MT_, OWN_) \
    if (s.d == D_ && x.q_f32 == F32_ && c.mt == MT_ && c.many_rows == OWN_)                                                                        \
        return launch(c.direct ? paged_attention_kernel<D_, MT_, F32_, OWN_, true> : paged_attention_kernel<D_, MT_, F32_, OWN_, false>)
#define KVPR_CASES(D_, F32_)                                                                    \
    KVPR_CASE(D_, F32_, 1, false); KVPR_CASE(D_, F32_, 2, false); KVPR_CASE(D_, F32_, 2, true)
    KVPR_CASES(64, false);
    KVPR_CASES(64, true);
    KVPR_CASES(128, false);
    KVPR_CASES(128, true);
#undef KVPR_CASES
#undef KVPR_CASE
    return fail(KVPR_E_STATE, "no kernel for %d tiles", c.mt);
}

}  // namespace kvpr
