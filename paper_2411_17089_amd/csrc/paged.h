// Pages of the 4-bit cache that ragged batches share: geometry, places inside a page, launchers.
#pragma once
#include "kvpr_internal.h"

namespace kvpr {

// A page holds `page` positions of every key/value head; the block of one head is page * 9 d / 8 bytes:
//   key codes    [page][d / 2]: the row's words of 8 columns, word 4 s + g at place g (d / 32) + s
//   value codes  [page / 4][d / 2][4]: the bytes of four positions side by side, byte 32 u + 2 m + w at place m (d / 32) + 2 u + w
//   key pairs    [page][d / 64] of (scale, minimum), float16; value pairs likewise
// Both orders are those in which lanes of a matrix instruction take their operands, so that 16 bytes of a lane are one load and
// 16 positions of one head are 1 KiB in a row (d = 128): a key lane (position, g) needs the columns 8 (4 s + g) .. + 8 for all s, a
// value lane m needs four positions of columns that it writes next to each other.  One position's bytes are never shared with
// another's, so rows may be appended in any order and from any number of workgroups.
struct PagedShape {
    int heads, kv_heads, d, page, page_log2, n_pages, width;
    __host__ __device__ int64_t block_bytes() const { return (int64_t)page * 9 * d / 8; }
    __host__ __device__ int64_t page_bytes() const { return block_bytes() * kv_heads; }
};

template <int D>
__device__ __forceinline__ int key_place(int k) {              // place of byte k of a row of key codes
    const int j = k >> 2;
    return ((j & 3) * (D / 32) + (j >> 2)) * 4 + (k & 3);
}
template <int D>
__device__ __forceinline__ int value_place(int k) {            // place of byte k of a row of value codes, in units of four positions
    return ((k & 31) >> 1) * (D / 32) + (k >> 5) * 2 + (k & 1);
}

constexpr int kMaxRequests = 8192;

struct PagedPlan {
    const int32_t *base_len, *new_len, *held_in, *count_in;
    int32_t *table, *held_out, *free_pages, *count_out, *row_start, *seq_len, *slots, *positions, *refused;
    int n, max_rows;
};
int launch_paged_plan(const PagedShape& s, const PagedPlan& p, hipStream_t st);
int launch_paged_append(const PagedShape& s, const void* qkv, int64_t ld, const int32_t* slots, const int32_t* positions, int rows,
                        const void* rope, int n_pos, void* q_out, int64_t ldq, void* pages, hipStream_t st);
int launch_paged_read(const PagedShape& s, const void* pages, const int32_t* slots, int rows, void* kv, int64_t ld, hipStream_t st);

struct PagedAttention {
    const void *q, *pages;
    const int32_t *table, *row_start, *seq_len;
    void* z;
    int64_t ldq, ldz;
    int n, rows, max_new, max_len;
    bool q_f32;
};
size_t paged_attention_workspace_bytes(const PagedShape& s, int n, int rows, int max_new, int max_len);
int launch_paged_attention(const PagedShape& s, const PagedAttention& a, void* ws, size_t ws_bytes, hipStream_t st);

struct Verify {
    const void *target, *draft;
    int64_t ld_target, ld_draft;
    const int32_t *tokens, *row_start, *len_in;
    const int32_t *seq_len, *certain;           // null: no request was refused; one certain token each
    const float *temperature, *u_accept, *u_sample;
    int32_t *len_out, *kept, *out;
    int vocab, n, rows;
    bool f16;
};
size_t verify_workspace_bytes(int n, int rows, int vocab);
int launch_verify(const Verify& v, void* ws, hipStream_t st);

}  // namespace kvpr
