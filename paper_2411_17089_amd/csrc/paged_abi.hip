// C entry points for ragged batches over a paged 4-bit cache: argument validation, then the launcher.
#include "paged.h"

using kvpr::fail;

namespace {

constexpr int MOST_ROWS = 1 << 30;      // row numbers and what is added to them stay in 32 bits

int log2_of(int v) {
    int l = 0;
    while ((1 << l) < v) ++l;
    return l;
}

int check_shape(const kvpr_paged_desc* d, kvpr::PagedShape& s) {
    if (!d) return fail(KVPR_E_INVAL, "desc is null");
    if (d->head_dim != 64 && d->head_dim != 128) return fail(KVPR_E_INVAL, "head_dim must be 64 or 128");
    if (d->n_heads < 1 || d->n_kv_heads < 1 || d->n_heads > 16384) return fail(KVPR_E_RANGE, "n_heads=%d n_kv_heads=%d out of range", d->n_heads, d->n_kv_heads);
    if (d->n_heads % d->n_kv_heads) return fail(KVPR_E_INVAL, "n_kv_heads=%d does not divide n_heads=%d", d->n_kv_heads, d->n_heads);
    if (d->page_size < 16 || d->page_size > 256 || (d->page_size & (d->page_size - 1)))
        return fail(KVPR_E_INVAL, "page_size=%d must be 16, 32, 64, 128 or 256", d->page_size);
    if (d->n_pages < 1 || (int64_t)d->n_pages * d->page_size > 0x7fffffff) return fail(KVPR_E_RANGE, "n_pages=%d out of range (slots are 32-bit)", d->n_pages);
    if (d->table_width < 1 || (int64_t)d->table_width * d->page_size > (1 << 30)) return fail(KVPR_E_RANGE, "table_width=%d out of range", d->table_width);
    s = kvpr::PagedShape{d->n_heads, d->n_kv_heads, d->head_dim, d->page_size, log2_of(d->page_size), d->n_pages, d->table_width};
    return KVPR_OK;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace

extern "C" size_t kvpr_page_bytes(const kvpr_paged_desc* desc) {
    kvpr::PagedShape s;
    return check_shape(desc, s) ? 0 : (size_t)s.page_bytes();
}

extern "C" int kvpr_paged_plan(const kvpr_paged_desc* desc, const int32_t* base_len, const int32_t* new_len, int n_requests, int32_t* block_table,
                               const int32_t* held_in, int32_t* held_out, int32_t* free_pages, const int32_t* free_count_in, int32_t* free_count_out,
                               int max_rows, int32_t* row_start, int32_t* seq_len, int32_t* slots, int32_t* positions, int32_t* refused, void* stream) {
    kvpr::PagedShape s;
    if (int rc = check_shape(desc, s)) return rc;
    if (n_requests < 1 || n_requests > kvpr::kMaxRequests || max_rows < 0 || max_rows > MOST_ROWS)
        return fail(KVPR_E_RANGE, "n_requests=%d (1 to %d) max_rows=%d (0 to 2^30) out of range", n_requests, kvpr::kMaxRequests, max_rows);
    if (!base_len || !new_len || !block_table || !held_in || !held_out || !free_pages || !free_count_in || !free_count_out || !row_start || !seq_len || !refused)
        return fail(KVPR_E_INVAL, "null pointer");
    if (max_rows > 0 && (!slots || !positions)) return fail(KVPR_E_INVAL, "slots / positions is null");
    const kvpr::PagedPlan p{base_len, new_len, held_in, free_count_in, block_table, held_out, free_pages, free_count_out, row_start, seq_len, slots, positions,
                            refused, n_requests, max_rows};
    return kvpr::launch_paged_plan(s, p, (hipStream_t)stream);
}

extern "C" int kvpr_paged_append(const kvpr_paged_desc* desc, const void* qkv, int64_t ld, const int32_t* slots, const int32_t* positions, int n_rows,
                                 const void* rope_table, int n_pos, void* q_out, int64_t ldq, void* pages, void* stream) {
    kvpr::PagedShape s;
    if (int rc = check_shape(desc, s)) return rc;
    if (n_rows < 0 || n_rows > MOST_ROWS) return fail(KVPR_E_RANGE, "n_rows=%d (0 to 2^30) out of range", n_rows);
    const int64_t q_cols = (int64_t)s.heads * s.d, cols = q_cols + 2 * (int64_t)s.kv_heads * s.d;
    if (ld < cols || ld % 8) return fail(KVPR_E_INVAL, "need ld >= %lld, ld %% 8 == 0 (16-byte row pieces)", (long long)cols);
    if (rope_table && n_pos < 1) return fail(KVPR_E_RANGE, "n_pos=%d out of range", n_pos);
    if (!rope_table && q_out) return fail(KVPR_E_INVAL, "q_out without a rope table: q stays as it is");
    if (q_out && (ldq < q_cols || ldq % 8)) return fail(KVPR_E_INVAL, "need ldq >= %lld, ldq %% 8 == 0", (long long)q_cols);
    if (n_rows == 0) return KVPR_OK;
    if (!qkv || !slots || !pages || (rope_table && !positions)) return fail(KVPR_E_INVAL, "qkv / slots / positions / pages is null");
    if (!aligned16(qkv) || !aligned16(q_out) || !aligned16(pages) || ((uintptr_t)rope_table & 7)) return fail(KVPR_E_INVAL, "qkv, q_out and pages must be 16-byte aligned");
    return kvpr::launch_paged_append(s, qkv, ld, slots, positions, n_rows, rope_table, n_pos, q_out, ldq, pages, (hipStream_t)stream);
}

extern "C" int kvpr_paged_read(const kvpr_paged_desc* desc, const void* pages, const int32_t* slots, int n_rows, void* kv, int64_t ld, void* stream) {
    kvpr::PagedShape s;
    if (int rc = check_shape(desc, s)) return rc;
    if (n_rows < 0 || n_rows > MOST_ROWS) return fail(KVPR_E_RANGE, "n_rows=%d (0 to 2^30) out of range", n_rows);
    const int64_t cols = 2 * (int64_t)s.kv_heads * s.d;
    if (ld < cols || ld % 8) return fail(KVPR_E_INVAL, "need ld >= %lld, ld %% 8 == 0 (16-byte row pieces)", (long long)cols);
    if (n_rows == 0) return KVPR_OK;
    if (!pages || !slots || !kv) return fail(KVPR_E_INVAL, "pages / slots / kv is null");
    if (!aligned16(pages) || !aligned16(kv)) return fail(KVPR_E_INVAL, "pages and kv must be 16-byte aligned");
    return kvpr::launch_paged_read(s, pages, slots, n_rows, kv, ld, (hipStream_t)stream);
}

static int check_batch(int n_requests, int n_rows, int max_new, int max_len) {
    if (n_requests < 1 || n_requests > kvpr::kMaxRequests || n_rows < 0 || max_new < 1 || max_len < 1)
        return fail(KVPR_E_RANGE, "n_requests=%d (1 to %d) n_rows=%d max_new=%d max_len=%d out of range", n_requests, kvpr::kMaxRequests, n_rows, max_new, max_len);
    return KVPR_OK;
}

extern "C" size_t kvpr_paged_attention_workspace_bytes(const kvpr_paged_desc* desc, int n_requests, int n_rows, int max_new, int max_len) {
    kvpr::PagedShape s;
    if (check_shape(desc, s) || check_batch(n_requests, n_rows, max_new, max_len)) return 0;
    return kvpr::paged_attention_workspace_bytes(s, n_requests, n_rows, max_new, max_len);
}

extern "C" int kvpr_paged_attention(const kvpr_paged_desc* desc, const void* q, int q_type, int64_t ldq, const void* pages, const int32_t* block_table,
                                    const int32_t* row_start, const int32_t* seq_len, int n_requests, int n_rows, int max_new, int max_len, void* z,
                                    int64_t ldz, void* ws, size_t ws_bytes, void* stream) {
    kvpr::PagedShape s;
    if (int rc = check_shape(desc, s)) return rc;
    if (int rc = check_batch(n_requests, n_rows, max_new, max_len)) return rc;
    if (q_type != KVPR_F16 && q_type != KVPR_F32) return fail(KVPR_E_INVAL, "q_type must be KVPR_F16 or KVPR_F32");
    if ((int64_t)n_rows * (s.heads / s.kv_heads) > MOST_ROWS) return fail(KVPR_E_RANGE, "n_rows=%d times %d heads per key/value head is beyond 2^30", n_rows, s.heads / s.kv_heads);
    const int64_t cols = (int64_t)s.heads * s.d;
    if (ldq < cols || ldq % 8 || ldz < cols || ldz % 8) return fail(KVPR_E_INVAL, "need ldq, ldz >= %lld and multiples of 8", (long long)cols);
    if (n_rows == 0) return KVPR_OK;
    if (!q || !pages || !block_table || !row_start || !seq_len || !z) return fail(KVPR_E_INVAL, "q / pages / block_table / row_start / seq_len / z is null");
    if (!aligned16(q) || !aligned16(pages) || !aligned16(z) || !aligned16(ws)) return fail(KVPR_E_INVAL, "q, pages, z and ws must be 16-byte aligned");
    const size_t need = kvpr::paged_attention_workspace_bytes(s, n_requests, n_rows, max_new, max_len);
    if (!ws || ws_bytes < need) return fail(KVPR_E_INVAL, "the workspace must hold %zu bytes", need);
    const kvpr::PagedAttention a{q, pages, block_table, row_start, seq_len, z, ldq, ldz, n_requests, n_rows, max_new, max_len, q_type == KVPR_F32};
    return kvpr::launch_paged_attention(s, a, ws, ws_bytes, (hipStream_t)stream);
}

static int check_verify(int n_requests, int n_rows, int vocab) {
    if (n_requests < 1 || n_requests > kvpr::kMaxRequests || n_rows < 0 || vocab < 1 || vocab > (1 << 24))
        return fail(KVPR_E_RANGE, "n_requests=%d (1 to %d) n_rows=%d vocab=%d (1 to 2^24) out of range", n_requests, kvpr::kMaxRequests, n_rows, vocab);
    if ((int64_t)n_rows * ((vocab + 2047) / 2048) > 0x7fffff) return fail(KVPR_E_RANGE, "n_rows=%d of vocab=%d logits are too many", n_rows, vocab);
    return KVPR_OK;
}

extern "C" size_t kvpr_verify_workspace_bytes(int n_requests, int n_rows, int vocab) {
    if (check_verify(n_requests, n_rows, vocab)) return 0;
    return kvpr::verify_workspace_bytes(n_requests, n_rows, vocab);
}

extern "C" int kvpr_verify_step(const void* target_logits, const void* draft_logits, int logits_type, int64_t ld_target, int64_t ld_draft, int vocab,
                                const int32_t* tokens, const int32_t* row_start, const int32_t* seq_len, const int32_t* certain, int n_requests,
                                int n_rows, const float* temperature, const float* u_accept, const float* u_sample, const int32_t* len_in, int32_t* len_out,
                                int32_t* kept, int32_t* out_tokens, void* ws, size_t ws_bytes, void* stream) {
    if (int rc = check_verify(n_requests, n_rows, vocab)) return rc;
    if (logits_type != KVPR_F16 && logits_type != KVPR_F32) return fail(KVPR_E_INVAL, "logits_type must be KVPR_F16 or KVPR_F32");
    if (ld_target < vocab || (draft_logits && ld_draft < vocab)) return fail(KVPR_E_INVAL, "row strides must be at least vocab");
    if (!row_start || !temperature || !u_sample || !kept || (n_rows > 0 && (!target_logits || !tokens || !u_accept || !out_tokens)))
        return fail(KVPR_E_INVAL, "null pointer");
    if (!len_in != !len_out) return fail(KVPR_E_INVAL, "len_in and len_out go together");
    const unsigned elem = logits_type == KVPR_F16 ? 1 : 3;
    if (((uintptr_t)target_logits | (uintptr_t)draft_logits) & elem || !aligned16(ws)) return fail(KVPR_E_INVAL, "logits or ws not aligned");
    const size_t need = kvpr::verify_workspace_bytes(n_requests, n_rows, vocab);
    if (!ws || ws_bytes < need) return fail(KVPR_E_INVAL, "the workspace must hold %zu bytes", need);
    const kvpr::Verify v{target_logits, draft_logits, ld_target, ld_draft, tokens, row_start, len_in, seq_len, certain, temperature, u_accept, u_sample, len_out, kept,
                         out_tokens, vocab, n_requests, n_rows, logits_type == KVPR_F16};
    return kvpr::launch_verify(v, ws, (hipStream_t)stream);
}

extern "C" int kvpr_verify_drafts(const void* target_logits, const void* draft_logits, int logits_type, int64_t ld_target, int64_t ld_draft, int vocab,
                                  const int32_t* tokens, const int32_t* row_start, int n_requests, int n_rows, const float* temperature,
                                  const float* u_accept, const float* u_sample, const int32_t* len_in, int32_t* len_out, int32_t* kept,
                                  int32_t* out_tokens, void* ws, size_t ws_bytes, void* stream) {
    return kvpr_verify_step(target_logits, draft_logits, logits_type, ld_target, ld_draft, vocab, tokens, row_start, nullptr, nullptr, n_requests, n_rows,
                            temperature, u_accept, u_sample, len_in, len_out, kept, out_tokens, ws, ws_bytes, stream);
}
