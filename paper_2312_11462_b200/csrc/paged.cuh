// The paged cache as the kernels see it: checks of the caller's structs, the batch's lengths, and where a position lies.
#pragma once
#include "common.cuh"

namespace csd {

struct PagedView {
    const unsigned char* k; const unsigned char* v;      // [page][head][slot] rows of row_bytes
    const uint8_t* k_exp; const uint8_t* v_exp;          // null: bf16 rows
    const int32_t* table; const int32_t* row_start; const int32_t* kv_len;
    int* status;
    int n_pages, page_shift, heads, n_seqs, max_pages, total_rows, max_rows;
    int capacity;                                        // positions of a sequence: max_pages * page_size
};

// Checks the structs and fills in the view, without a device call.
inline csd_status paged_view(const csd_kv_pool* pool, const csd_paged_batch* batch, PagedView* out) {
    if (!pool || !batch) return CSD_ERR_INVALID_ARG;
    if (pool->kind != CSD_KV_BF16 && pool->kind != CSD_KV_E4M3) return CSD_ERR_INVALID_ARG;
    if (pool->n_pages < 1 || pool->n_kv_heads < 1) return CSD_ERR_INVALID_ARG;
    if (pool->d_head != 64 && pool->d_head != 128) return CSD_ERR_SHAPE;
    int shift = 4;
    while (shift < 7 && (1 << shift) != pool->page_size) ++shift;
    if ((1 << shift) != pool->page_size) return CSD_ERR_SHAPE;
    if ((long long)pool->n_pages * pool->n_kv_heads >= (1ll << 31) >> shift) return CSD_ERR_SHAPE;
    if (!pool->k_dev || !pool->v_dev || (((uintptr_t)pool->k_dev) & 15) || (((uintptr_t)pool->v_dev) & 15)) return CSD_ERR_INVALID_ARG;
    if (pool->kind == CSD_KV_E4M3 &&
        (!pool->k_exp_dev || !pool->v_exp_dev || (((uintptr_t)pool->k_exp_dev) & 15) || (((uintptr_t)pool->v_exp_dev) & 15)))
        return CSD_ERR_INVALID_ARG;
    if (batch->n_seqs < 1 || batch->n_seqs > CSD_MAX_SEQS || batch->max_pages < 1 || batch->total_rows < 0 || batch->max_rows < 1)
        return CSD_ERR_INVALID_ARG;
    if ((long long)batch->max_pages << shift >= 1ll << 30) return CSD_ERR_INVALID_ARG;
    if (!batch->page_table_dev || !batch->row_start_dev || !batch->kv_len_dev) return CSD_ERR_INVALID_ARG;
    PagedView& w = *out;
    w.k = (const unsigned char*)pool->k_dev; w.v = (const unsigned char*)pool->v_dev;
    w.k_exp = pool->kind == CSD_KV_E4M3 ? pool->k_exp_dev : nullptr;
    w.v_exp = pool->kind == CSD_KV_E4M3 ? pool->v_exp_dev : nullptr;
    w.table = batch->page_table_dev; w.row_start = batch->row_start_dev; w.kv_len = batch->kv_len_dev;
    w.n_pages = pool->n_pages; w.page_shift = shift; w.heads = pool->n_kv_heads; w.n_seqs = batch->n_seqs;
    w.max_pages = batch->max_pages; w.total_rows = batch->total_rows; w.max_rows = batch->max_rows;
    w.capacity = batch->max_pages << shift;
    w.status = nullptr;                                  // (the launching call fills it in, behind its own checks)
    return CSD_OK;
}

inline bool paged_rows_ok(const void* p, int64_t ld, int64_t width) {
    return p && ld >= width && (ld & 7) == 0 && (((uintptr_t)p) & 15) == 0;
}

// Rotary tables [positions][d_head / 2] of a model whose rows still have to be turned (null: they come turned).
struct RopeView { const float* cos; const float* sin; int positions; };

// ---- device side
struct PagedSeq { int start, rows, kv; };               // first row, rows, positions before them

// A sequence's lengths, cut to their ranges.
__device__ __forceinline__ PagedSeq paged_seq(const PagedView& w, int s) {
    const int a = w.row_start[s], b = w.row_start[s + 1], kv = w.kv_len[s];
    const int lo = min(max(a, 0), w.total_rows), hi = min(max(b, lo), w.total_rows);
    PagedSeq q;
    q.start = lo; q.rows = min(hi - lo, w.max_rows); q.kv = min(max(kv, 0), w.capacity);
    if (lo != a || hi != b || q.rows != hi - lo || kv < 0) set_status(w.status, CSD_ERR_INVALID_ARG);
    if (q.rows > 0 && (long long)max(kv, 0) + q.rows > w.capacity) set_status(w.status, CSD_ERR_CAPACITY);
    return q;
}

// Rotary position of row i of a chunk of `rows`: behind its ancestors, which are the rows of its mask other than itself (bits behind the
// chunk's rows are nobody); without masks all rows before it.
__device__ __forceinline__ int rope_position(const PagedView& w, const RopeView& r, int kv, int i, int rows, const unsigned long long* mask) {
    const int pos = kv + (mask ? __popcll(*mask & ~(1ull << (i & 63)) & (rows < 64 ? (1ull << rows) - 1 : ~0ull)) : i);
    if (pos >= r.positions) set_status(w.status, CSD_ERR_CAPACITY);
    return min(pos, r.positions - 1);
}
// Turns 8 neighbouring dimensions x, of column col of a row, with those half a row away.
__device__ __forceinline__ void rope8(const RopeView& r, int pos, int half, int col, float* x, const float* other) {
    const bool upper = col >= half;
    const float* c = r.cos + (size_t)pos * half + (col - (upper ? half : 0));
    const float* s = r.sin + (size_t)pos * half + (col - (upper ? half : 0));
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = upper ? other[j] * s[j] + x[j] * c[j] : x[j] * c[j] - other[j] * s[j];
}

// Page of position t of sequence s; -1 where there is none.
__device__ __forceinline__ int paged_page(const PagedView& w, int s, int t) {
    if (t >= w.capacity) return -1;
    const int page = w.table[(size_t)s * w.max_pages + (t >> w.page_shift)];
    if (page < 0 || page >= w.n_pages) { set_status(w.status, CSD_ERR_BAD_PAGE); return -1; }
    return page;
}

// Row of the pool (of d_head elements) that holds slot t % page_size of a page, for one head.
__device__ __forceinline__ size_t paged_row(const PagedView& w, int page, int head, int t) {
    return ((size_t)page * w.heads + head << w.page_shift) + (t & ((1 << w.page_shift) - 1));
}

// Scale of an 8-bit row: 2^(e - 127), NaN for 255.
__device__ __forceinline__ float row_scale(unsigned e) { return __uint_as_float(e << 23 | (e == 255u ? 1u << 22 : 0u)); }

}  // namespace csd
