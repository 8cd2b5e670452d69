// csd_paged_attention: checks, and which kernel takes a call.
#include "paged_attention.cuh"

using namespace csd;

// Shapes of a call, without its pointers.
static csd_status check_attend(const csd_kv_pool* pool, const csd_paged_batch* batch, int n_heads, int row_type, PagedView* w) {
    const csd_status ok = paged_view(pool, batch, w);
    if (ok != CSD_OK) return ok;
    if (n_heads < 1 || n_heads % pool->n_kv_heads || n_heads / pool->n_kv_heads > 64) return CSD_ERR_SHAPE;
    if (row_type != CSD_F32 && row_type != CSD_BF16) return CSD_ERR_INVALID_ARG;
    if ((long long)pool->n_kv_heads * (w->capacity / 128 + 8) >= 1ll << 31) return CSD_ERR_CAPACITY;       // units of a row block (paged_schedule.cuh)
    return (long long)batch->max_rows * (n_heads / pool->n_kv_heads) < 1 << 30 ? CSD_OK : CSD_ERR_CAPACITY;
}

// (row, query head) pairs of one sequence and kv head at most
static int packed_rows(const csd_paged_batch* batch, const csd_kv_pool* pool, int n_heads) {
    return batch->max_rows * (n_heads / pool->n_kv_heads);
}

// Which kernel takes bf16 rows.  Up to 32 pairs are one or two blocks of 16 of the rows kernel, which then reads the cache once; from 33 on it
// reads it several times, and the chunk kernel's block of 256 once.  32 heads on 8, us in the rows and the chunk kernel:
//             1 sequence x 16000         16 x 4000                64 x 2000
//   pairs    bf16   8 bits  64 dims    bf16   8 bits  64 dims    bf16    8 bits   64 dims
//    16     29 37   25 41   23 34     57 77   51 95   37 70    104 148   94 181   66 130
//    32     39 37   35 41   27 34     74 77   78 96   52 70    139 148  148 180   93 130
//    48     49 37   48 41   35 34    130 77  142 96   91 70    258 149  272 180  174 130
//   128     72 38   73 42   49 34    231 78  254 96  157 71    490 151  524 182  326 131
// The longest chunk decides for all sequences of a call: 500 rows of one and a row of each of 63 others behind 2000 positions take 256 and 185 us (8
// bits: 280 and 222).
static bool takes_chunks(int packed, int row_type) { return row_type == CSD_BF16 && packed > 32; }

extern "C" size_t csd_paged_attention_workspace_bytes(const csd_kv_pool* pool, const csd_paged_batch* batch, int n_heads, int row_type) {
    PagedView w;
    if (check_attend(pool, batch, n_heads, row_type, &w) != CSD_OK) return 0;
    // (the call's scale and masks are not known here: room for either kernel)
    const int packed = packed_rows(batch, pool, n_heads);
    const size_t rows = paged_rows_workspace(pool->d_head), chunk = paged_chunk_workspace(pool->d_head);
    return takes_chunks(packed, row_type) && chunk > rows ? chunk : rows;
}

static csd_status attend(const csd_kv_pool* pool, const csd_paged_batch* batch, const void* q_dev, int64_t ldq, int n_heads, int row_type, float scale,
                         const RopeView& rope, const uint64_t* tree_mask_dev, void* out_dev, int64_t ldo, void* workspace_dev, size_t workspace_bytes,
                         void* stream) {
    PagedView w;
    const csd_status ok = check_attend(pool, batch, n_heads, row_type, &w);
    if (ok != CSD_OK) return ok;
    const int64_t width = (int64_t)n_heads * pool->d_head;
    if (!(scale > -INFINITY && scale < INFINITY) || (tree_mask_dev && batch->max_rows > 64)) return CSD_ERR_INVALID_ARG;
    if (w.total_rows == 0) return CSD_OK;
    if (!paged_rows_ok(q_dev, ldq, width) || !paged_rows_ok(out_dev, ldo, width)) return CSD_ERR_INVALID_ARG;
    if (!workspace_dev || (((uintptr_t)workspace_dev) & 255)) return CSD_ERR_INVALID_ARG;
    if (workspace_bytes < csd_paged_attention_workspace_bytes(pool, batch, n_heads, row_type)) return CSD_ERR_CAPACITY;
    w.status = status_word_device();
    if (!w.status) return CSD_ERR_CUDA;
    AttendArgs a{q_dev, out_dev, (const u64*)tree_mask_dev, ldq, ldo, n_heads / pool->n_kv_heads, scale, rope, nullptr, nullptr};
    const int packed = packed_rows(batch, pool, n_heads);
    if (takes_chunks(packed, row_type) && !tree_mask_dev && scale > 0.f)
        return launch_paged_chunk(w, a, pool->d_head, workspace_dev, (cudaStream_t)stream);
    return launch_paged_rows(w, a, pool->d_head, packed, row_type, workspace_dev, (cudaStream_t)stream);
}

csd_status csd::paged_attention_turned(const csd_kv_pool* pool, const csd_paged_batch* batch, const float* q, int64_t ldq, int n_heads, float scale,
                                       const RopeView& rope, const uint64_t* tree, float* out, int64_t ldo, void* workspace, size_t workspace_bytes,
                                       void* stream) {
    return attend(pool, batch, q, ldq, n_heads, CSD_F32, scale, rope, tree, out, ldo, workspace, workspace_bytes, stream);
}

extern "C" csd_status csd_paged_attention(const csd_kv_pool* pool, const csd_paged_batch* batch, const void* q_dev, int64_t ldq, int n_heads,
                                          int row_type, float scale, const uint64_t* tree_mask_dev, void* out_dev, int64_t ldo,
                                          void* workspace_dev, size_t workspace_bytes, void* stream) {
    return attend(pool, batch, q_dev, ldq, n_heads, row_type, scale, RopeView{}, tree_mask_dev, out_dev, ldo, workspace_dev, workspace_bytes, stream);
}
