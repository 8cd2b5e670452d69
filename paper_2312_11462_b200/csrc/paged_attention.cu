// Attention of a batch's new rows over the paged cache.  A warp takes one row of one query head: a lane a key for the scores,
// a lane a share of the head dimension for the sums.
#include "paged.cuh"
#include <cuda_fp8.h>

namespace csd {

struct AttendArgs {
    const void* q; void* out; const unsigned long long* tree;
    long long ldq, ldo;
    int heads, group;
    float scale;
};

__device__ __forceinline__ float pool_value(const unsigned char* base, size_t i, bool e4m3) {
    if (!e4m3) return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(base)[i]);
    return __half2float(__half(__nv_cvt_fp8_to_halfraw(base[i], __NV_E4M3)));
}

template <int DH, bool ROWS16>
__global__ void __launch_bounds__(32)
paged_attention_kernel(const PagedView w, const AttendArgs a) {
    const int s = blockIdx.z, i = blockIdx.x, h = blockIdx.y, lane = threadIdx.x, kvh = h / a.group;
    const PagedSeq q = paged_seq(w, s);
    if (i >= q.rows) return;
    const int r = q.start + i;
    const bool e4m3 = w.k_exp != nullptr;
    auto load = [&](const void* p, size_t at) { return ROWS16 ? __bfloat162float(((const __nv_bfloat16*)p)[at]) : ((const float*)p)[at]; };
    const unsigned long long mask = a.tree ? a.tree[r] : 0ull;
    const int total = min(q.kv + (a.tree ? q.rows : i + 1), w.capacity);
    float m = -INFINITY, l = 0.f, o[DH / 32] = {};
    for (int t0 = 0; t0 < total; t0 += 32) {
        const int t = t0 + lane;
        bool seen = t < total && (t < q.kv || !a.tree || (t - q.kv < 64 && (mask >> (t - q.kv) & 1)));
        size_t row = 0;
        if (seen) {
            const int page = paged_page(w, s, t);
            seen = page >= 0;
            if (seen) row = paged_row(w, page, kvh, t);
        }
        float x = -INFINITY;
        if (seen) {
            x = 0.f;
            for (int d = 0; d < DH; ++d) x = fmaf(load(a.q, (size_t)r * a.ldq + h * DH + d), pool_value(w.k, row * DH + d, e4m3), x);
            x *= a.scale * (e4m3 ? exp_scale(w.k_exp[row]) : 1.f);
        }
        const float nm = fmaxf(m, warp_max(x));
        if (nm == -INFINITY) continue;
        const float p = expf(x - nm), keep = expf(m - nm);
        l = l * keep + warp_sum(p);
        m = nm;
        const float sv = seen ? p * (e4m3 ? exp_scale(w.v_exp[row]) : 1.f) : 0.f;
        for (int c = 0; c < DH / 32; ++c) o[c] *= keep;
        for (int j = 0; j < 32; ++j) {
            const float pj = __shfl_sync(0xffffffffu, sv, j);
            const bool see = __shfl_sync(0xffffffffu, (int)seen, j);
            const size_t rj = __shfl_sync(0xffffffffu, (unsigned long long)row, j);
            if (see)
                for (int c = 0; c < DH / 32; ++c) o[c] = fmaf(pj, pool_value(w.v, rj * DH + lane + 32 * c, e4m3), o[c]);
        }
    }
    for (int c = 0; c < DH / 32; ++c) {
        const float y = l > 0.f ? o[c] / l : 0.f;
        const size_t at = (size_t)r * a.ldo + h * DH + lane + 32 * c;
        if constexpr (ROWS16) ((__nv_bfloat16*)a.out)[at] = __float2bfloat16_rn(y);
        else ((float*)a.out)[at] = y;
    }
}

}  // namespace csd

using namespace csd;

// Shapes of a call, without its pointers.
static csd_status check_attend(const csd_kv_pool* pool, const csd_paged_batch* batch, int n_heads, int row_type, PagedView* w) {
    const csd_status ok = paged_view(pool, batch, w);
    if (ok != CSD_OK) return ok;
    if (n_heads < 1 || n_heads % pool->n_kv_heads || n_heads / pool->n_kv_heads > 64) return CSD_ERR_SHAPE;
    return row_type == CSD_F32 || row_type == CSD_BF16 ? CSD_OK : CSD_ERR_INVALID_ARG;
}

extern "C" size_t csd_paged_attention_workspace_bytes(const csd_kv_pool* pool, const csd_paged_batch* batch, int n_heads, int row_type) {
    PagedView w;
    if (check_attend(pool, batch, n_heads, row_type, &w) != CSD_OK) return 0;
    return 256;
}

extern "C" csd_status csd_paged_attention(const csd_kv_pool* pool, const csd_paged_batch* batch, const void* q_dev, int64_t ldq, int n_heads,
                                          int row_type, float scale, const uint64_t* tree_mask_dev, void* out_dev, int64_t ldo,
                                          void* workspace_dev, size_t workspace_bytes, void* stream) {
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
    AttendArgs a{q_dev, out_dev, (const unsigned long long*)tree_mask_dev, ldq, ldo, n_heads, n_heads / pool->n_kv_heads, scale};
    const dim3 grid((unsigned)batch->max_rows, (unsigned)n_heads, (unsigned)batch->n_seqs);
    cudaStream_t st = (cudaStream_t)stream;
    if (pool->d_head == 64) {
        if (row_type == CSD_BF16) paged_attention_kernel<64, true><<<grid, 32, 0, st>>>(w, a);
        else paged_attention_kernel<64, false><<<grid, 32, 0, st>>>(w, a);
    } else {
        if (row_type == CSD_BF16) paged_attention_kernel<128, true><<<grid, 32, 0, st>>>(w, a);
        else paged_attention_kernel<128, false><<<grid, 32, 0, st>>>(w, a);
    }
    CSD_CUDA(cudaGetLastError());
    count_launch();
    return CSD_OK;
}
