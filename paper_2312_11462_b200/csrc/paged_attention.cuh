// Kernels behind csd_paged_attention.
#pragma once
#include "paged_schedule.cuh"

namespace csd {

constexpr size_t PAGED_TICKET_BYTES = 4096;      // tickets at the start of the workspace: zero between calls, whatever their shapes

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ uint32_t pack_bf16(float x, float y) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
// whether either of two bf16 is an infinity or NaN
__device__ __forceinline__ bool odd_bf16(uint32_t two) { return (two & 0x7f80u) == 0x7f80u || (two & 0x7f800000u) == 0x7f800000u; }

// The model's own calls: fp32 rows that are still to be turned (paged_cache.cu, paged_attention.cu).
csd_status paged_append_turned(const csd_kv_pool* pool, const csd_paged_batch* batch, const float* k, const float* v, int64_t ld, const RopeView& rope,
                               const unsigned long long* tree, void* stream);
csd_status paged_attention_turned(const csd_kv_pool* pool, const csd_paged_batch* batch, const float* q, int64_t ldq, int n_heads, float scale,
                                  const RopeView& rope, const uint64_t* tree, float* out, int64_t ldo, void* workspace, size_t workspace_bytes, void* stream);

// Few rows (decode, reviews, trees) or fp32 rows: paged_rows.cu
size_t paged_rows_workspace(int d_head);
csd_status launch_paged_rows(const PagedView& w, AttendArgs a, int d_head, int packed_rows, int row_type, void* workspace, cudaStream_t st);

// Chunks of many bf16 rows, causal, positive scale: paged_chunk.cu
size_t paged_chunk_workspace(int d_head);
csd_status launch_paged_chunk(const PagedView& w, AttendArgs a, int d_head, void* workspace, cudaStream_t st);

}  // namespace csd
