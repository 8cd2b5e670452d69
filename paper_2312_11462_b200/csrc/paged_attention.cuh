// Kernels behind csd_paged_attention.
#pragma once
#include "paged_schedule.cuh"

namespace csd {

constexpr size_t PAGED_TICKET_BYTES = 4096;      // tickets at the start of the workspace: zero between calls, whatever their shapes

// Few rows (decode, reviews, trees) or fp32 rows: paged_rows.cu
size_t paged_rows_workspace(int d_head, int packed_rows, int row_type, bool e4m3);
csd_status launch_paged_rows(const PagedView& w, AttendArgs a, int d_head, int packed_rows, int row_type, void* workspace, cudaStream_t st);

// Chunks of many bf16 rows, causal, positive scale: paged_chunk.cu
size_t paged_chunk_workspace(int d_head);
csd_status launch_paged_chunk(const PagedView& w, AttendArgs a, int d_head, void* workspace, cudaStream_t st);

}  // namespace csd
