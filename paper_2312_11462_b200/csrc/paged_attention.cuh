// Kernels behind csd_paged_attention.
#pragma once
#include "paged_schedule.cuh"

namespace csd {

// Few rows (decode, reviews, trees) or fp32 rows: paged_rows.cu
size_t paged_rows_workspace(int d_head, int packed_rows, int row_type, bool e4m3);
csd_status launch_paged_rows(const PagedView& w, AttendArgs a, int d_head, int packed_rows, int row_type, void* workspace, cudaStream_t st);

}  // namespace csd
