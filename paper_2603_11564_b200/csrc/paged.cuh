// The paged cache: geometry, page lookup and the 4-bit format (include/dapq.h states both).
#pragma once
#include <cuda_fp16.h>
#include <cuda_fp4.h>
#include <cuda_fp8.h>

#include "dapq_internal.cuh"

namespace dapq {

struct PagedDev {
  char *k, *v;
  unsigned char *k_scales, *v_scales;             // 4-bit format only
  int64_t page_stride, head_stride, row_stride;   // channels
  const int32_t *table, *len;
  int32_t table_stride, n_pages, page_shift, fp4;
  float k_scale, v_scale;
};

// New rows of the sequences of a call (by value, like SeqTable).
struct NewRows {
  int32_t batch;
  int32_t cu[kMaxBatch + 1];
};

struct NewTokensDev {
  const void *k, *v, *q;
  void* q_rot;
  int64_t k_stride, v_stride, q_stride;           // elements between tokens
  const int32_t* positions;
};

struct ReadRows {
  NewRows rows;                                   // cu: rows read before each sequence's
  int32_t first[kMaxBatch], row_at[kMaxBatch];
};

cudaError_t launch_paged_append(int dtype, const PagedDev& pg, const NewRows& t, const NewTokensDev& nt, const double* inv_freq_dev, const Dims& dm,
                                int* status, cudaStream_t s, LaunchLog* log);
cudaError_t launch_paged_compact(int dtype, const PagedDev& pg, const CacheDev& cv, const int32_t* idx, const SeqTable& t, int n_kv_heads, int* status,
                                 cudaStream_t s, LaunchLog* log);
cudaError_t launch_paged_read(int dtype, const PagedDev& pg, const ReadRows& t, int n_kv_heads, void* k_out, void* v_out, int64_t out_head_stride,
                              int* status, cudaStream_t s, LaunchLog* log);

// Attention (paged_attend.cu).  part: attend_part_floats(n_sm) floats; sync: attend_sync_words(n_sm) words, all 0 between calls.
size_t attend_part_floats(int n_sm);
size_t attend_sync_words(int n_sm);
cudaError_t launch_paged_attend(int dtype, const PagedDev& pg, const NewRows& t, const Dims& dm, const void* q, int64_t q_stride, float softcap, void* out,
                                float* lse, float* part, uint32_t* sync, int n_sm, int* status, cudaStream_t s, LaunchLog* log);

// Channel offset of row `row` of sequence b and head `head`; negative if the sequence has no such row.
__device__ __forceinline__ int64_t paged_row(const PagedDev& pg, int b, int64_t row, int head) {
  const int64_t p = row >> pg.page_shift;
  if (p >= pg.table_stride) return -1;
  const int page = pg.table[(int64_t)b * pg.table_stride + p];
  if ((unsigned)page >= (unsigned)pg.n_pages) return -1;
  return page * pg.page_stride + head * pg.head_stride + (row & ((1 << pg.page_shift) - 1)) * pg.row_stride;
}

// Two codes of a byte as fp16 (exact).
__device__ __forceinline__ __half2 fp4x2_to_half2(uint32_t byte) {
  return __half2(__nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)byte, __NV_E2M1));
}
// Two e4m3 scales as fp16 (exact).
__device__ __forceinline__ __half2 scales_to_half2(uint32_t two) {
  return __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3));
}
__device__ __forceinline__ float scale_to_float(uint32_t one) { return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)one, __NV_E4M3))); }

}  // namespace dapq
