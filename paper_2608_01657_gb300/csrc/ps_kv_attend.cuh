// Arguments and helpers of the attention kernels (narrow and wide tiles).
#pragma once

#include <cuda.h>

#include "ps_kv.cuh"

namespace pskv {

struct AttendArgs {
  Pool pool;
  Plan plan;
  const char *k, *v;  // the pool at the call's layer
  const char* q;
  char* out;
  float* lse;
  int64_t q_stride[2], out_stride[2];
  const int32_t* tables;
  int64_t table_stride;
  const int32_t* q_offsets;
  int32_t* status;
  int32_t layer, after_wide;  // after_wide: the wide tiles' kernel was launched
  float scale2;  // scale log2(e)
};

// The log of a row's sum of exponentials, from its base-2 maximum and sum.
__device__ __forceinline__ float log_sum(float m, float l) {
  return l == 0 ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

// The wide tiles' kernel (ps_kv_attend_wide.cu).
cudaError_t launch_wide(const AttendArgs& a, const PoolMaps& maps, cudaStream_t st);
cudaError_t configure_wide(const Pool& p);

}  // namespace pskv
