// ps_step_blocks: the block ids of every request of the last step.
//
// A step leaves each position's key in the workspace; a warp per request looks
// its keys up in the table as the step left it, 32 blocks at a time, up to the
// first that is not resident.  A warp has its request's next 32 keys, then their
// buckets, under way and nothing behind them, so the longest request's chain of
// reads sets the time: 82 us for the 600,000 blocks of 4096 requests, 118 with a
// cold L2 (34.6 MB from HBM, 5 us' worth).
#include "prefixshield_kv.h"
#include "ps_device.cuh"

struct ps_handle;
namespace ps {
const DevState* handle_state(const ps_handle_t* h);
int32_t handle_scratch_requests(const ps_handle_t* h);

namespace {

// The resident block of (key, group), kNone if there is none: the home bucket,
// then following buckets while the overflow count says that a key passed.
__device__ __forceinline__ uint32_t resident_block(const DevState& s, uint64_t key, uint32_t g) {
  const uint32_t mask = (1u << s.tb_nbuckets_log2) - 1;
  uint32_t b = table_home(key, g, s.tb_nbuckets_log2);
  for (uint32_t it = 0; it <= mask; ++it, b = (b + 1) & mask) {
    const TableEntry* e = s.table + (size_t)b * kTableWays;
    uint32_t hit = kNone;
#pragma unroll
    for (int w = 0; w < kTableWays; ++w) {
      const TableEntry x = e[w];
      if (x.blk != kNone && x.key == key && x.grp == g) hit = x.blk;
    }
    if (hit != kNone || s.table_ovf[b] == 0) return hit;
  }
  return kNone;
}

__global__ void __launch_bounds__(256) k_step_blocks(DevState s, int R, const int32_t* groups, int32_t* tables,
                                                     int64_t stride, int32_t* counts, int32_t* status) {
  const int i = (int)((blockIdx.x * (int64_t)blockDim.x + threadIdx.x) >> 5), lane = lane_id();
  if (i >= R) return;
  const int st = s.ctl->status;
  if (st != PS_OK) {
    if (lane == 0) {
      counts[i] = 0;
      if (status) atomicMin(status, st);
    }
    return;
  }
  const int n = s.rq_n[i];
  const int64_t base = s.rq_pbase[i];
  const uint32_t g = (uint32_t)groups[i];
  int found = 0;
  for (int m0 = 0; m0 < n; m0 += 32) {
    const int m = m0 + lane;
    uint32_t blk = kNone;
    if (m < n) blk = resident_block(s, s.pos_key[base + m], g);
    const unsigned miss = __ballot_sync(kFull, blk == kNone);
    const int here = miss ? __ffs(miss) - 1 : 32;
    if (lane < here && m < stride) tables[i * stride + m] = (int32_t)blk;
    found += here;
    if (miss) break;
  }
  if (lane == 0) {
    if (found > stride && status) atomicMin(status, PS_ERR_CAPACITY);
    counts[i] = found < stride ? found : (int32_t)stride;
  }
}

}  // namespace
}  // namespace ps

extern "C" int32_t ps_step_blocks(ps_handle_t* h, void* stream, int32_t num_requests, const int32_t* d_group_ids,
                                  int32_t* d_tables, int64_t table_stride, int32_t* d_counts, int32_t* d_status) {
  if (!h || num_requests < 0 || table_stride < 0) return PS_ERR_INVALID_ARG;
  const ps::DevState& s = *ps::handle_state(h);
  // only what a step wrote may be read: the rest of the scratch was never set
  if (num_requests > ps::handle_scratch_requests(h)) return PS_ERR_INVALID_ARG;
  if (num_requests == 0) return PS_OK;
  if (!d_group_ids || !d_counts || (!d_tables && table_stride > 0)) return PS_ERR_INVALID_ARG;
  const int64_t threads = (int64_t)num_requests * 32;
  ps::k_step_blocks<<<(unsigned)((threads + 255) / 256), 256, 0, static_cast<cudaStream_t>(stream)>>>(
      s, num_requests, d_group_ids, d_tables, table_stride, d_counts, d_status);
  return cudaGetLastError() == cudaSuccess ? PS_OK : PS_ERR_CUDA;
}
