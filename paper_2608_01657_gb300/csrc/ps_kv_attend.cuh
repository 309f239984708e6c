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
  const int32_t *q_offsets, *kv_lens;
  int32_t* status;
  int32_t after_wide;  // the wide tiles' kernel was launched
  int32_t causal;
  // Which of the header's two marks this call sets where an output is not finite:
  // the calls take turns, and each one's join clears the other mark for the next
  // call, so that finite layers after one that was not do not look at rows again.
  int32_t turn;
  int32_t fill, num_tokens;  // the outputs' rows become NaN after an empty plan
  float scale2;  // scale log2(e)
};

// ---- barriers and asynchronous copies, shared by both kernels ----------------------
__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint64_t* b, int count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(b)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t* b) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(b)) : "memory");
}
__device__ __forceinline__ void bar_expect(uint64_t* b, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_addr(b)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_test(uint64_t* b, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
      : "=r"(ok) : "r"(smem_addr(b)), "r"(parity) : "memory");
  return ok != 0;
}
// Bound of every wait: far beyond any tile's time, so it only ends a wait that
// would never end.
constexpr int kWaitLimit = 1 << 20;
// False if the wait ran out.
__device__ __forceinline__ bool bar_wait(uint64_t* b, uint32_t parity) {
#pragma unroll 1
  for (int i = 0; i < kWaitLimit; ++i)
    if (bar_test(b, parity)) return true;
  return false;
}
// The same by a whole warp, with one answer.
__device__ __forceinline__ bool warp_wait(uint64_t* b, uint32_t parity) { return __all_sync(0xFFFFFFFFu, bar_wait(b, parity)); }
// True in one lane of a converged warp.  The matrix and bulk copy instructions'
// operands are uniform registers: issued by the elected lane a matrix instruction
// takes 5 instructions, under a test of the lane's number up to 44.
__device__ __forceinline__ bool elect() {
  uint32_t e;
  asm volatile("{ .reg .pred p; elect.sync _|p, 0xFFFFFFFF; selp.u32 %0, 1, 0, p; }" : "=r"(e));
  return e != 0;
}
// A box of one page, see PoolMaps: 64 elements from x on, or a head's elements.
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, uint64_t* bar, int x, int head, int token, int page) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"(map), "r"(x), "r"(head), "r"(token), "r"(page), "r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void tma_load_whole(uint32_t dst, const CUtensorMap* map, uint64_t* bar, int head, int token, int page) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %2, %4, %5}], [%6];" ::"r"(dst),
      "l"(map), "r"(0), "r"(token), "r"(head), "r"(page), "r"(smem_addr(bar)) : "memory");
}
// 16 bytes into shared memory, or zeros where !ok (src is not read then).
__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool ok) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void to_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// The log of a row's sum of exponentials, from its base-2 maximum and sum.
__device__ __forceinline__ float log_sum(float m, float l) {
  return l == 0 ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

// x is added to z as 0, or as NaN if it is not finite.
__device__ __forceinline__ float spoil(float z, float x) { return fmaf(x, 0.0f, z); }
// An output of (tile, head) is not finite: the join looks at its rows (mend_row).
__device__ __forceinline__ void ask_mend(const AttendArgs& a, int list, int tile, int head) {
  a.plan.mend[list][(int64_t)tile * a.pool.kv_heads + head] = 1;
  a.plan.hdr->mend[a.turn] = 1;
}

// The wide tiles' kernel (ps_kv_attend_wide.cu).
cudaError_t launch_wide(const AttendArgs& a, const PoolMaps& maps, cudaStream_t st);
cudaError_t configure_wide(const Pool& p);
void make_query_map(const Pool& p, const void* q, const int64_t* stride, int32_t tokens, PoolMaps* m);

}  // namespace pskv
