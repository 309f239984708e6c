// Device code that the calls on pages and rows share: copying parts of pages,
// scans over a CTA, ranks of flagged elements, free pages by rank.
#pragma once

#include "ps_kv.cuh"

namespace pskv {

constexpr int kCopyThreads = 256;

// ---- moving keys and values ---------------------------------------------------
constexpr int kCopyWords = 512;  // 16-byte words of a page that a warp copies at a time
constexpr int kCopyWarps = kCopyThreads / 32;

__host__ __device__ __forceinline__ int copy_parts(const Pool& p, int tok) {
  return (tok * p.kv_heads * (p.head_dim / 8) + kCopyWords - 1) / kCopyWords;
}
// Part 'part' of copying 'tok' tokens of one page of one layer (slice / 2; keys
// or values by slice mod 2), by a warp.  Bound by HBM: one read and one write of
// the page, eight words a lane in flight.  (A CTA of 256 threads for a page had
// two words a thread in flight where a page is 8 KB: 5.1 TB/s of the 6.8 that
// copies reach.)  1.07 GB read and written in pages of 16 KB: 161 us, 6.7 TB/s; the
// moves of a compaction, 1.16 GB: 178 us.  A page that is one run of memory is copied as such; otherwise
// a word's token, head and place are found by division.
__device__ __forceinline__ void copy_part(const Pool& p, int64_t src, int64_t dst, int slice, int tok, int part, int lane) {
  const int words = p.head_dim / 8;  // 16-byte words of a head
  const int n = min(tok * p.kv_heads * words, (part + 1) * kCopyWords);
  char* base = ((slice & 1) ? p.v : p.k) + 2 * (slice >> 1) * p.layer_stride;
  const uint4* s = reinterpret_cast<const uint4*>(base + 2 * src * p.page_stride);
  uint4* d = reinterpret_cast<uint4*>(base + 2 * dst * p.page_stride);
  const bool token_major = p.head_stride == p.head_dim && p.token_stride == (int64_t)p.kv_heads * p.head_dim;
  const bool head_major = tok == p.page_size && p.token_stride == p.head_dim &&
                          p.head_stride == (int64_t)p.page_size * p.head_dim;
  const bool run = token_major || head_major;
  for (int i0 = part * kCopyWords + lane; i0 < n; i0 += 8 * 32) {
    uint4 w[8];
    int64_t at[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int i = i0 + 32 * u;
      at[u] = i;
      if (!run) {
        const int r = i / words, h = r % p.kv_heads, t = r / p.kv_heads;
        at[u] = (t * p.token_stride + h * p.head_stride) / 8 + i % words;
      }
      if (i < n) w[u] = __ldcs(s + at[u]);
    }
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (i0 + 32 * u < n) __stcs(d + at[u], w[u]);
  }
}

// ---- scans ----------------------------------------------------------------------
// Exclusive scan over the CTA of one value a thread, in the type of its sums.
template <typename T>
__device__ __forceinline__ T block_scan(T v, T* total) {
  __shared__ T wsum[kScanThreads / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  T incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T x = __shfl_up_sync(0xFFFFFFFFu, incl, o);
    if (lane >= o) incl += x;
  }
  if (lane == 31) wsum[warp] = incl;
  __syncthreads();
  T base = 0, tot = 0;
#pragma unroll
  for (int w = 0; w < kScanThreads / 32; ++w) {
    if (w < warp) base += wsum[w];
    tot += wsum[w];
  }
  __syncthreads();
  *total = tot;
  return base + incl - v;
}
// Exclusive scan of in[0, n) into out by one CTA; returns the total.
__device__ __forceinline__ int scan_array(const int32_t* in, int32_t* out, int n) {
  int carry = 0;
  for (int i0 = 0; i0 < n; i0 += kScanThreads) {
    const int i = i0 + threadIdx.x;
    int tot;
    const int e = block_scan(i < n ? __ldcg(in + i) : 0, &tot);
    if (i < n) out[i] = carry + e;
    carry += tot;
  }
  return carry;
}
// Ranks of flagged elements in a tile of kTile: thread t holds the flags of
// elements u kScanThreads + t, u = 0..kEach-1, and gets the flagged elements
// before each; *total of the tile.  One pass over the tile's loads.
constexpr int kEach = 8, kTile = kEach * kScanThreads;
__device__ __forceinline__ void tile_ranks(const bool (&flag)[kEach], int (&rank)[kEach], int* total) {
  constexpr int kWarps = kScanThreads / 32;
  __shared__ int count[kEach * kWarps + 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    const unsigned m = __ballot_sync(0xFFFFFFFFu, flag[u]);
    rank[u] = __popc(m & ((1u << lane) - 1));
    if (lane == 0) count[u * kWarps + warp] = __popc(m);
  }
  __syncthreads();
  if (warp == 0) {  // exclusive sums of the 64 counts, two a lane
    static_assert(kEach * kWarps == 64, "two counts a lane");
    const int a = count[2 * lane], b = count[2 * lane + 1];
    int incl = a + b;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xFFFFFFFFu, incl, o);
      if (lane >= o) incl += x;
    }
    __syncwarp();
    count[2 * lane] = incl - a - b;
    count[2 * lane + 1] = incl - b;
    if (lane == 31) count[64] = incl;
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kEach; ++u) rank[u] += count[u * kWarps + warp];
  *total = count[64];
}
// True in every thread of the last CTA of the grid to come here; what the other
// CTAs wrote before is then visible.  The count returns to 0 for the next call.
__device__ __forceinline__ bool last_cta(int32_t* done) {
  __shared__ bool last;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) {
    last = atomicAdd(done, 1) == (int)gridDim.x - 1;
    if (last) *done = 0;
  }
  __syncthreads();
  if (last) __threadfence();
  return last;
}

// The free page of rank r (ascending ids), as an index into the reference array;
// base: the free pages before each chunk.
__device__ __forceinline__ int free_page(const PageScratch& w, const int* base, int r) {
  int lo = 0, hi = w.chunks - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (base[mid] <= r) lo = mid;
    else hi = mid - 1;
  }
  return w.list[(int64_t)lo * w.chunk_size + (r - base[lo])];
}

}  // namespace pskv
