// ps_kv_layout: where a batch's new tokens go, from the requests' rows and counts.
//
// With o the exclusive sums of the requests' counts c, token t of request i (o_i
// <= t < o_{i + 1}) has position p = s_i + t - o_i (s_i: the tokens before the new
// ones) and slot table[row_i][p / page_size] page_size + p mod page_size.
//
// Integers only: bound by latency, a chain of three reads (a request's row, the
// row's length, a page id) around a scan.  Up to kFused requests every CTA scans
// all of them for itself, so that the call is one launch; of more, a first kernel
// scans 256 requests a CTA, its last CTA the totals.  The rest is a list of units
// of equal size for the warps: 128 columns of a request's table, 128 tokens.  A
// token finds its request by bisection of the offsets.
//
// Each read of the chain is 0.6 to 0.8 us from L2, a launch 2 to 3: decoding 256
// requests of up to 4096 tokens takes 4.3 us, the prompts of 64 requests (49,000
// tokens) 3.8, drafted tokens of 333 requests, padded, 4.7, and two kernels for 3000
// decoding requests 14, whose 4.8 MB need 0.7.  The runs of requests that share a prefix cost nothing beside
// the tables, as CTA 0 compares the ids while the others fill: a thread one of the
// leading ids of neighbouring requests, 8 or 24 of them side by side (a pair of ids a
// thread, 8 at a time, took 2.4 us longer for the drafted tokens; 8 ids alone, whatever
// their number, take 0.2 longer there and 1.5 for 1000 prompts, 24 alone 0.2 for decoding
// and 0.8 for 1000 requests of drafted tokens).  A lane's four
// tokens go through each read together.  8 CTAs an SM in place of 4 took 1 us longer
// for 3000 requests: each reads all offsets.
#include "ps_kv_pages.cuh"

namespace pskv {
namespace {

constexpr int kFused = 1024;             // requests that every CTA scans for itself
constexpr int kNear = 8192;              // and whose offsets every CTA takes to shared memory
constexpr int kItems = kFused / kScanThreads;
constexpr int kUnit = 128;               // columns or tokens of a warp's unit
constexpr int kUnitsPerCta = kScanThreads / 32;

// The total of requests of which one is out of range: more than any real total (2^18
// requests of 2^30 tokens), and 2^10 of them, one a part, add up.
constexpr int64_t kBad = 1ll << 50;

struct Args {
  ps_kv_layout_t l;
  const int32_t *tables, *lens, *held;
  int64_t stride, num_pages;
  LayoutScratch w;
  int32_t* status;
  int32_t num_rows, row_pages, page_log2, lead, lead_log2, most;  // lead: pages that members of a group have in common; most: new tokens of a member
};

template <int N>
struct Count {
  static constexpr int value = N;
};
struct Item {
  int row, start, count;
};
// Requests i, i + step, ...: their reads go side by side.  False if one is out of
// range; such a request has no tokens.
template <int K>
__device__ __forceinline__ bool items_of(const Args& a, int i, int step, int n, Item (&it)[K]) {
  int row[K], start[K], count[K], held[K];
#pragma unroll
  for (int j = 0; j < K; ++j) {
    const int k = i + j * step;
    row[j] = k < n ? (a.l.rows ? a.l.rows[k] : k) : 0;
    start[j] = k < n && a.l.starts ? a.l.starts[k] : 0;
    count[j] = k < n && a.l.counts ? a.l.counts[k] : 1;
  }
#pragma unroll
  for (int j = 0; j < K; ++j) {
    const bool on = row[j] >= 0 && row[j] < a.num_rows;
    held[j] = on ? a.held[row[j]] : -1;
    if (on && !a.l.starts) start[j] = a.lens[row[j]];
  }
  bool ok = true;
#pragma unroll
  for (int j = 0; j < K; ++j) {
    it[j] = Item{row[j], start[j], count[j]};
    const bool good = start[j] >= 0 && count[j] >= 0 && held[j] >= 0 && held[j] <= a.row_pages &&
                      (int64_t)start[j] + count[j] <= (int64_t)held[j] << a.page_log2;
    const bool on = i + j * step < n;
    ok = ok && (good || !on);
    if (!good || !on) it[j] = Item{-1, 0, 0};
  }
  return ok;
}
// May a request share a prefix with its neighbours?
__device__ __forceinline__ bool fits(const Args& a, const Item& x) {
  return x.row >= 0 && x.start >= a.lead << a.page_log2 && x.count <= a.most;
}
// Marks the requests of first..n - 1 whose leading ids differ from those of the one before
// them.  rows: -1 where a request does not share.  A thread takes one of the ids, of
// neighbouring requests, whose ids it reads side by side.
__device__ __forceinline__ void compare_leads(const Args& a, const int* rows, unsigned char* differs, int first, int n) {
  const int threads = kScanThreads >> a.lead_log2, each = (n - first + threads - 1) / threads, k = threadIdx.x & (a.lead - 1);
  const int begin = first + (threadIdx.x >> a.lead_log2) * each, end = min(n, begin + each);
  auto id = [&](int row) { return row >= 0 ? a.tables[row * a.stride + k] : 0; };
  int before = begin > 0 && begin < end ? rows[begin - 1] : -1, last = id(before);
  auto compare = [&](int i0, auto count) {
    constexpr int kIds = decltype(count)::value;
    int row[kIds], x[kIds];
#pragma unroll
    for (int u = 0; u < kIds; ++u) {
      row[u] = i0 + u < end ? rows[i0 + u] : -1;
      x[u] = id(row[u]);
    }
#pragma unroll
    for (int u = 0; u < kIds; ++u) {
      if (before >= 0 && row[u] >= 0 && x[u] != last) differs[i0 + u] = 1;
      before = row[u];
      last = x[u];
    }
  };
  for (int i = begin; i < end;) {  // (256 requests have 8 a thread where pages are of 16)
    if (end - i > 8) compare(i, Count<24>()), i += 24;
    else compare(i, Count<8>()), i += 8;
  }
}

// The offsets of all requests, in shared memory.
struct Near {
  const int* off;
  const Item* item;
  int n;
  __device__ __forceinline__ int offset(int i) const { return off[i]; }
  __device__ __forceinline__ Item at(const Args&, int i) const { return item[i]; }
};
// The offsets in shared memory, the requests in the workspace.
struct Far {
  const int* off;
  const int4* item;
  int n;
  __device__ __forceinline__ int offset(int i) const { return off[i]; }
  __device__ __forceinline__ Item at(const Args&, int i) const {
    const int4 x = item[i];
    return {x.x, x.y, x.z};
  }
};
// Both in the workspace, each part's offsets from 0 on.
struct Farther : Far {
  const int32_t *local, *base;
  __device__ __forceinline__ int offset(int i) const { return i < n ? local[i] + base[i / kLayoutPart] : base[(n + kLayoutPart - 1) / kLayoutPart]; }
};

// 'over': the batch is left out, for a request out of range or more tokens than there is room for.
template <typename O>
__device__ __forceinline__ void fill(const Args& a, const O& o, bool over, int cta, int ctas) {
  const ps_kv_layout_t& l = a.l;
  const int lane = threadIdx.x & 31, n = o.n, rows = n + (l.pad ? 1 : 0);
  const int total = over ? 0 : o.offset(n);
  const int64_t chunks = (a.stride + kUnit - 1) / kUnit;
  const int64_t units = rows * chunks + (l.num_tokens + kUnit - 1) / kUnit;
  for (int64_t u = (int64_t)cta * kUnitsPerCta + (threadIdx.x >> 5); u < units; u += (int64_t)ctas * kUnitsPerCta) {
    if (u < rows * chunks) {  // a request's table
      const int i = (int)(u / chunks);
      const int64_t k0 = u % chunks * kUnit + lane;
      Item it{-1, 0, 0};
      if (i < n && !over) it = o.at(a, i);
      const int64_t pages = it.row < 0 ? 0 : ((int64_t)it.start + it.count + (1 << a.page_log2) - 1) >> a.page_log2;
      const int32_t* src = a.tables + it.row * a.stride;
      int32_t* dst = l.tables + i * a.stride;
#pragma unroll
      for (int j = 0; j < kUnit / 32; ++j) {
        const int64_t k = k0 + 32 * j;
        if (k < a.stride) dst[k] = k < pages ? src[k] : -1;
      }
    } else {
      const int64_t t0 = (u - rows * chunks) * kUnit + lane;
      constexpr int kEachLane = kUnit / 32;
      int of[kEachLane], pos[kEachLane], id[kEachLane], from[kEachLane];
#pragma unroll
      for (int j = 0; j < kEachLane; ++j) {  // the last request that begins at or before t; empty ones lie before it
        const int64_t t = t0 + 32 * j;
        int lo = 0, hi = t < total ? n - 1 : 0;
        while (lo < hi) {
          const int mid = (lo + hi + 1) / 2;
          if (o.offset(mid) <= t) lo = mid;
          else hi = mid - 1;
        }
        of[j] = lo;
      }
#pragma unroll
      for (int j = 0; j < kEachLane; ++j) {
        const int64_t t = t0 + 32 * j;
        pos[j] = from[j] = 0;
        id[j] = -1;
        if (t < total) {
          const Item it = o.at(a, of[j]);
          pos[j] = it.start + (int)t - o.offset(of[j]);
          id[j] = a.tables[it.row * a.stride + (pos[j] >> a.page_log2)];
          from[j] = l.written ? l.written[of[j]] : it.start;
        }
      }
#pragma unroll
      for (int j = 0; j < kEachLane; ++j) {
        const int64_t t = t0 + 32 * j;
        if (t >= l.num_tokens) break;
        int64_t slot = -1;
        if (t < total) {
          if (id[j] < 0 || id[j] >= a.num_pages) set_error(a.status, PS_ERR_INVALID_ARG);
          else if (pos[j] >= from[j]) slot = ((int64_t)id[j] << a.page_log2) + (pos[j] & ((1 << a.page_log2) - 1));
        }
        l.positions[t] = pos[j];
        l.slots[t] = slot;
      }
    }
  }
}

// The offsets' and groups' ends: written by one thread.  The offsets of a batch
// that is left out do not end at its tokens, so that no plan is made of it.
__device__ __forceinline__ void ends(const Args& a, bool over, int total, int groups) {
  const ps_kv_layout_t& l = a.l;
  const int n = l.num_requests;
  l.q_offsets[n] = total;
  if (l.pad) {  // a request without keys takes the tokens that are left, in a group of its own
    l.q_offsets[n + 1] = over ? 0 : l.num_tokens;
    l.kv_lens[n] = 0;
  }
  if (l.group_offsets && l.pad) l.group_offsets[groups] = n;
}

// CTA 0 writes the requests' own numbers, the others fill the tables and tokens.
__global__ void __launch_bounds__(kScanThreads) k_layout(Args a) {
  __shared__ int off[kFused + 1];
  __shared__ Item item[kFused];
  __shared__ unsigned char differs[kFused];
  __shared__ int lead_row[kFused];
  chain();
  const ps_kv_layout_t& l = a.l;
  const int n = l.num_requests, tid = threadIdx.x, i0 = tid * kItems;
  Item it[kItems];
  bool bad = !items_of(a, tid, kScanThreads, n, it);
#pragma unroll
  for (int j = 0; j < kItems; ++j) {
    item[j * kScanThreads + tid] = it[j];
    differs[j * kScanThreads + tid] = 0;
  }
  bad = __syncthreads_or(bad);
  int64_t sum = 0, total;
#pragma unroll
  for (int j = 0; j < kItems; ++j) {
    it[j] = item[i0 + j];
    sum += it[j].count;
  }
  int64_t o = block_scan(sum, &total);
  const bool over = bad || total > l.num_tokens;
#pragma unroll
  for (int j = 0; j < kItems; ++j) {
    off[i0 + j] = over ? 0 : (int)o;
    o += it[j].count;
  }
  if (tid == kScanThreads - 1) off[kFused] = over ? 0 : (int)total;
  __syncthreads();
  if (blockIdx.x > 0) {
    fill(a, Near{off, item, n}, over, blockIdx.x - 1, gridDim.x - 1);
    return;
  }
  if (over && tid == 0) set_error(a.status, bad ? PS_ERR_INVALID_ARG : PS_ERR_CAPACITY);
  for (int i = tid; i < n; i += kScanThreads) {
    l.q_offsets[i] = off[i];
    l.kv_lens[i] = over ? 0 : item[i].start + item[i].count;
  }
  int groups = 0;
  if (l.group_offsets) {
    for (int i = tid; i < n; i += kScanThreads) lead_row[i] = fits(a, item[i]) ? item[i].row : -1;
    __syncthreads();
    compare_leads(a, lead_row, differs, 0, over ? 0 : n);
    __syncthreads();
    int begins = 0;
#pragma unroll
    for (int j = 0; j < kItems; ++j) {
      const int i = i0 + j;
      if (i < n && (i == 0 || over || differs[i] || lead_row[i] < 0 || lead_row[i - 1] < 0)) begins |= 1 << j;
    }
    int g = block_scan(__popc(begins), &groups);
#pragma unroll
    for (int j = 0; j < kItems; ++j)
      if (begins >> j & 1) l.group_offsets[g++] = i0 + j;
    for (int g = groups + (l.pad ? 1 : 0) + tid; g <= n + (l.pad ? 1 : 0); g += kScanThreads) l.group_offsets[g] = n + (l.pad ? 1 : 0);
  }
  if (tid == 0) ends(a, over, over ? 0 : (int)total, groups);
}

// Many requests: a part of them a CTA, one a thread.  Their offsets and groups from the
// CTA's first on, and the CTA's totals, which the last CTA turns into offsets.
__global__ void __launch_bounds__(kScanThreads) k_layout_scan(Args a) {
  static_assert(kLayoutPart == kScanThreads, "one a thread");
  __shared__ int lead_row[kLayoutPart + 1];  // of the request before the part, and the part's
  __shared__ unsigned char differs[kLayoutPart + 1];
  chain();
  const ps_kv_layout_t& l = a.l;
  const int n = l.num_requests, tid = threadIdx.x, i0 = blockIdx.x * kLayoutPart, i = i0 + tid;
  Item both[2];  // the thread's, after the one before the part in thread 0
  const int step = tid == 0 && i0 > 0 ? 1 : 0;
  bool bad = !items_of(a, i - step, step, n, both);
  const Item it = both[1];
  bool begins = i < n;
  if (l.group_offsets) {
    lead_row[tid + 1] = fits(a, it) ? it.row : -1;
    differs[tid + 1] = 0;
    if (tid == 0) lead_row[0] = step && fits(a, both[0]) ? both[0].row : -1;
    __syncthreads();
    compare_leads(a, lead_row, differs, 1, min(kLayoutPart, n - i0) + 1);
    __syncthreads();
    begins = i < n && (differs[tid + 1] || lead_row[tid + 1] < 0 || lead_row[tid] < 0);
  }
  int64_t total;
  int groups;
  const int64_t o = block_scan((int64_t)it.count, &total);
  bad = __syncthreads_or(bad);
  const int g = block_scan((int)begins, &groups);
  if (i < n) {
    // a batch that is left out has offsets past 2^31 perhaps: none is looked at
    const int32_t off = (int32_t)(o < 0x7FFFFFFF ? o : 0x7FFFFFFF);
    a.w.item[i] = make_int4(it.row, it.start, it.count, 0);
    a.w.offset[i] = off;
    a.w.group[i] = begins ? g : -1;
  }
  if (threadIdx.x == 0) {
    a.w.total[blockIdx.x] = bad ? kBad : total;
    a.w.groups[blockIdx.x] = groups;
  }
  if (!last_cta(a.w.done)) return;
  int64_t carry = 0;
  int gcarry = 0;
  for (int c0 = 0; c0 < (int)gridDim.x; c0 += kScanThreads) {
    const int c = c0 + threadIdx.x;
    const bool on = c < (int)gridDim.x;
    int64_t tot;
    int gtot;
    const int64_t e = block_scan<int64_t>(on ? __ldcg(a.w.total + c) : 0, &tot);
    const int ge = block_scan(on ? __ldcg(a.w.groups + c) : 0, &gtot);
    if (on) {
      a.w.base[c] = (int32_t)(carry + e < 0x7FFFFFFF ? carry + e : 0x7FFFFFFF);
      a.w.group_base[c] = gcarry + ge;
    }
    carry += tot;
    gcarry += gtot;
  }
  if (threadIdx.x == 0) {
    a.w.base[gridDim.x] = (int32_t)(carry < 0x7FFFFFFF ? carry : 0x7FFFFFFF);
    a.w.group_base[gridDim.x] = gcarry;
    if (carry > l.num_tokens) set_error(a.status, carry >= kBad ? PS_ERR_INVALID_ARG : PS_ERR_CAPACITY);
  }
}

__global__ void __launch_bounds__(kScanThreads) k_layout_fill(Args a) {
  chain();
  const ps_kv_layout_t& l = a.l;
  const int n = l.num_requests, parts = (n + kLayoutPart - 1) / kLayoutPart;
  const int total = a.w.base[parts], groups = a.w.group_base[parts];
  const bool over = total > l.num_tokens, near = n <= kNear;
  const int64_t id = (int64_t)blockIdx.x * kScanThreads + threadIdx.x, step = (int64_t)gridDim.x * kScanThreads;
  extern __shared__ int off[];
  if (near) {
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += kScanThreads) off[i] = a.w.offset[i] + a.w.base[i / kLayoutPart];
    if (threadIdx.x == 0) off[n] = total;
    __syncthreads();
  }
  const Far o{off, a.w.item, n};
  const Farther far{o, a.w.offset, a.w.base};
  for (int64_t i = id; i < n; i += step) {
    const Item it = o.at(a, (int)i);
    l.q_offsets[i] = over ? 0 : far.offset((int)i);
    l.kv_lens[i] = over ? 0 : it.start + it.count;
    if (l.group_offsets) {
      const int g = a.w.group[i];
      if (over) l.group_offsets[i] = (int)i;
      else if (g >= 0) l.group_offsets[g + a.w.group_base[i / kLayoutPart]] = (int)i;
    }
  }
  const int shown = over ? n : groups, all = n + (l.pad ? 1 : 0);
  if (l.group_offsets)
    for (int64_t g = shown + (l.pad ? 1 : 0) + id; g <= all; g += step) l.group_offsets[g] = all;
  if (id == 0) ends(a, over, over ? 0 : total, shown);
  if (near) fill(a, o, over, blockIdx.x, gridDim.x);
  else fill(a, far, over, blockIdx.x, gridDim.x);
}

}  // namespace

int32_t launch_layout(const Pool& p, const LayoutScratch& w, const ps_kv_layout_t& l, const ps_kv_rows_t& rows,
                      int32_t row_pages, int32_t* status, int nsm, cudaStream_t st) {
  Args a{};
  a.l = l;
  a.tables = rows.tables; a.lens = rows.lens; a.held = rows.held; a.stride = rows.table_stride;
  a.num_pages = p.num_pages; a.w = w; a.status = status;
  a.num_rows = rows.num_rows; a.row_pages = row_pages; a.page_log2 = p.page_log2;
  static_assert(kShareTokens == 128, "whole pages of 2 to 64 tokens");
  a.lead_log2 = 7 - p.page_log2;
  a.lead = 1 << a.lead_log2;
  a.most = kShareRows / p.ratio;
  const int64_t n = l.num_requests;
  const int64_t units = (n + (l.pad ? 1 : 0)) * ((a.stride + kUnit - 1) / kUnit) + ((int64_t)l.num_tokens + kUnit - 1) / kUnit;
  const int64_t want = (units + kUnitsPerCta - 1) / kUnitsPerCta;
  const int64_t most = (int64_t)nsm * 4;
  const int grid = (int)(want < 1 ? 1 : (want > most ? most : want));
  if (n <= kFused) return status_of(launch(k_layout, dim3((unsigned)(grid + 1)), kScanThreads, 0, st, a));
  cudaError_t e = launch(k_layout_scan, dim3((unsigned)((n + kLayoutPart - 1) / kLayoutPart)), kScanThreads, 0, st, a);
  if (e == cudaSuccess) e = launch(k_layout_fill, dim3((unsigned)grid), kScanThreads, n <= kNear ? 4 * (n + 1) : 0, st, a);
  return status_of(e);
}

}  // namespace pskv
