// ps_kv_copy, ps_kv_fork, ps_kv_release, ps_kv_compact: page copies, forks of
// sequences, freeing and compaction.
#include "ps_kv_pages.cuh"

namespace pskv {
namespace {

// Whole pages src(i) -> dst(i), all layers, by all warps of the grid.
template <typename Pair>
__device__ __forceinline__ void copy_pages(const Pool& p, int64_t n, Pair pair) {
  const int lane = threadIdx.x & 31, slices = 2 * p.num_layers, parts = copy_parts(p, p.page_size);
  const int64_t total = n * slices * parts, step = (int64_t)gridDim.x * kCopyWarps;
  for (int64_t u = (int64_t)blockIdx.x * kCopyWarps + (threadIdx.x >> 5); u < total; u += step) {
    const int64_t i = u / (slices * parts);
    const int rest = (int)(u % (slices * parts));
    int64_t s, d;
    if (pair(i, &s, &d)) copy_part(p, s, d, rest / parts, p.page_size, rest % parts, lane);
  }
}

__global__ void __launch_bounds__(kCopyThreads) k_page_copy(Pool p, const int32_t* src, const int32_t* dst, int n,
                                                            int32_t* status) {
  chain();
  copy_pages(p, n, [&](int64_t i, int64_t* s, int64_t* d) {
    *s = src[i];
    *d = dst[i];
    const bool ok = *s >= 0 && *s < p.num_pages && *d >= 0 && *d < p.num_pages;
    if (!ok && (threadIdx.x & 31) == 0) set_error(status, PS_ERR_INVALID_ARG);
    return ok;
  });
}

// ---- fork -------------------------------------------------------------------------
struct ForkArgs {
  const int32_t *parents, *children, *room;
  int32_t *tables, *lens, *held;
  int64_t table_stride;
  const int32_t* refs_in;
  int32_t* refs_out;
  int32_t* status;
  int32_t n, num_rows, row_pages;
};

// What item i needs; *total and *full are the child's pages and the pages that
// it shares.  False: out of range.
__device__ __forceinline__ bool fork_item(const Pool& p, const ForkArgs& a, int i, int* len, int* full, int* total) {
  const int pr = a.parents[i], ch = a.children[i], room = a.room[i];
  if (pr < -1 || pr >= a.num_rows || ch < 0 || ch >= a.num_rows || room < 0) return false;
  const int n = pr >= 0 ? a.lens[pr] : 0;
  const int held = pr >= 0 ? a.held[pr] : 0;
  if (n < 0 || held < 0 || held > a.row_pages || n > (int64_t)held << p.page_log2) return false;
  const int most = n > room ? n : room;
  int tot = (int)(((int64_t)most + p.page_size - 1) >> p.page_log2);
  if (tot > a.row_pages) return false;
  *len = n;
  if (pr == ch) {  // in place: the pages held stay
    *full = held;
    *total = tot > held ? tot : held;
  } else {
    *full = n >> p.page_log2;
    *total = tot;
  }
  return true;
}

// CTAs below w.chunks list the free pages of one chunk of the reference array
// each (and copy it to refs_out); the others check one item each.  The last CTA
// to finish turns the counts into offsets and decides whether the call goes
// ahead, so that the second kernel needs no further pass.  Both are bound by the
// latency of a few dependent reads: 7.8 us for 7 forks, 19.5 us for 512 forks of
// 2048-token rows and their release (8.8 us of it the partial pages' copies).
__global__ void __launch_bounds__(kScanThreads) k_fork_scan(Pool p, PageScratch w, ForkArgs a) {
  chain();
  const int64_t np = p.num_pages - p.first_page;
  if ((int)blockIdx.x < w.chunks) {
    const int64_t c0 = (int64_t)blockIdx.x * w.chunk_size;
    const int64_t c1 = c0 + w.chunk_size < np ? c0 + w.chunk_size : np;
    int count = 0;
    for (int64_t i0 = c0; i0 < c1; i0 += kTile) {
      int r[kEach], rank[kEach], tot;
      bool free[kEach];
#pragma unroll
      for (int u = 0; u < kEach; ++u) {
        const int64_t i = i0 + u * kScanThreads + threadIdx.x;
        r[u] = i < c1 ? a.refs_in[i] : 1;
        free[u] = r[u] == 0;
      }
      tile_ranks(free, rank, &tot);
#pragma unroll
      for (int u = 0; u < kEach; ++u) {
        const int64_t i = i0 + u * kScanThreads + threadIdx.x;
        if (i < c1 && a.refs_out != a.refs_in) a.refs_out[i] = r[u];
        if (free[u]) w.list[c0 + count + rank[u]] = (int32_t)i;
      }
      count += tot;
    }
    if (threadIdx.x == 0) w.chunk_cnt[blockIdx.x] = count;
  } else {
    const int i = (int)blockIdx.x - w.chunks;
    int len = 0, full = 0, total = 0;
    bool ok = fork_item(p, a, i, &len, &full, &total);
    const int pr = a.parents[i], ch = a.children[i];
    if (ok && pr >= 0) {  // the ids that the child takes over or copies from
      const int part = pr != ch && (len & (p.page_size - 1)) ? 1 : 0;
      const int32_t* row = a.tables + pr * a.table_stride;
      for (int k = threadIdx.x; k < full + part; k += kScanThreads) {
        const int64_t id = row[k];
        if (id < 0 || id >= p.num_pages || (id >= p.first_page && a.refs_in[id - p.first_page] <= 0)) ok = false;
      }
    }
    // no child is another item's child or parent
    for (int j = threadIdx.x; j < a.n; j += kScanThreads)
      if (j != i && (a.children[j] == ch || a.parents[j] == ch)) ok = false;
    ok = __syncthreads_and(ok);
    if (threadIdx.x == 0) {
      w.need[i] = ok ? total - full : 0;
      w.bad[i] = !ok;
    }
  }
  if (!last_cta(&w.hdr->done)) return;
  const int free_pages = scan_array(w.chunk_cnt, w.chunk_base, w.chunks);
  // the items' needs in 64 bits: the sum of a few may pass 2^31
  int64_t need = 0;
  int any_bad = 0;
  for (int i0 = 0; i0 < a.n; i0 += kScanThreads) {
    const int i = i0 + threadIdx.x;
    int64_t tot;
    const int64_t e = block_scan<int64_t>(i < a.n ? __ldcg(w.need + i) : 0, &tot);
    if (i < a.n) {
      const int64_t s = need + e;
      w.start[i] = s < 0x7FFFFFFF ? (int)s : 0x7FFFFFFF;
      any_bad |= __ldcg(w.bad + i);
    }
    need += tot;
  }
  any_bad = __syncthreads_or(any_bad);
  if (threadIdx.x == 0) {
    const int st = any_bad ? PS_ERR_INVALID_ARG : (need > free_pages ? PS_ERR_CAPACITY : PS_OK);
    w.hdr->status = st;
    w.hdr->free_pages = free_pages;
    if (st != PS_OK) set_error(a.status, st);
  }
}

// blockIdx.x: the item; blockIdx.y: a slice of the layers' keys and values.
// Slice 0 also writes the child's row and the references.  The items and their
// parents' rows are read before the wait for k_fork_scan, which only reads them
// and lets this kernel start when all that came before it is done.
__global__ void __launch_bounds__(kCopyThreads) k_fork_apply(Pool p, PageScratch w, ForkArgs a) {
  __shared__ int base[kMaxChunks];
  const int i = blockIdx.x;
  const int pr = a.parents[i], ch = a.children[i];
  int len = 0, full = 0, total = 0;
  const bool ok = fork_item(p, a, i, &len, &full, &total);
  const int part = len & (p.page_size - 1);
  const bool copies = ok && pr >= 0 && pr != ch && part > 0;
  const int64_t from = copies ? a.tables[pr * a.table_stride + full] : 0;
  chain();
  for (int c = threadIdx.x; c < w.chunks; c += kCopyThreads) base[c] = w.chunk_base[c];
  const int start = w.start[i];
  if (w.hdr->status != PS_OK || (pr == ch && blockIdx.y > 0)) return;
  __syncthreads();  // (the row's lengths are read by every thread before they change, too)
  if (blockIdx.y == 0) {
    const int32_t* src = a.tables + pr * a.table_stride;
    int32_t* row = a.tables + ch * a.table_stride;
    for (int k = threadIdx.x; k < total; k += kCopyThreads) {
      if (k < full) {
        if (pr == ch) continue;
        const int32_t id = src[k];
        row[k] = id;
        if (id >= p.first_page) atomicAdd(a.refs_out + (id - p.first_page), 1);
      } else {
        const int f = free_page(w, base, start + (k - full));
        row[k] = (int32_t)(p.first_page + f);
        a.refs_out[f] = 1;
      }
    }
    if (threadIdx.x == 0) {
      a.lens[ch] = len;
      a.held[ch] = total;
    }
  }
  if (!copies) return;
  const int64_t to = p.first_page + free_page(w, base, start);
  const int parts = copy_parts(p, part), n = 2 * p.num_layers * parts;
  for (int u = blockIdx.y * kCopyWarps + (threadIdx.x >> 5); u < n; u += gridDim.y * kCopyWarps)
    copy_part(p, from, to, u / parts, part, u % parts, threadIdx.x & 31);
}

// ---- release ----------------------------------------------------------------------
__global__ void __launch_bounds__(kScanThreads) k_release(Pool p, const int32_t* list, ps_kv_rows_t rows, int row_pages,
                                                          int32_t* refs, int32_t* status) {
  chain();
  const int r = list[blockIdx.x];
  if (r < 0 || r >= rows.num_rows) {
    if (threadIdx.x == 0) set_error(status, PS_ERR_INVALID_ARG);
    return;
  }
  const int held = rows.held[r];
  __syncthreads();
  if (held < 0 || held > row_pages) {
    if (threadIdx.x == 0) set_error(status, PS_ERR_INVALID_ARG);
    return;
  }
  for (int k = threadIdx.x; k < held; k += kScanThreads) {
    const int64_t id = rows.tables[r * rows.table_stride + k];
    if (id >= 0 && id < p.first_page) continue;  // the prefix cache's
    if (id < 0 || id >= p.num_pages) {
      set_error(status, PS_ERR_INVALID_ARG);
    } else if (atomicSub(refs + (id - p.first_page), 1) <= 0) {
      atomicAdd(refs + (id - p.first_page), 1);
      set_error(status, PS_ERR_INVALID_ARG);
    }
  }
  if (threadIdx.x == 0) {
    rows.held[r] = 0;
    rows.lens[r] = 0;
  }
}

// ---- compaction ---------------------------------------------------------------------
// With L pages in use, those at index >= L move to the free pages below L.
// Both ends are counted by one quantity, the pages in use before an index:
// a free index i < L is hole number i - before(i), and a used index i >= L is
// mover number L - 1 - before(i) counted from the top; the two kernels need no
// count of the pages in use below L.
__global__ void __launch_bounds__(kScanThreads) k_compact_count(Pool p, PageScratch w, const int32_t* refs) {
  chain();
  const int64_t np = p.num_pages - p.first_page;
  const int64_t c0 = (int64_t)blockIdx.x * w.chunk_size;
  const int64_t c1 = c0 + w.chunk_size < np ? c0 + w.chunk_size : np;
  int count = 0;
#pragma unroll 8
  for (int64_t i = c0 + threadIdx.x; i < c1; i += kScanThreads) count += refs[i] > 0;
  int tot;
  block_scan(count, &tot);
  if (threadIdx.x == 0) w.chunk_cnt[blockIdx.x] = tot;
  if (!last_cta(&w.hdr->done)) return;
  const int live = scan_array(w.chunk_cnt, w.chunk_base, w.chunks);
  if (threadIdx.x == 0) w.hdr->live = live;
}

__global__ void __launch_bounds__(kScanThreads) k_compact_lists(Pool p, PageScratch w, const int32_t* refs,
                                                                int32_t* refs_out) {
  chain();
  const int64_t np = p.num_pages - p.first_page;
  const int64_t c0 = (int64_t)blockIdx.x * w.chunk_size;
  const int64_t c1 = c0 + w.chunk_size < np ? c0 + w.chunk_size : np;
  const int live = w.hdr->live;
  int before = w.chunk_base[blockIdx.x];
  for (int64_t i0 = c0; i0 < c1; i0 += kTile) {
    int ref[kEach], rank[kEach], tot;
    bool used[kEach];
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      const int64_t i = i0 + u * kScanThreads + threadIdx.x;
      ref[u] = i < c1 ? refs[i] : 0;
      used[u] = ref[u] > 0;
    }
    tile_ranks(used, rank, &tot);
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      const int64_t i = i0 + u * kScanThreads + threadIdx.x;
      const int r = ref[u], b = before + rank[u];
      if (i >= c1) continue;
      if (i < live) {
        if (r > 0) {
          if (refs_out != refs) refs_out[i] = r;
        } else {
          w.list[i - b] = (int32_t)i;  // its count comes with the mover's
        }
      } else {
        if (r > 0) {
          const int m = live - 1 - b;
          w.movers[m] = (int32_t)i;
          w.mover_refs[m] = r;
          w.inv[i] = m;
        } else {
          w.inv[i] = -1;
        }
        refs_out[i] = 0;
        if (i == live) w.hdr->free_pages = live - b;  // movers: the pages in use from here on
      }
    }
    before += tot;
  }
  // every page in use lies below 'live' if the array ends there: no movers
  if (blockIdx.x == 0 && threadIdx.x == 0 && live == np) w.hdr->free_pages = 0;
}

__global__ void __launch_bounds__(kCopyThreads) k_compact_move(Pool p, PageScratch w, ps_kv_rows_t rows,
                                                               int32_t* tables_out, int32_t* refs_out, int32_t* counts,
                                                               int32_t* status) {
  chain();
  const int live = w.hdr->live, moved = w.hdr->free_pages;
  const int64_t np = p.num_pages - p.first_page;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    counts[0] = live;
    counts[1] = moved;
  }
  for (int64_t m = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x; m < moved; m += (int64_t)gridDim.x * kCopyThreads)
    refs_out[w.list[m]] = w.mover_refs[m];
  for (int r = blockIdx.x; r < rows.num_rows; r += gridDim.x) {
    const int64_t held = rows.held[r], width = rows.table_stride;
    if ((held < 0 || held > width) && threadIdx.x == 0) set_error(status, PS_ERR_INVALID_ARG);
    // in place, what is past the held pages stays as it is
    const int64_t n = tables_out == rows.tables && held < width ? held : width;
    for (int64_t k = threadIdx.x; k < n; k += kCopyThreads) {
      int64_t id = rows.tables[r * rows.table_stride + k];
      if (k < held) {
        if (id < 0 || id >= p.num_pages) {
          set_error(status, PS_ERR_INVALID_ARG);
        } else if (id - p.first_page >= live && id - p.first_page < np) {
          const int m = w.inv[id - p.first_page];
          if (m >= 0) id = p.first_page + w.list[m];
          else set_error(status, PS_ERR_INVALID_ARG);  // a held page without a reference
        }
      }
      tables_out[r * rows.table_stride + k] = (int32_t)id;
    }
  }
  copy_pages(p, moved, [&](int64_t m, int64_t* s, int64_t* d) {
    *s = p.first_page + w.movers[m];
    *d = p.first_page + w.list[m];
    return true;
  });
}

}  // namespace

int32_t launch_copy(const Pool& p, int32_t n, const int32_t* src, const int32_t* dst, int32_t* status, int nsm,
                    cudaStream_t st) {
  const int64_t warps = (int64_t)n * 2 * p.num_layers * copy_parts(p, p.page_size), total = (warps + kCopyWarps - 1) / kCopyWarps;
  const int grid = (int)(total < (int64_t)nsm * 8 ? total : (int64_t)nsm * 8);
  return status_of(launch(k_page_copy, dim3((unsigned)grid), kCopyThreads, 0, st, p, src, dst, n, status));
}

int32_t launch_fork(const Pool& p, const PageScratch& w, int32_t n, const int32_t* parents, const int32_t* children,
                    const int32_t* room, const ps_kv_rows_t& rows, int32_t row_pages, const int32_t* refs_in,
                    int32_t* refs_out, int32_t* status, int nsm, cudaStream_t st) {
  ForkArgs a{};
  a.parents = parents; a.children = children; a.room = room;
  a.tables = rows.tables; a.lens = rows.lens; a.held = rows.held; a.table_stride = rows.table_stride;
  a.refs_in = refs_in; a.refs_out = refs_out; a.status = status;
  a.n = n; a.num_rows = rows.num_rows; a.row_pages = row_pages;
  cudaError_t e = launch(k_fork_scan, dim3((unsigned)(w.chunks + n)), kScanThreads, 0, st, p, w, a);
  if (e != cudaSuccess) return status_of(e);
  if (n == 0) return PS_OK;
  // enough CTAs for a few waves, at most a warp for each part of the copies
  const int most = (2 * p.num_layers * copy_parts(p, p.page_size) + kCopyWarps - 1) / kCopyWarps;
  int ny = 8 * nsm / n;
  ny = ny < 1 ? 1 : (ny > most ? most : ny);
  return status_of(launch(k_fork_apply, dim3((unsigned)n, (unsigned)ny), kCopyThreads, 0, st, p, w, a));
}

int32_t launch_release(const Pool& p, int32_t n, const int32_t* list, const ps_kv_rows_t& rows, int32_t row_pages,
                       int32_t* refs, int32_t* status, cudaStream_t st) {
  return status_of(launch(k_release, dim3((unsigned)n), kScanThreads, 0, st, p, list, rows, row_pages, refs, status));
}

int32_t launch_compact(const Pool& p, const PageScratch& w, const ps_kv_rows_t& rows, const int32_t* refs_in,
                       int32_t* tables_out, int32_t* refs_out, int32_t* counts,
                       int32_t* status, int nsm, cudaStream_t st) {
  cudaError_t e = launch(k_compact_count, dim3((unsigned)w.chunks), kScanThreads, 0, st, p, w, refs_in);
  if (e == cudaSuccess)
    e = launch(k_compact_lists, dim3((unsigned)w.chunks), kScanThreads, 0, st, p, w, refs_in, refs_out);
  if (e == cudaSuccess)
    e = launch(k_compact_move, dim3((unsigned)(nsm * 8)), kCopyThreads, 0, st, p, w, rows, tables_out,
               refs_out, counts, status);
  return status_of(e);
}

}  // namespace pskv
