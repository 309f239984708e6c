// ps_kv_reorder: the rows of a request's beams follow the beams that they continue.
//
// New row j takes over the pages and the length of old row q = parents[j].  Full
// pages are shared by all children of q; its last pages, from the partly filled
// one on, go to the first child, and the others copy that page's tokens to a page
// of their own.  With c children, a full page's references grow by c - 1, those of
// the last pages by 0, or by -1 where c = 0: no sum depends on an order, and a page
// that reaches 0 is free for this very call (nothing reads it any more).
//
// Three kernels: the first checks the rows, adds up the changes, one CTA for 256
// columns of a request's rows, and lists the copies; the second applies the changes to
// a copy of the references and lists the free pages, and its last CTA decides whether
// the call goes ahead; the third writes tables, lengths and references and copies the
// partial pages.  A column of the tables is read and rewritten by one thread, so the
// rows are permuted in place.
//
// Bound by latency: chains of dependent reads (parent, length, page, reference, change;
// free pages, their sums; new page, its tokens) in kernels that follow one another.
// Each reads what it can before it waits for the one before it.  One request of four
// beams takes 8 us; 64 of eight beams of 2048 tokens, whose copies are 21 MB (3.2 us),
// 15.8: 4.5 for the changes, 4.7 to the decision, 3 to 5 for the copies.
#include "ps_kv_pages.cuh"

namespace pskv {
namespace {

constexpr int kCols = kScanThreads;  // columns that a CTA takes at a time
constexpr int kColCtas = 64;         // CTAs of a request at most
constexpr int kAtOnce = 8;           // beams whose ids a thread reads together
constexpr int kNoPage = -1;
constexpr int kRoom = 3;             // CTAs of the last kernel on an SM

struct Args {
  const int32_t *rows, *parents;
  int32_t *tables, *lens, *held;
  int64_t stride;
  const int32_t* refs_in;
  int32_t* refs_out;
  int32_t* status;
  int32_t n, beams, grow, num_rows, row_pages, col_ctas;
};

// Of a request: col_ctas CTAs for the changes, and one for the rows.
__global__ void __launch_bounds__(kScanThreads) k_reorder_scan(Pool p, PageScratch w, ReorderScratch o, Args a) {
  __shared__ int s_row[PS_KV_MAX_BEAMS], s_parent[PS_KV_MAX_BEAMS], s_len[PS_KV_MAX_BEAMS], s_held[PS_KV_MAX_BEAMS];
  __shared__ int s_children[PS_KV_MAX_BEAMS];
  chain();
  const int B = a.beams, b = threadIdx.x, y = blockIdx.x % (a.col_ctas + 1);
  const int64_t i0 = (int64_t)(blockIdx.x / (a.col_ctas + 1)) * B;
  bool ok = true;
  if (b < B) {
    const int row = a.rows[i0 + b], parent = a.parents[i0 + b];
    int len = 0, held = 0;
    if (row >= 0 && row < a.num_rows) {
      len = a.lens[row];
      held = a.held[row];
    } else {
      ok = false;
    }
    if (parent < -1 || parent >= B || len < 0 || held < 0 || held > a.row_pages || len > (int64_t)held << p.page_log2) ok = false;
    s_row[b] = row;
    s_parent[b] = parent;
    s_len[b] = len;
    s_held[b] = held;
    s_children[b] = 0;
  }
  ok = __syncthreads_and(ok);
  if (ok && y < a.col_ctas) {
    if (b < B && s_parent[b] >= 0) atomicAdd(&s_children[s_parent[b]], 1);
    __syncthreads();
    int most = 0;
    for (int q = 0; q < B; ++q) most = max(most, s_held[q]);
    for (int k = y * kCols + threadIdx.x; k < most; k += a.col_ctas * kCols) {
      // neighbouring beams mostly hold the same page: their changes go together
      int64_t at = -1;
      int change = 0;
      for (int q0 = 0; q0 < B; q0 += kAtOnce) {
        int ids[kAtOnce], held[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const int q = q0 + u;
          ids[u] = q < B && k < s_held[q] ? a.tables[s_row[q] * a.stride + k] : kNoPage;
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {  // (a page that the beam before has, too, is looked at there)
          const int64_t id = ids[u];
          held[u] = 1;
          if (id >= p.first_page && id < p.num_pages && (u == 0 || ids[u] != ids[u ? u - 1 : 0])) held[u] = a.refs_in[id - p.first_page];
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const int64_t id = ids[u];
          const int q = q0 + u;
          if (ids[u] == kNoPage && (q >= B || k >= s_held[q])) continue;
          const int c = s_children[q], d = k < s_len[q] >> p.page_log2 ? c - 1 : (c > 0 ? 0 : -1);
          if (id < 0 || id >= p.num_pages || held[u] <= 0) {  // (looked at first: -1 may be a row's id, too)
            ok = false;
            continue;
          }
          if (id == at) {
            change += d;
            continue;
          }
          if (change != 0 && at >= p.first_page) atomicAdd(o.delta + (at - p.first_page), change);
          at = id;
          change = d;
        }
      }
      if (change != 0 && at >= p.first_page) atomicAdd(o.delta + (at - p.first_page), change);
    }
  } else if (y == a.col_ctas) {
    ReorderRec r{};
    int need = 0;
    if (ok && b < B) {
      const int q = s_parent[b];
      r.row = s_row[b];
      r.src = q;
      if (q >= 0) {
        bool heir = true;
        for (int j = 0; j < b; ++j) heir = heir && s_parent[j] != q;
        r.len = s_len[q];
        const int64_t total = ((int64_t)r.len + a.grow + p.page_size - 1) >> p.page_log2;
        r.have = heir ? s_held[q] : r.len >> p.page_log2;
        if (total > a.row_pages) ok = false;
        r.total = total > r.have ? (int)total : r.have;
        need = ok ? r.total - r.have : 0;
        r.part = heir ? 0 : r.len & (p.page_size - 1);
        r.from = r.part ? a.tables[s_row[q] * a.stride + r.have] : 0;
      }
      o.rec[i0 + b] = r;
    }
    if (b < B) w.need[i0 + b] = need;
    static_assert(PS_KV_MAX_BEAMS == 32, "a warp's");
    if (b < 32) {
      const unsigned m = __ballot_sync(0xFFFFFFFFu, r.part > 0);
      int to = 0;
      if (b == 0 && m) to = atomicAdd(&w.hdr->parts, __popc(m));
      to = __shfl_sync(0xFFFFFFFFu, to, 0) + __popc(m & ((1u << b) - 1));
      if (r.part > 0) o.copy[to] = (int)i0 + b;
    }
    // a row is named once
    for (int64_t j = threadIdx.x; j < a.n; j += kScanThreads) {
      const int row = a.rows[j];
      for (int q = 0; q < B; ++q)
        if (j != i0 + q && row == s_row[q]) ok = false;
    }
  }
  if (!ok) atomicMin(&w.hdr->refused, (int32_t)PS_ERR_INVALID_ARG);
}

// CTA c: chunk c of the references; the last one: the pages that the rows need.  The
// references are read before the wait for
// k_reorder_scan, which only reads them and lets this kernel start when all that came
// before it is done.  (Without requests there is no such kernel, and what came before
// may write them.)
__global__ void __launch_bounds__(kScanThreads) k_reorder_free(Pool p, PageScratch w, ReorderScratch o, Args a) {
  const int64_t np = p.num_pages - p.first_page;
  const int64_t c0 = (int64_t)blockIdx.x * w.chunk_size;
  const int64_t c1 = c0 + w.chunk_size < np ? c0 + w.chunk_size : np;
  const bool chunk = (int)blockIdx.x < w.chunks;
  int count = 0;
  bool ok = true;
  if (a.n == 0 || !chunk) chain();
  if (!chunk) {
    int64_t need = 0;
    for (int i0 = 0; i0 < a.n; i0 += kScanThreads) {
      const int i = i0 + threadIdx.x;
      int64_t tot;
      const int64_t e = block_scan<int64_t>(i < a.n ? __ldcg(w.need + i) : 0, &tot);
      const int64_t s = need + e;
      if (i < a.n) w.start[i] = s < 0x7FFFFFFF ? (int)s : 0x7FFFFFFF;
      need += tot;
    }
    if (threadIdx.x == 0) w.hdr->need = need < 0x7FFFFFFF ? (int)need : 0x7FFFFFFF;
  }
  for (int64_t i0 = c0; chunk && (i0 < c1 || i0 == c0); i0 += kTile) {
    int r[kEach], rank[kEach], tot;
    bool free[kEach];
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      const int64_t i = i0 + u * kScanThreads + threadIdx.x;
      r[u] = i < c1 ? __ldcg(a.refs_in + i) : 1;
    }
    if (i0 == c0 && a.n > 0) chain();
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      const int64_t i = i0 + u * kScanThreads + threadIdx.x;
      if (i < c1) r[u] += o.delta[i];
      free[u] = r[u] == 0;
      ok = ok && r[u] >= 0;
    }
    tile_ranks(free, rank, &tot);
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      const int64_t i = i0 + u * kScanThreads + threadIdx.x;
      if (i < c1) {
        o.delta[i] = 0;
        o.refs[i] = r[u];
      }
      if (free[u]) w.list[c0 + count + rank[u]] = (int32_t)i;
    }
    count += tot;
  }
  if (threadIdx.x == 0 && chunk) w.chunk_cnt[blockIdx.x] = count;
  if (!ok) atomicMin(&w.hdr->refused, (int32_t)PS_ERR_INVALID_ARG);
  if (!last_cta(&w.hdr->done)) return;
  const int refused = __ldcg(&w.hdr->refused), need = __ldcg(&w.hdr->need), copies = __ldcg(&w.hdr->parts);
  const int free_pages = scan_array(w.chunk_cnt, w.chunk_base, w.chunks);
  if (threadIdx.x == 0) {
    const int st = refused ? refused : (need > free_pages ? PS_ERR_CAPACITY : PS_OK);
    w.hdr->refused = w.hdr->parts = 0;
    w.hdr->status = st;
    w.hdr->copies = copies;
    w.hdr->free_pages = st == PS_OK ? need : 0;  // taken
    if (st != PS_OK) set_error(a.status, st);
  }
}

// A record, not from the SM's own cache: it is read before the wait.
__device__ __forceinline__ ReorderRec record(const ReorderScratch& o, int64_t i) {
  const int4 a = __ldcg(reinterpret_cast<const int4*>(o.rec + i)), b = __ldcg(reinterpret_cast<const int4*>(o.rec + i) + 1);
  return {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
}

// CTAs, in order: a chunk of the references each; 256 columns of a request's rows;
// the copies, warp by warp.  What k_reorder_scan wrote, and the tables, are read before
// the wait for k_reorder_free, which lets this kernel start when that one is done.
__global__ void __launch_bounds__(kScanThreads) k_reorder_apply(Pool p, PageScratch w, ReorderScratch o, Args a) {
  __shared__ int base[kMaxChunks];
  __shared__ ReorderRec s_rec[PS_KV_MAX_BEAMS];
  __shared__ int s_start[PS_KV_MAX_BEAMS];
  extern __shared__ int ids[][kCols];  // [beams]; no more, so that an SM has room for 8 CTAs of few beams
  const int B = a.beams, requests = a.n / B, tables = requests * a.col_ctas;
  int cta = blockIdx.x;
  if (cta < w.chunks) {
    chain();
    const int st = __ldcg(&w.hdr->status);
    const int64_t np = p.num_pages - p.first_page, c0 = (int64_t)cta * w.chunk_size;
    const int64_t c1 = c0 + w.chunk_size < np ? c0 + w.chunk_size : np;
    if (st != PS_OK) {
      if (a.refs_out != a.refs_in)
        for (int64_t i = c0 + threadIdx.x; i < c1; i += kScanThreads) a.refs_out[i] = a.refs_in[i];
      return;
    }
#pragma unroll 8
    for (int64_t i = c0 + threadIdx.x; i < c1; i += kScanThreads) a.refs_out[i] = o.refs[i];
    __syncthreads();
    const int before = w.chunk_base[cta], taken = min(w.hdr->free_pages - before, w.chunk_cnt[cta]);
    for (int j = threadIdx.x; j < taken; j += kScanThreads) a.refs_out[w.list[c0 + j]] = 1;
    return;
  }
  cta -= w.chunks;
  if (cta < tables) {
    const int r = cta / a.col_ctas, y = cta % a.col_ctas, b = threadIdx.x;
    if (b < B) s_rec[b] = record(o, (int64_t)r * B + b);
    __syncthreads();
    int most = 0;
    bool sane = true;  // (after a refusal the records may be anything)
    for (int j = 0; j < B; ++j) {
      most = max(most, s_rec[j].total);
      sane = sane && s_rec[j].row >= 0 && s_rec[j].row < a.num_rows;
    }
    if (most > a.row_pages || !sane) most = 0;
    int k = y * kCols + threadIdx.x;
    auto read = [&]() {
      for (int j0 = 0; j0 < B; j0 += kAtOnce) {
        int id[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
          if (j0 + u < B) id[u] = __ldcg(a.tables + s_rec[j0 + u].row * a.stride + k);
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
          if (j0 + u < B) ids[j0 + u][threadIdx.x] = id[u];
      }
    };
    if (k < most) read();
    chain();
    const int status = __ldcg(&w.hdr->status);
    for (int c = threadIdx.x; c < w.chunks; c += kScanThreads) base[c] = w.chunk_base[c];
    if (b < B) s_start[b] = __ldcg(w.start + (int64_t)r * B + b);
    if (status != PS_OK) return;
    __syncthreads();
    for (; k < most; k += a.col_ctas * kCols) {
      if (k >= a.col_ctas * kCols) read();
      for (int j = 0; j < B; ++j) {
        const ReorderRec& x = s_rec[j];
        if (k >= x.total) continue;
        const int old = ids[j][threadIdx.x];
        const int id = k < x.have ? ids[x.src][threadIdx.x] : (int)(p.first_page + free_page(w, base, s_start[j] + (k - x.have)));
        if (id != old) a.tables[x.row * a.stride + k] = id;
      }
    }
    if (y == 0 && b < B) {
      a.lens[s_rec[b].row] = s_rec[b].len;
      a.held[s_rec[b].row] = s_rec[b].total;
    }
    return;
  }
  cta -= tables;
  const int parts = copy_parts(p, p.page_size), slices = 2 * p.num_layers;
  const int64_t step = ((int64_t)gridDim.x - w.chunks - tables) * kCopyWarps;
  int64_t u = (int64_t)cta * kCopyWarps + (threadIdx.x >> 5);
  auto row = [&]() {  // of unit u; where there are fewer, any row's
    const int64_t c = u / (slices * parts);
    const int i = c < a.n ? __ldcg(o.copy + c) : 0;
    return i >= 0 && i < a.n ? i : 0;
  };
  int i = row();
  ReorderRec x = record(o, i);
  chain();
  // all that the first copy needs side by side
  const int status = __ldcg(&w.hdr->status), copies = __ldcg(&w.hdr->copies);
  int start = __ldcg(w.start + i);
  for (int c = threadIdx.x; c < w.chunks; c += kScanThreads) base[c] = w.chunk_base[c];
  if (status != PS_OK) return;
  const int64_t units = (int64_t)copies * slices * parts;
  if ((int64_t)cta * kCopyWarps >= units) return;
  __syncthreads();
  while (u < units) {
    const int rest = (int)(u % (slices * parts));
    const int64_t to = p.first_page + free_page(w, base, start);
    copy_part(p, x.from, to, rest / parts, x.part, rest % parts, threadIdx.x & 31);
    u += step;
    if (u >= units) break;
    i = row();
    x = record(o, i);
    start = __ldcg(w.start + i);
  }
}

}  // namespace

int32_t launch_reorder(const Pool& p, const PageScratch& w, const ReorderScratch& o, int32_t requests, int32_t beams, const int32_t* list,
                       const int32_t* parents, int32_t grow, const ps_kv_rows_t& rows, int32_t row_pages,
                       const int32_t* refs_in, int32_t* refs_out, int32_t* status, int nsm, cudaStream_t st) {
  Args a{};
  a.rows = list; a.parents = parents;
  a.tables = rows.tables; a.lens = rows.lens; a.held = rows.held; a.stride = rows.table_stride;
  a.refs_in = refs_in; a.refs_out = refs_out; a.status = status;
  a.n = requests * beams; a.beams = beams; a.grow = grow; a.num_rows = rows.num_rows; a.row_pages = row_pages;
  a.col_ctas = (row_pages + kCols - 1) / kCols;
  if (a.col_ctas > kColCtas) a.col_ctas = kColCtas;
  cudaError_t e = cudaSuccess;
  if (requests > 0) e = launch(k_reorder_scan, dim3((unsigned)(requests * (a.col_ctas + 1))), kScanThreads, 0, st, p, w, o, a);
  if (e == cudaSuccess) e = launch(k_reorder_free, dim3((unsigned)w.chunks + 1), kScanThreads, 0, st, p, w, o, a);
  if (e != cudaSuccess) return status_of(e);
  const int64_t units = (int64_t)a.n * 2 * p.num_layers * copy_parts(p, p.page_size);
  // of the copies as many as an SM has room for with the others, three CTAs in all
  const int64_t others = w.chunks + (int64_t)requests * a.col_ctas, room = (int64_t)nsm * kRoom - others;
  const int64_t want = (units + kCopyWarps - 1) / kCopyWarps, most = room > nsm ? room : nsm;
  const int64_t grid = others + (want < most ? want : most);
  return status_of(launch(k_reorder_apply, dim3((unsigned)grid), kScanThreads, (size_t)beams * kCols * 4, st, p, w, o, a));
}

}  // namespace pskv
