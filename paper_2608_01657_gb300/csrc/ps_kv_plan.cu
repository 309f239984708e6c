// ps_kv_plan: shared prefixes, tiles and the division of a batch's attention
// into equal parts (see ps_kv.cuh for the plan's shape).  Three kernels bound by
// the latency of their dependent reads and scans: 16 us for one request, 20 for
// 256 in 32 groups, 22 for eight prompts, about half of it k_plan_tiles, one CTA;
// once a step, for all of its layers.
#include "ps_kv.cuh"

namespace pskv {
namespace {

constexpr int kReqThreads = 128;
constexpr int kPlanThreads = 1024;
constexpr int kAnyPages = 0x7FFFFFFF;

// Cycles of one unit as the division weighs them: a wide one on its SM (128
// keys; 2800 measured for prompts, 3900 beside narrow tiles, up to 5900 where a
// tile has one or two units), a narrow one in its warp (16 keys).  Both are those
// of heads of 128 elements and are used for all, so the division of the SMs does
// not follow the head's size.  Measured over 4000 to 7800 and 1900 to 3400: 256
// tenants' decode 366 to 420 us (371 as it stands), 128 requests on one prefix 75
// to 88 (76).
constexpr double kWideCycles = 5250, kNarrowCycles = 2400;
// A narrow worker has at least so many units: more workers would cost the join
// more than they save (one request of 700 keys, 8 heads: 10.6 us a call with 2,
// 9.9 with 4, 10.9 with 5, 12.0 with 8; 33 requests of up to 7 tokens 17.2 and 16.8).
constexpr int kLeastUnits = 4;

// Pages of a request that every one of its queries sees whole.
__device__ __forceinline__ int whole_pages(const Pool& p, const Batch& b, int r) {
  const int n = b.q_offsets[r + 1] - b.q_offsets[r], len = b.kv_lens[r];
  const int seen = b.causal ? len - n : len;
  return seen > 0 ? seen >> p.page_log2 : 0;
}

// One CTA a request: its offsets, length and page ids are in range; the leading
// pages that it has in common with its group's first request; its tokens' map.
__global__ void __launch_bounds__(kReqThreads) k_plan_requests(Pool p, Plan plan, Batch b) {
  chain();
  const int r = blockIdx.x;
  const int q0 = b.q_offsets[r], q1 = b.q_offsets[r + 1], len = b.kv_lens[r];
  bool ok = q0 >= 0 && q1 >= q0 && q1 <= b.num_tokens && len >= 0 && len <= (int64_t)b.row_pages << p.page_log2;
  if (r == 0) ok = ok && q0 == 0;
  if (r == b.num_requests - 1) ok = ok && q1 == b.num_tokens;
  const bool sane = ok;
  const int32_t* row = b.tables + r * b.table_stride;
  int common = kAnyPages;
  if (sane) {
    const int pages = (int)(((int64_t)len + p.page_size - 1) >> p.page_log2);
    for (int k = threadIdx.x; k < pages; k += kReqThreads) {
      const int id = row[k];
      if (id < 0 || id >= p.num_pages) ok = false;
    }
    for (int t = q0 + threadIdx.x; t < q1; t += kReqThreads) plan.tok_req[t] = r;
    // the group that holds r: the last one that starts at or before it
    int lo = 0, hi = b.group_offsets ? b.num_groups - 1 : 0;
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (b.group_offsets[mid] <= r) lo = mid;
      else hi = mid - 1;
    }
    if (threadIdx.x == 0) plan.group[r] = lo;
    if (b.group_offsets && q1 > q0) {
      const int first = b.group_offsets[lo];
      common = 0;
      if (first >= 0 && first <= r) {
        const int f0 = b.kv_lens[first], w = whole_pages(p, b, r);
        if (f0 >= 0 && f0 <= (int64_t)b.row_pages << p.page_log2) {
          const int wf = whole_pages(p, b, first);
          common = w < wf ? w : wf;
          const int32_t* lead = b.tables + first * b.table_stride;
          // wf may be out of range where the first request's offsets are: bounded by its length's pages
          const int most = (int)((int64_t)f0 >> p.page_log2);
          common = common < most ? common : most;
          if (first != r)
            for (int k = threadIdx.x; k < common; k += kReqThreads)
              if (row[k] != lead[k]) {
                common = k;
                break;
              }
        }
      }
    }
  }
  __shared__ int s_common;
  if (threadIdx.x == 0) s_common = kAnyPages;
  __syncthreads();
  atomicMin(&s_common, common);
  ok = __syncthreads_and(ok);
  if (threadIdx.x == 0) {
    plan.common[r] = s_common;
    plan.bad[r] = !ok;
  }
}

// Exclusive scan of one 64-bit value a thread over the CTA.
__device__ int64_t scan64(int64_t v, int64_t* total) {
  __shared__ int64_t wsum[kPlanThreads / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t x = __shfl_up_sync(0xFFFFFFFFu, incl, o);
    if (lane >= o) incl += x;
  }
  if (lane == 31) wsum[warp] = incl;
  __syncthreads();
  if (warp == 0) {
    int64_t w = wsum[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t x = __shfl_up_sync(0xFFFFFFFFu, w, o);
      if (lane >= o) w += x;
    }
    wsum[lane] = w;
  }
  __syncthreads();
  const int64_t base = warp ? wsum[warp - 1] : 0;
  *total = wsum[kPlanThreads / 32 - 1];
  __syncthreads();
  return base + incl - v;
}

// The rows of one item (a group's shared prefix, or a request's own keys).
struct Item {
  int tok0, rows, kv0, kv1, req, ctx, list;
  bool shared;
};
__device__ __forceinline__ int tile_end(const Item& it, const Pool& p, int last_row) {
  // keys past the last row's bound are never seen
  const int64_t bound = (int64_t)it.ctx + 1 + last_row / p.ratio;
  return bound < it.kv1 ? (int)(bound > it.kv0 ? bound : it.kv0) : it.kv1;
}
__device__ __forceinline__ int unit_count(int keys, int unit) { return keys > 0 ? (keys + unit - 1) / unit : 1; }


__global__ void __launch_bounds__(kPlanThreads) k_plan_tiles(Pool p, Plan plan, Batch b, int32_t* status) {
  chain();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int bad = 0;
  for (int r = tid; r < b.num_requests; r += kPlanThreads) bad |= plan.bad[r];
  if (b.group_offsets) {
    for (int g = tid; g < b.num_groups; g += kPlanThreads) bad |= b.group_offsets[g] > b.group_offsets[g + 1];
    if (tid == 0) bad |= b.group_offsets[0] != 0 || b.group_offsets[b.num_groups] != b.num_requests;
  }
  if (__syncthreads_or(bad)) {
    if (tid == 0) {
      PlanHdr h{};
      h.status = PS_ERR_INVALID_ARG;
      *plan.hdr = h;
      set_error(status, PS_ERR_INVALID_ARG);
    }
    return;
  }
  // the groups' shared tokens, kept in common[] for each member (0: none)
  if (b.group_offsets) {
    for (int g = warp; g < b.num_groups; g += kPlanThreads / 32) {
      const int r0 = b.group_offsets[g], r1 = b.group_offsets[g + 1];
      int common = kAnyPages, members = 0, most = 0;
      for (int r = r0 + lane; r < r1; r += 32) {
        const int n = b.q_offsets[r + 1] - b.q_offsets[r];
        if (n == 0) continue;
        common = min(common, plan.common[r]);
        members += 1;
        most = max(most, n);
      }
      common = __reduce_min_sync(0xFFFFFFFFu, common);
      members = __reduce_add_sync(0xFFFFFFFFu, members);
      most = __reduce_max_sync(0xFFFFFFFFu, most);
      const bool share = members > 1 && (int64_t)most * p.ratio <= kShareRows &&
                         ((int64_t)common << p.page_log2) >= kShareTokens;
      for (int r = r0 + lane; r < r1; r += 32) plan.common[r] = share ? common << p.page_log2 : 0;
    }
  } else {
    for (int r = tid; r < b.num_requests; r += kPlanThreads) plan.common[r] = 0;
  }
  __syncthreads();
  // items: the groups' prefixes, then the requests
  const int ngroups = b.group_offsets ? b.num_groups : 0;
  const int nitems = ngroups + b.num_requests;
  int64_t tiles[kLists] = {}, units[kLists] = {}, shared[kLists] = {};  // units: their cost
  for (int i0 = 0; i0 < nitems; i0 += kPlanThreads) {
    const int i = i0 + tid;
    Item it{};
    if (i < ngroups) {
      const int r0 = b.group_offsets[i], r1 = b.group_offsets[i + 1];
      if (r1 > r0 && plan.common[r0] > 0) {
        it.tok0 = b.q_offsets[r0];
        it.rows = (b.q_offsets[r1] - it.tok0) * p.ratio;
        it.kv1 = plan.common[r0];
        it.req = r0;
        it.ctx = kNoMask;
        it.shared = true;
      }
    } else if (i < nitems) {
      const int r = i - ngroups, n = b.q_offsets[r + 1] - b.q_offsets[r];
      it.tok0 = b.q_offsets[r];
      it.rows = n * p.ratio;
      it.kv0 = plan.common[r];
      it.kv1 = b.kv_lens[r];
      it.req = r;
      it.ctx = b.causal ? b.kv_lens[r] - n : kNoMask;
      it.shared = plan.common[r] > 0;
    }
    it.list = list_of(it.rows);
    const int H = tile_rows(it.list), unit = unit_keys(it.list);
    const int nt = (it.rows + H - 1) / H;
    int64_t nu = 0;
    for (int t = 0; t < nt; ++t) {
      const int last = min(it.rows, (t + 1) * H) - 1;
      nu += unit_count(tile_end(it, p, last) - it.kv0, unit) + tile_cost(it.list);
    }
    int64_t tile_at = 0, unit_at = 0, shared_at = 0;
    for (int l = 0; l < kLists; ++l) {
      int64_t tot;
      const bool mine = it.list == l;
      int64_t e = scan64(mine ? nt : 0, &tot);
      if (mine) tile_at = tiles[l] + e;
      tiles[l] += tot;
      e = scan64(mine ? nu * p.kv_heads : 0, &tot);
      if (mine) unit_at = units[l] + e;
      units[l] += tot;
      e = scan64(mine && it.shared ? (int64_t)it.rows * p.kv_heads : 0, &tot);
      if (mine) shared_at = shared[l] + e;
      shared[l] += tot;
    }
    for (int t = 0; t < nt; ++t) {
      const int last = min(it.rows, (t + 1) * H) - 1;
      Tile x;
      x.tok0 = it.tok0;
      x.row0 = t * H;
      x.nrows = last + 1 - t * H;
      x.kv0 = it.kv0;
      x.kv1 = tile_end(it, p, last);
      x.req = it.req;
      x.ctx = it.ctx;
      x.sidx = it.shared ? (int)shared_at + t * H * p.kv_heads : -1;
      plan.tiles[it.list][tile_at + t] = x;
      plan.ucum[it.list][tile_at + t] = unit_at;
      unit_at += (int64_t)(unit_count(x.kv1 - x.kv0, unit) + tile_cost(it.list)) * p.kv_heads;
    }
    if (i < ngroups) {
      plan.grp_tile[i] = it.rows > 0 ? (int)tile_at : -1;
      plan.grp_list[i] = it.list;
    } else if (i < nitems) {
      ReqRec q{};
      q.tile0 = (int)tile_at;
      q.list = it.list;
      q.ptile0 = -1;
      plan.req[i - ngroups] = q;
    }
  }
  __syncthreads();
  if (b.group_offsets) {  // the requests' places in their groups' prefix tiles
    for (int r = tid; r < b.num_requests; r += kPlanThreads) {
      const int g = plan.group[r];
      plan.req[r].ptile0 = plan.grp_tile[g];
      plan.req[r].plist = plan.grp_list[g];
      plan.req[r].prow0 = (b.q_offsets[r] - b.q_offsets[b.group_offsets[g]]) * p.ratio;
    }
  }
  // SMs for the wide tiles, the rest for the narrow ones, so that both lists end
  // together: thread x weighs x SMs.
  __shared__ unsigned long long s_best;
  if (tid == 0) s_best = ~0ull;
  __syncthreads();
  const int sms = plan.max_workers[1], per_sm = plan.max_workers[0] / sms;
  if (tid <= sms) {
    const bool can = (tid > 0 || units[1] == 0) && (tid < sms || units[0] == 0);
    const double wide = units[1] > 0 && tid > 0 ? (double)units[1] * kWideCycles / tid : 0;
    const double narrow = units[0] > 0 && tid < sms ? (double)units[0] * kNarrowCycles / (per_sm * (sms - tid)) : 0;
    if (can) atomicMin(&s_best, (unsigned long long)fmax(wide, narrow) << 10 | tid);
  }
  __syncthreads();
  const int wide_sms = (int)(s_best & 1023);
  const int64_t room[kLists] = {(int64_t)per_sm * (sms - wide_sms), wide_sms};
  int workers[kLists];
  for (int l = 0; l < kLists; ++l) {
    const int64_t want = l ? units[l] : (units[l] + kLeastUnits - 1) / kLeastUnits;
    workers[l] = (int)(want < room[l] ? want : room[l]);
    if (tid == 0) plan.ucum[l][tiles[l]] = units[l];
  }
  __syncthreads();
  for (int l = 0; l < kLists; ++l) {
    for (int c = tid; c < workers[l]; c += kPlanThreads) {
      const int64_t u = units[l] * c / workers[l];
      int lo = 0, hi = (int)tiles[l] - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (plan.ucum[l][mid] <= u) lo = mid;
        else hi = mid - 1;
      }
      plan.first_tile[l][c] = lo;
    }
  }
  if (tid == 0) {
    PlanHdr h{};
    h.status = PS_OK;
    h.narrow_ctas = (int)room[0] / kNarrowWarps;
    for (int l = 0; l < kLists; ++l) {
      h.ntiles[l] = (int)tiles[l];
      h.workers[l] = workers[l];
      h.cost[l] = units[l];
    }
    *plan.hdr = h;
  }
}

// The partial results of a (tile, head).
template <int H>
__device__ __forceinline__ Parts4 parts_of(const Plan& plan, const Pool& p, const PlanHdr& h, int list, int tile, int head) {
  const int64_t U = h.cost[list], b = plan.ucum[list][tile];
  const int C = h.workers[list];
  const int64_t each = (plan.ucum[list][tile + 1] - b) / p.kv_heads;
  const int64_t ua = b + head * each + tile_cost(list);  // the place of unit 0
  const int ca = worker_of(ua, U, C), cb = worker_of(b + (head + 1) * each - 1, U, C);
  const Tile& t = plan.tiles[list][tile];
  Parts4 r;
  r.count = t.sidx < 0 && ca == cb ? 0 : cb - ca + 1;  // a whole one is written where it is computed
  r.first = (int)part_row<H>(t.sidx, t.nrows, head, ca, false, C);  // worker ca begins the (tile, head): unit 0 is its
  r.second = (int)part_row<H>(t.sidx, t.nrows, head, ca + 1, true, C);
  r.stride = t.sidx < 0 ? 2 * H : H;
  return r;
}
__device__ __forceinline__ Parts4 parts_of(const Plan& plan, const Pool& p, const PlanHdr& h, int list, int tile, int head) {
  return list ? parts_of<tile_rows(1)>(plan, p, h, 1, tile, head) : parts_of<tile_rows(0)>(plan, p, h, 0, tile, head);
}

// One CTA a request: the (tile, head)s whose rows have partial results (and the
// bytes of mend[] cleared).  It lets the next kernel start only when the tiles
// above are written, so that an attention kernel may read them before it waits.
// Their
// order is left to the counter: each is joined by itself.
__global__ void __launch_bounds__(kReqThreads) k_plan_joins(Pool p, Plan plan, Batch b) {
  chain();
  const PlanHdr h = *plan.hdr;
  if (h.status != PS_OK) return;
  const ReqRec rec = plan.req[blockIdx.x];
  const int H = tile_rows(rec.list);
  const int rows = (b.q_offsets[blockIdx.x + 1] - b.q_offsets[blockIdx.x]) * p.ratio;
  const int n = (rows + H - 1) / H * p.kv_heads;
  for (int i = threadIdx.x; i < n; i += kReqThreads) {
    const int tile = rec.tile0 + i / p.kv_heads, head = i % p.kv_heads;
    plan.mend[rec.list][(int64_t)tile * p.kv_heads + head] = 0;
    JoinRec j{};
    j.own = parts_of(plan, p, h, rec.list, tile, head);
    if (j.own.count == 0) continue;
    const Tile& t = plan.tiles[rec.list][tile];
    j.tok0 = t.tok0;
    j.row0 = t.row0;
    j.nrows = t.nrows;
    j.head = head;
    j.plist = -1;
    if (rec.ptile0 >= 0) {
      const int PH = tile_rows(rec.plist), prow = rec.prow0 + t.row0, pt = rec.ptile0 + prow / PH;
      j.plist = rec.plist;
      j.pofs = prow % PH;
      j.psplit = PH - j.pofs;
      j.pa = parts_of(plan, p, h, rec.plist, pt, head);
      if (j.psplit < t.nrows) j.pb = parts_of(plan, p, h, rec.plist, pt + 1, head);
    }
    plan.joins[rec.list][atomicAdd(&plan.hdr->joins[rec.list], 1)] = j;
  }
}

}  // namespace

int32_t launch_plan(const Pool& p, const Plan& plan, const Batch& b, int32_t* status, cudaStream_t st) {
  if (b.num_requests > 0) {
    const cudaError_t e = launch(k_plan_requests, dim3((unsigned)b.num_requests), kReqThreads, 0, st, p, plan, b);
    if (e != cudaSuccess) return status_of(e);
  }
  cudaError_t e = launch(k_plan_tiles, dim3(1), kPlanThreads, 0, st, p, plan, b, status);
  if (e == cudaSuccess && b.num_requests > 0)
    e = launch(k_plan_joins, dim3((unsigned)b.num_requests), kReqThreads, 0, st, p, plan, b);
  return status_of(e);
}

}  // namespace pskv
