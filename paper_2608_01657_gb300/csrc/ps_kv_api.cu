// C ABI of the operators on KV pages (declared in include/prefixshield_kv.h).
//
// Host side only: argument checks, the workspace layout and the handle.
#include <new>

#include "ps_kv.cuh"
#include "ps_kv_overlap.cuh"

using namespace pskv;

struct ps_kv {
  Pool pool;
  PoolMaps* maps = nullptr;  // [layers]
  Plan plan;
  PageScratch pages;
  LayoutScratch layout;
  ReorderScratch reorder;
  Batch batch;
  bool planned;
  int32_t turn;  // of the next attention, 0 or 1
  int32_t dev, nsm, max_requests, max_tokens, max_row_pages;
};

namespace {

inline cudaStream_t as_stream(void* s) { return static_cast<cudaStream_t>(s); }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
inline HeadRuns runs(const void* p, const int64_t stride[2], int64_t heads) { return {p, stride[0], stride[1], heads}; }
inline bool good_strides(const int64_t s[2]) { return s[0] >= 0 && s[1] >= 0 && s[0] % 8 == 0 && s[1] % 8 == 0; }

bool check_config(const ps_kv_config_t* c) {
  if (!c || !c->k || !c->v || !aligned16(c->k) || !aligned16(c->v)) return false;
  if (c->num_pages < 1 || c->num_pages > (1ll << 30) || c->first_page < 0) return false;
  const int32_t ps = c->page_size;
  if (ps != 2 && ps != 4 && ps != 8 && ps != 16 && ps != 32 && ps != 64) return false;
  for (int64_t s : {c->layer_stride, c->page_stride, c->token_stride, c->head_stride})
    if (s < 0 || s % 8 != 0) return false;
  if (c->num_layers < 1 || c->num_kv_heads < 1 || c->num_q_heads < c->num_kv_heads ||
      c->num_q_heads > PS_KV_MAX_HEADS || c->num_q_heads % c->num_kv_heads != 0)
    return false;
  if (c->head_dim < 8 || c->head_dim > PS_KV_MAX_HEAD_DIM || c->head_dim % 8 != 0) return false;
  // an axis of several places steps over a head's elements at least, or elements share addresses
  const struct { int64_t places, stride; } axes[] = {{c->num_layers, c->layer_stride}, {c->num_pages, c->page_stride},
                                                     {ps, c->token_stride}, {c->num_kv_heads, c->head_stride}};
  for (const auto& x : axes)
    if (x.places > 1 && x.stride < c->head_dim) return false;
  if (c->dtype != PS_KV_BF16 && c->dtype != PS_KV_F16) return false;
  if (c->max_requests < 1 || c->max_requests > PS_MAX_REQUESTS_PER_STEP) return false;
  if (c->max_tokens < 1 || c->max_tokens > (1 << 22) || (int64_t)c->max_tokens * c->num_q_heads >= (1ll << 30))
    return false;
  if (c->max_row_pages < 1 || (int64_t)c->max_row_pages * ps >= (1ll << 30)) return false;
  return true;
}

Pool make_pool(const ps_kv_config_t& c) {
  Pool p{};
  p.k = static_cast<char*>(c.k);
  p.v = static_cast<char*>(c.v);
  p.num_pages = c.num_pages;
  p.first_page = c.first_page < c.num_pages ? c.first_page : c.num_pages;  // no private pages past the end
  p.layer_stride = c.layer_stride; p.page_stride = c.page_stride;
  p.token_stride = c.token_stride; p.head_stride = c.head_stride;
  p.num_layers = c.num_layers; p.page_size = c.page_size;
  while ((1 << p.page_log2) < c.page_size) ++p.page_log2;
  p.kv_heads = c.num_kv_heads; p.q_heads = c.num_q_heads; p.ratio = c.num_q_heads / c.num_kv_heads;
  p.head_dim = c.head_dim; p.dtype = c.dtype;
  return p;
}

struct Carver {
  char* base;
  size_t off = 0;
  template <typename T>
  T* take(size_t count) {
    off = (off + 255) / 256 * 256;
    T* p = base ? reinterpret_cast<T*>(base + off) : nullptr;
    off += sizeof(T) * (count ? count : 1);
    return p;
  }
};

// The workspace: sizes with base == nullptr, pointers otherwise.  Every region
// starts on a 256-byte boundary.  The page header comes first (cleared once).
size_t carve(const ps_kv_config_t& c, const int32_t workers[kLists], char* base, Plan* plan, PageScratch* pages,
             LayoutScratch* layout, ReorderScratch* reorder) {
  Carver cv{base};
  const int64_t R = c.max_requests, T = c.max_tokens, ratio = c.num_q_heads / c.num_kv_heads;
  PageScratch w{};
  w.hdr = cv.take<PageHdr>(1);
  const int64_t np = c.first_page < c.num_pages ? c.num_pages - c.first_page : 0;
  // chunks of at least 2048 references, at most kMaxChunks of them
  int64_t chunk = (np + kMaxChunks - 1) / kMaxChunks;
  chunk = chunk < 2048 ? 2048 : (chunk + kScanThreads - 1) / kScanThreads * kScanThreads;
  w.chunk_size = (int32_t)chunk;
  w.chunks = (int32_t)((np + chunk - 1) / chunk);
  if (w.chunks < 1) w.chunks = 1;
  w.chunk_cnt = cv.take<int32_t>(w.chunks);
  w.chunk_base = cv.take<int32_t>(w.chunks);
  w.list = cv.take<int32_t>((size_t)w.chunks * chunk);
  w.movers = cv.take<int32_t>((size_t)np);
  w.inv = cv.take<int32_t>((size_t)np);
  w.mover_refs = cv.take<int32_t>((size_t)np);
  w.need = cv.take<int32_t>((size_t)R);
  w.start = cv.take<int32_t>((size_t)R);
  w.bad = cv.take<int32_t>((size_t)R);
  Plan p{};
  p.hdr = cv.take<PlanHdr>(1);
  p.req = cv.take<ReqRec>((size_t)R);
  p.tok_req = cv.take<int32_t>((size_t)T);
  p.group = cv.take<int32_t>((size_t)R);
  p.grp_tile = cv.take<int32_t>((size_t)R);
  p.grp_list = cv.take<int32_t>((size_t)R);
  p.common = cv.take<int32_t>((size_t)R);
  p.bad = cv.take<int32_t>((size_t)R);
  for (int l = 0; l < kLists; ++l) {
    const PlanBounds b = plan_bounds(l, R, T * ratio);
    const int64_t shared = b.shared * c.num_kv_heads;
    p.max_workers[l] = workers[l];
    const size_t part_rows = (size_t)(3 * (int64_t)workers[l] * tile_rows(l) + shared);
    p.tiles[l] = cv.take<Tile>((size_t)b.tiles);
    p.ucum[l] = cv.take<int64_t>((size_t)b.tiles + 1);
    p.first_tile[l] = cv.take<int32_t>((size_t)workers[l]);
    p.joins[l] = cv.take<JoinRec>((size_t)b.own_tiles * c.num_kv_heads);
    p.mend[l] = cv.take<uint8_t>((size_t)b.tiles * c.num_kv_heads);
    p.part_o[l] = cv.take<float4>((part_rows + 7) / 8 * 8 * (c.head_dim / 4));
    p.part_ml[l] = cv.take<float2>(part_rows);
  }
  LayoutScratch y{};
  const size_t parts = ((size_t)R + kLayoutPart - 1) / kLayoutPart;
  y.offset = w.start;
  y.group = w.need;
  y.done = &w.hdr->done;
  y.item = cv.take<int4>((size_t)R);
  y.total = cv.take<int64_t>(parts);
  y.groups = cv.take<int32_t>(parts);
  y.base = cv.take<int32_t>(parts + 1);
  y.group_base = cv.take<int32_t>(parts + 1);
  if (layout) *layout = y;
  ReorderScratch o{};
  o.rec = cv.take<ReorderRec>((size_t)R);
  o.copy = cv.take<int32_t>((size_t)R);
  o.delta = cv.take<int32_t>((size_t)np);
  o.refs = w.inv;
  if (reorder) *reorder = o;
  if (plan) *plan = p;
  if (pages) *pages = w;
  return (cv.off + 255) / 256 * 256;
}

// The workspace has the same size wherever it is asked for: the worker counts are
// bounded by the device's at ps_kv_create().
constexpr int32_t kSizedWorkers[kLists] = {kMaxSms * 4 * kNarrowWarps, kMaxSms};

// References to private pages: none are needed, and an empty array may have no address, where there are no such pages.
bool refs_ok(const ps_kv* kv, const int32_t* in, const int32_t* out) {
  return (in && out) || kv->pool.first_page == kv->pool.num_pages;
}
// Do two arrays of n int32 overlap without being the same one?
bool partly_same(const int32_t* a, const int32_t* b, int64_t n) {
  const int64_t d = ((intptr_t)a - (intptr_t)b) / 4;
  return a != b && d < n && d > -n;
}
bool rows_ok(const ps_kv* kv, const ps_kv_rows_t* r) {
  return r && r->tables && r->lens && r->held && r->num_rows >= 1 && r->table_stride >= 1;
}
int32_t row_pages(const ps_kv* kv, int64_t stride) {
  return stride < kv->max_row_pages ? (int32_t)stride : kv->max_row_pages;
}

}  // namespace

extern "C" {

size_t ps_kv_workspace_bytes(const ps_kv_config_t* cfg) {
  return check_config(cfg) ? carve(*cfg, kSizedWorkers, nullptr, nullptr, nullptr, nullptr, nullptr) : 0;
}

int32_t ps_kv_create(ps_kv_t** out, const ps_kv_config_t* cfg, void* d_workspace, size_t workspace_bytes,
                     void* stream) {
  if (!out || !check_config(cfg) || !d_workspace || (reinterpret_cast<uintptr_t>(d_workspace) & 255) != 0 ||
      workspace_bytes < carve(*cfg, kSizedWorkers, nullptr, nullptr, nullptr, nullptr, nullptr))
    return PS_ERR_INVALID_ARG;
  int dev = 0, nsm = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&nsm, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return PS_ERR_CUDA;
  ps_kv* kv = new (std::nothrow) ps_kv{};
  if (!kv) return PS_ERR_CUDA;
  kv->pool = make_pool(*cfg);
  kv->maps = new (std::nothrow) PoolMaps[(size_t)cfg->num_layers];
  if (!kv->maps) {
    delete kv;
    return PS_ERR_CUDA;
  }
  for (int32_t l = 0; l < cfg->num_layers; ++l) make_maps(kv->pool, l, kv->maps + l);
  kv->dev = dev;
  kv->nsm = nsm < kMaxSms ? nsm : kMaxSms;
  kv->max_requests = cfg->max_requests;
  kv->max_tokens = cfg->max_tokens;
  kv->max_row_pages = cfg->max_row_pages;
  int32_t workers[kLists];
  int32_t rc = configure_attention(kv->pool, kv->nsm, workers);
  for (int l = 0; l < kLists; ++l)
    if (workers[l] > kSizedWorkers[l]) workers[l] = kSizedWorkers[l];
  if (rc == PS_OK) {
    carve(*cfg, kSizedWorkers, static_cast<char*>(d_workspace), &kv->plan, &kv->pages, &kv->layout, &kv->reorder);
    for (int l = 0; l < kLists; ++l) kv->plan.max_workers[l] = workers[l];
    // and a plan that is empty, for an attention that runs before its plan has (one that was only captured into a graph)
    static_assert(PS_ERR_INVALID_ARG == -1, "the status word of all ones");
    PlanHdr* hdr = kv->plan.hdr;
    const size_t np = (size_t)(kv->pool.num_pages - kv->pool.first_page);
    if (cudaMemsetAsync(kv->pages.hdr, 0, sizeof(PageHdr), as_stream(stream)) != cudaSuccess ||
        (np > 0 && cudaMemsetAsync(kv->reorder.delta, 0, 4 * np, as_stream(stream)) != cudaSuccess) ||
        cudaMemsetAsync(hdr, 0, sizeof(PlanHdr), as_stream(stream)) != cudaSuccess ||
        cudaMemsetAsync(&hdr->status, 0xFF, sizeof(hdr->status), as_stream(stream)) != cudaSuccess)
      rc = PS_ERR_CUDA;
  }
  if (rc != PS_OK) {
    ps_kv_destroy(kv);
    return rc;
  }
  *out = kv;
  return PS_OK;
}

void ps_kv_destroy(ps_kv_t* kv) {
  if (!kv) return;
  delete[] kv->maps;
  delete kv;
}

int32_t ps_kv_append(ps_kv_t* kv, void* stream, int32_t layer, const ps_kv_append_t* a, int32_t* d_status) {
  if (!kv || !a || layer < 0 || layer >= kv->pool.num_layers || a->num_tokens < 0 || a->num_tokens > (1 << 30))
    return PS_ERR_INVALID_ARG;
  if (a->num_tokens == 0) return PS_OK;
  if (!a->q || !a->k || !a->v || !a->q_out || !a->slots) return PS_ERR_INVALID_ARG;
  for (const void* p : {a->q, a->k, a->v, (const void*)a->q_out, a->q_weight, a->k_weight, (const void*)a->rope})
    if (!aligned16(p)) return PS_ERR_INVALID_ARG;
  if (!good_strides(a->q_stride) || !good_strides(a->k_stride) || !good_strides(a->v_stride) ||
      !good_strides(a->q_out_stride))
    return PS_ERR_INVALID_ARG;
  if ((a->q_weight || a->k_weight) && !(a->eps > 0)) return PS_ERR_INVALID_ARG;
  if (a->rope && (!a->positions || a->rope_rows < 1 || a->rope_dim < 8 || a->rope_dim % 8 != 0 ||
                  a->rope_dim > kv->pool.head_dim))
    return PS_ERR_INVALID_ARG;
  // q_out is q, or lies on none of the inputs: warps read ahead of what others write
  const Pool& p = kv->pool;
  const int64_t T = a->num_tokens, hq = p.q_heads, hk = p.kv_heads, dim = p.head_dim;
  const HeadRuns q = runs(a->q, a->q_stride, hq), out = runs(a->q_out, a->q_out_stride, hq);
  const bool in_place = q.p == out.p && (T == 1 || q.s0 == out.s0) && (hq == 1 || q.s1 == out.s1);
  if (heads_overlap(out, out, T, dim, true) || (!in_place && heads_overlap(out, q, T, dim)) ||
      heads_overlap(out, runs(a->k, a->k_stride, hk), T, dim) || heads_overlap(out, runs(a->v, a->v_stride, hk), T, dim))
    return PS_ERR_INVALID_ARG;
  return launch_append(kv->pool, layer, *a, d_status, kv->nsm, as_stream(stream));
}

int32_t ps_kv_plan(ps_kv_t* kv, void* stream, const ps_kv_batch_t* b, int32_t* d_status) {
  if (!kv || !b) return PS_ERR_INVALID_ARG;
  if (b->num_requests < 0 || b->num_requests > kv->max_requests || b->num_tokens < 0 ||
      b->num_tokens > kv->max_tokens || b->table_stride < 0)
    return PS_ERR_INVALID_ARG;
  if (b->num_requests == 0 && b->num_tokens > 0) return PS_ERR_INVALID_ARG;
  if (b->num_requests > 0 && (!b->q_offsets || !b->kv_lens || (!b->tables && b->table_stride > 0)))
    return PS_ERR_INVALID_ARG;
  const bool grouped = b->group_offsets && b->num_requests > 0;  // an empty batch has nothing to group
  if (grouped && (b->num_groups < 1 || b->num_groups > b->num_requests)) return PS_ERR_INVALID_ARG;
  Batch x{};
  x.q_offsets = b->q_offsets; x.kv_lens = b->kv_lens; x.tables = b->tables;
  x.group_offsets = grouped ? b->group_offsets : nullptr;
  x.table_stride = b->table_stride;
  x.num_requests = b->num_requests; x.num_groups = b->num_groups; x.num_tokens = b->num_tokens;
  x.causal = b->causal != 0;
  x.row_pages = row_pages(kv, b->table_stride);
  const int32_t rc = launch_plan(kv->pool, kv->plan, x, d_status, as_stream(stream));
  kv->batch = x;
  kv->planned = rc == PS_OK;
  return rc;
}

int32_t ps_kv_attention(ps_kv_t* kv, void* stream, int32_t layer, const ps_kv_attention_t* a,
                        int32_t* d_status) {
  if (!kv || !a || !kv->planned || layer < 0 || layer >= kv->pool.num_layers) return PS_ERR_INVALID_ARG;
  if (kv->batch.num_tokens == 0 || kv->batch.num_requests == 0) return PS_OK;
  if (!a->q || !a->out || !aligned16(a->q) || !aligned16(a->out) || !good_strides(a->q_stride) ||
      !good_strides(a->out_stride) || !(a->scale - a->scale == 0))
    return PS_ERR_INVALID_ARG;
  const HeadRuns q = runs(a->q, a->q_stride, kv->pool.q_heads), out = runs(a->out, a->out_stride, kv->pool.q_heads);
  if (heads_overlap(out, out, kv->batch.num_tokens, kv->pool.head_dim, true) ||
      heads_overlap(out, q, kv->batch.num_tokens, kv->pool.head_dim))
    return PS_ERR_INVALID_ARG;
  kv->turn ^= 1;
  return launch_attention(kv->pool, kv->maps[layer], kv->plan, kv->batch, layer, kv->turn, *a, d_status, as_stream(stream));
}

int32_t ps_kv_layout(ps_kv_t* kv, void* stream, const ps_kv_rows_t* rows, const ps_kv_layout_t* l, int32_t* d_status) {
  if (!kv || !l || !rows_ok(kv, rows) || (l->pad != 0 && l->pad != 1)) return PS_ERR_INVALID_ARG;
  const int64_t n = l->num_requests, all = n + l->pad, T = l->num_tokens, stride = rows->table_stride;
  if (n < 0 || all > kv->max_requests || T < 0 || T > kv->max_tokens || stride >= (1ll << 30)) return PS_ERR_INVALID_ARG;
  if (!l->q_offsets || (all > 0 && (!l->kv_lens || !l->tables)) || (T > 0 && (!l->positions || !l->slots))) return PS_ERR_INVALID_ARG;
  if (!l->rows && n > rows->num_rows) return PS_ERR_INVALID_ARG;
  const Span spans[] = {{l->rows, 4 * n, false}, {l->counts, 4 * n, false}, {l->starts, 4 * n, false}, {l->written, 4 * n, false},
                        {rows->tables, 4ll * rows->num_rows * stride, false}, {rows->lens, 4ll * rows->num_rows, false},
                        {rows->held, 4ll * rows->num_rows, false}, {d_status, 4, false},
                        {l->q_offsets, 4 * (all + 1), true}, {l->kv_lens, 4 * all, true}, {l->tables, 4 * all * stride, true},
                        {l->positions, 4 * T, true}, {l->slots, 8 * T, true}, {l->group_offsets, 4 * (all + 1), true}};
  if (!outputs_apart(spans) || !on_device(kv->dev)) return PS_ERR_INVALID_ARG;
  return launch_layout(kv->pool, kv->layout, *l, *rows, row_pages(kv, stride), d_status, kv->nsm, as_stream(stream));
}

int32_t ps_kv_copy(ps_kv_t* kv, void* stream, int32_t n, const int32_t* d_src, const int32_t* d_dst,
                   int32_t* d_status) {
  if (!kv || n < 0 || (n > 0 && (!d_src || !d_dst))) return PS_ERR_INVALID_ARG;
  if (n == 0) return PS_OK;
  return launch_copy(kv->pool, n, d_src, d_dst, d_status, kv->nsm, as_stream(stream));
}

int32_t ps_kv_fork(ps_kv_t* kv, void* stream, int32_t n, const int32_t* d_parents, const int32_t* d_children,
                   const int32_t* d_room, const ps_kv_rows_t* rows, const int32_t* d_refs_in, int32_t* d_refs_out,
                   int32_t* d_status) {
  if (!kv || !rows_ok(kv, rows) || n < 0 || n > kv->max_requests || !refs_ok(kv, d_refs_in, d_refs_out)) return PS_ERR_INVALID_ARG;
  if (n > 0 && (!d_parents || !d_children || !d_room)) return PS_ERR_INVALID_ARG;
  if (partly_same(d_refs_in, d_refs_out, kv->pool.num_pages - kv->pool.first_page)) return PS_ERR_INVALID_ARG;
  return launch_fork(kv->pool, kv->pages, n, d_parents, d_children, d_room, *rows, row_pages(kv, rows->table_stride),
                     d_refs_in, d_refs_out, d_status, kv->nsm, as_stream(stream));
}

int32_t ps_kv_reorder(ps_kv_t* kv, void* stream, int32_t num_requests, int32_t beams, const int32_t* d_rows,
                      const int32_t* d_parents, int32_t grow, const ps_kv_rows_t* rows, const int32_t* d_refs_in,
                      int32_t* d_refs_out, int32_t* d_status) {
  if (!kv || !rows_ok(kv, rows) || num_requests < 0 || beams < 1 || beams > PS_KV_MAX_BEAMS || grow < 0 ||
      (int64_t)num_requests * beams > kv->max_requests || !refs_ok(kv, d_refs_in, d_refs_out) || rows->table_stride >= (1ll << 30))
    return PS_ERR_INVALID_ARG;
  if (num_requests > 0 && (!d_rows || !d_parents)) return PS_ERR_INVALID_ARG;
  const int64_t n = (int64_t)num_requests * beams, np = kv->pool.num_pages - kv->pool.first_page, m = rows->num_rows;
  const Span spans[] = {{d_rows, 4 * n, false}, {d_parents, 4 * n, false}, {d_status, 4, false},
                        {d_refs_in == d_refs_out ? nullptr : d_refs_in, 4 * np, false}, {d_refs_out, 4 * np, true},
                        {rows->tables, 4 * m * rows->table_stride, true}, {rows->lens, 4 * m, true}, {rows->held, 4 * m, true}};
  if (!outputs_apart(spans) || !on_device(kv->dev)) return PS_ERR_INVALID_ARG;
  return launch_reorder(kv->pool, kv->pages, kv->reorder, num_requests, beams, d_rows, d_parents, grow, *rows,
                        row_pages(kv, rows->table_stride), d_refs_in, d_refs_out, d_status, kv->nsm, as_stream(stream));
}

int32_t ps_kv_release(ps_kv_t* kv, void* stream, int32_t n, const int32_t* d_rows, const ps_kv_rows_t* rows,
                      int32_t* d_refs, int32_t* d_status) {
  if (!kv || !rows_ok(kv, rows) || n < 0 || n > kv->max_requests || !refs_ok(kv, d_refs, d_refs) || (n > 0 && !d_rows))
    return PS_ERR_INVALID_ARG;
  if (n == 0) return PS_OK;
  return launch_release(kv->pool, n, d_rows, *rows, row_pages(kv, rows->table_stride), d_refs, d_status,
                        as_stream(stream));
}

int32_t ps_kv_compact(ps_kv_t* kv, void* stream, const ps_kv_rows_t* rows, const int32_t* d_refs_in,
                      int32_t* d_tables_out, int32_t* d_refs_out, int32_t* d_counts, int32_t* d_status) {
  if (!kv || !rows || !rows->tables || !rows->held || rows->num_rows < 1 || rows->table_stride < 1 ||
      !refs_ok(kv, d_refs_in, d_refs_out) || !d_tables_out || !d_counts)
    return PS_ERR_INVALID_ARG;
  if (partly_same(d_refs_in, d_refs_out, kv->pool.num_pages - kv->pool.first_page) ||
      partly_same(rows->tables, d_tables_out, rows->num_rows * rows->table_stride))
    return PS_ERR_INVALID_ARG;
  return launch_compact(kv->pool, kv->pages, *rows, d_refs_in, d_tables_out, d_refs_out, d_counts, d_status, kv->nsm,
                        as_stream(stream));
}

}  // extern "C"
