// Internal declarations of the operators on KV pages (prefixshield_kv.h).
//
// Every kernel receives its arguments by value: the pool's description, the
// carved scratch pointers and the call's own pointers.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

#include "prefixshield_kv.h"

namespace pskv {

// ---- the pool ----------------------------------------------------------------
struct Pool {
  char* k;
  char* v;
  int64_t num_pages, first_page;
  int64_t layer_stride, page_stride, token_stride, head_stride;  // elements
  int32_t num_layers, page_size, page_log2, kv_heads, q_heads, ratio, head_dim, dtype;
};

// ---- a batch's plan ------------------------------------------------------------
// The work of a batch is a list of tiles: some query rows against a range of
// keys.  The rows of a tile are (token, query head of one kv head) pairs, token
// major, so a tile is run once for each kv head.  A tile's keys are cut into
// units.  A (tile, head) costs its units and tile_cost() more, for its beginning
// and end; of the whole list's cost U (tile major, then kv head) worker c of C
// (a CTA of the wide tiles' kernel, a warp of the narrow ones') gets
// [floor(U c / C), floor(U (c + 1) / C)): each the same, whatever the lengths
// are.  Within a (tile, head) the beginning's cost comes first, unit u is place
// tile_cost() + u.  A (tile, head) that several workers share, or whose rows also have a shared prefix, leaves partial results
// (a running maximum, a sum, an unnormalized output) that k_attend_join puts
// together in a fixed order.
struct __align__(32) Tile {
  int32_t tok0;   // token of row 0 of the tile's item (a request or a group)
  int32_t row0;   // the tile's first row within the item
  int32_t nrows;  // rows of the tile
  int32_t kv0;    // keys [kv0, kv1) of table row req
  int32_t kv1;
  int32_t req;
  int32_t ctx;    // row r of the item sees the keys < ctx + 1 + r / ratio
  int32_t sidx;   // rows of the shared (tile, head)s before (tile, head 0), -1: not shared
};

struct ReqRec {
  int32_t tile0;   // first tile of the request's own keys
  int32_t list;    // and the list it is in
  int32_t ptile0;  // first tile of its group's shared prefix, -1: none
  int32_t plist;
  int32_t prow0;   // the request's first row among the group's
};

constexpr int kLists = 2;        // 0: narrow tiles (mma), 1: wide tiles (tcgen05)
__host__ __device__ constexpr int tile_rows(int list) { return list ? 256 : 16; }
__host__ __device__ constexpr int unit_keys(int list) { return list ? 128 : 16; }
// What a (tile, head) costs beside its units, in units (wide: 11000 cycles measured
// for its beginning and end, of 2800 a unit; with 2 for it prompts took 293 us, with
// 4 281, on one input again).
__host__ __device__ constexpr int tile_cost(int list) { return list ? 4 : 1; }
// The list of an item of so many rows.
__host__ __device__ constexpr int list_of(int rows) { return rows > tile_rows(0) ? 1 : 0; }
constexpr int kNoMask = 1 << 30;

// A (tile, head)'s partial results: 'count' of them, the first at row 'first' of
// the list's partial rows, the others 'stride' rows apart from 'second' on.
struct Parts4 {
  int32_t first, second, count, stride;
};
// A (tile, head) of a request's own keys whose rows have partial results: its
// own, and those of its group's shared prefix.  The tile's rows may lie in two
// of the prefix's tiles: row r is row r + pofs of the first below psplit, and
// row r - psplit of the second from there on.
struct __align__(16) JoinRec {
  Parts4 own, pa, pb;
  int32_t tok0, row0, nrows, head;
  int32_t plist, pofs, psplit, pad0;  // plist -1: no prefix
};

struct __align__(16) PlanHdr {
  int32_t status;           // PS_OK, or why the plan is empty
  int32_t joins[kLists];    // entries of joins[]
  int32_t mend[2];          // some byte of mend[] was set by the last call with this place, see AttendArgs
  int32_t ntiles[kLists];
  int32_t workers[kLists];  // C, 0 without tiles
  int32_t narrow_ctas;      // CTAs that the narrow tiles' workers are spread over
  int64_t cost[kLists];     // U
};

// Requests of more rows than this fill tiles of their own; a prefix shared by
// smaller ones is read once for all of them.
constexpr int kShareRows = 64;
// Shared tokens below which the second part of a row costs more than it saves.
constexpr int kShareTokens = 128;
constexpr int kMaxSms = 160;

// Tiles of one list, and rows of one kv head that have a shared prefix (in its
// tiles, and in their own), for at most R requests of at most 'rows' rows in
// all.  An item (a request's own keys, or a group's prefix; at most R of each)
// of x rows has at most 1 + x / H tiles.
struct PlanBounds {
  int64_t tiles, own_tiles, shared;  // own_tiles: without the prefixes'
};
inline PlanBounds plan_bounds(int list, int64_t R, int64_t rows) {
  const int64_t own = R + rows / tile_rows(list) + 1;
  return {2 * own, own, 2 * (rows < R * kShareRows ? rows : R * kShareRows)};
}

// The worker of place u: the largest c with floor(U c / C) <= u.
__host__ __device__ __forceinline__ int worker_of(int64_t u, int64_t U, int64_t C) {
  return (int)(((u + 1) * C - 1) / U);
}

struct Plan {
  PlanHdr* hdr;
  ReqRec* req;        // [max_requests]
  int32_t* tok_req;   // [max_tokens] request of a token
  int32_t* group;     // [max_requests] group of a request
  int32_t* grp_tile;  // [max_requests] first tile of a group's shared prefix, -1: none
  int32_t* grp_list;  // [max_requests] and the list it is in
  int32_t* common;    // [max_requests] leading pages in common with the group's first request
  int32_t* bad;       // [max_requests]
  Tile* tiles[kLists];
  int64_t* ucum[kLists];      // [tiles + 1] cost before a tile, all heads
  int32_t* first_tile[kLists];  // [C] tile of a worker's first place
  JoinRec* joins[kLists];     // [tiles of requests x kv heads]
  uint8_t* mend[kLists];      // [tiles x kv heads] an output written by its tile is not finite, see mend_row
  float4* part_o[kLists];     // unnormalized outputs of the rows, see part_row and part_word
  float2* part_ml[kLists];    // [rows] (maximum, sum), base 2
  int32_t max_workers[kLists];
};

// The first row of the partial results of a (tile, head)'s part that worker c
// computed.  A worker leaves at most two partial results of (tile, head)s that are
// not shared, of the one it continues and of the one it leaves unfinished: two
// places of H rows each.  Along the list of shared (tile, head)s neither the
// rows before one nor c ever decreases, and one of them grows by as much as a
// part takes from each part to the next.
template <int H>
__host__ __device__ __forceinline__ int64_t part_row(int sidx, int nrows, int head, int c, bool continued, int C) {
  return sidx >= 0 ? (int64_t)(2 * C + c) * H + sidx + (int64_t)head * nrows : (int64_t)(2 * c + (continued ? 0 : 1)) * H;
}

// Tensor maps of one layer's keys and values: (element, head, token, page) with a
// box of 64 elements of min(page_size, 16) tokens, and, where a head is whole
// times 64 elements, (element, token, 64-element part, head, page) with a box of
// all of a head's elements.
struct PoolMaps {
  CUtensorMap k, v, whole_k, whole_v;
  CUtensorMap q;  // a call's queries: (element, head of a group, group, token), a box of 64 elements of 128 rows
  int32_t ok;     // 0: pages of fewer than 8 tokens, or no maps
  int32_t whole;  // whole_k and whole_v are there
  int32_t box;    // tokens of a box: 8 or 16
  int32_t q_ok;   // q is there
};
bool make_maps(const Pool& p, int32_t layer, PoolMaps* m);

// Place of the four elements from 4 c on of partial row r: eight rows' words lie
// side by side, so that a warp of 32 rows (wide tiles) and one of eight rows by
// four words (narrow tiles, the join) write and read whole lines.
__device__ __forceinline__ int64_t part_word(int64_t r, int c, int head_dim) {
  return ((r >> 3) * (head_dim >> 2) + c) * 8 + (r & 7);
}

// A worker's part of a list, one (tile, head) at a time.
template <int LIST>
struct Parts {
  static constexpr int K = tile_cost(LIST);
  const Tile* tiles;
  const int64_t* ucum;
  int heads, left, tile, head, unit, nunits, count;  // units [unit, unit + count) of nunits; left: cost from the head's begin
  Tile t;
  // False if there is no unit in it.
  __device__ __forceinline__ bool start(const Plan& plan, int kv_heads, int c, int64_t u0, int64_t u1) {
    tiles = plan.tiles[LIST];
    ucum = plan.ucum[LIST];
    heads = kv_heads;
    tile = plan.first_tile[LIST][c];
    t = tiles[tile];
    const int64_t b = ucum[tile];
    const int each = (int)((ucum[tile + 1] - b) / heads);
    nunits = each - K;
    head = (int)((u0 - b) / each);
    const int at = (int)((u0 - b) % each);
    left = (int)(u1 - u0) + at;
    unit = at > K ? at - K : 0;
    count = (left < each ? left : each) - K - unit;
    return count > 0;
  }
  __device__ __forceinline__ bool next() {
    left -= nunits + K;
    if (left <= K) return false;
    unit = 0;
    if (++head == heads) {
      head = 0;
      ++tile;
      t = tiles[tile];
      nunits = (int)((ucum[tile + 1] - ucum[tile]) / heads) - K;
    }
    count = (left < nunits + K ? left : nunits + K) - K;
    return true;
  }
};

struct Batch {
  const int32_t *q_offsets, *kv_lens, *tables, *group_offsets;
  int64_t table_stride;
  int32_t num_requests, num_groups, num_tokens, causal, row_pages;
};

// ---- page calls -----------------------------------------------------------------
struct PageHdr {
  int32_t done;    // CTAs of the scan that have finished (back to 0 after each call)
  int32_t status;  // verdict of the call
  int32_t live;    // pages in use (compact)
  int32_t free_pages;
  int32_t refused; // an error that a reorder's kernels found (back to 0 after each call)
  int32_t need;    // pages that a reorder takes
  int32_t parts;   // rows of a reorder that copy a page, as they are found (back to 0 after each call)
  int32_t copies;  // and all of them
};
constexpr int kScanThreads = 256;
constexpr int kMaxChunks = 1024;  // chunks of the reference array: one CTA each

struct PageScratch {
  PageHdr* hdr;
  int32_t* chunk_cnt;   // [chunks] free (fork) or used (compact) pages of a chunk
  int32_t* chunk_base;  // [chunks] those of the chunks before it
  int32_t* list;        // [private pages] fork: each chunk's free pages; compact: holes
  int32_t* movers;      // [private pages]
  int32_t* inv;         // [private pages] rank of a mover
  int32_t* mover_refs;  // [private pages]
  int32_t* need;        // [max_requests]
  int32_t* start;       // [max_requests]
  int32_t* bad;         // [max_requests]
  int32_t chunks, chunk_size;
};

// What becomes of one row of a reorder.
struct __align__(16) ReorderRec {
  int32_t row, src;     // the row, and the beam of its request that it continues, -1: none
  int32_t len, have, total;  // tokens, pages that it takes over or shares, pages in all
  int32_t part, from;   // tokens to copy, and the page that they are in
  int32_t pad0;
};
struct ReorderScratch {
  ReorderRec* rec;  // [max_requests]
  int32_t* copy;    // [max_requests] the rows that copy a page, in any order
  int32_t* delta;   // [private pages] changes of the references, 0 between calls
  int32_t* refs;    // [private pages] the references to be, the page calls' inv
};

// ---- layout --------------------------------------------------------------------
// Of batches that a CTA does not scan for itself: the requests, offsets and groups from
// a part's first on, the parts' totals, and where each part begins.
constexpr int kLayoutPart = 256;
struct LayoutScratch {
  int4* item;               // [max_requests] row, start, count, offset
  int32_t *offset, *group;  // [max_requests], the page calls' start and need
  int64_t* total;           // [parts]
  int32_t* groups;          // [parts]
  int32_t *base, *group_base;  // [parts + 1]
  int32_t* done;
};

// Is the current device the one that a handle was made on (host code)?  A launch on another
// one would follow addresses that are not its own.
inline bool on_device(int32_t dev) {
  int d;
  return cudaGetDevice(&d) == cudaSuccess && d == dev;
}

// ---- device helpers ----------------------------------------------------------------
__device__ __forceinline__ void set_error(int32_t* status, int32_t code) {
  if (status) atomicMin(status, code);
}
// Wait for the kernels before this one, then let the next one be scheduled (its
// CTAs wait here in turn).  Every kernel of these operators starts with it, but
// for the attention's, which read the plan first.
__device__ __forceinline__ void chain() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

template <typename T>
struct Num;
template <>
struct Num<__nv_bfloat16> {
  static constexpr bool kBf16 = true;
  static constexpr uint32_t kNan2 = 0x7FC07FC0u;
  static __device__ __forceinline__ float2 unpack(uint32_t x) {
    return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xFFFF0000u));
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
  }
};
template <>
struct Num<__half> {
  static constexpr bool kBf16 = false;
  static constexpr uint32_t kNan2 = 0x7E007E00u;
  static __device__ __forceinline__ float2 unpack(uint32_t x) {
    return __half22float2(*reinterpret_cast<const __half2*>(&x));
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
  }
};
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Two 32-bit numbers in one 64-bit register, worked on by one instruction.
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 unpack2(uint64_t x) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// ---- host ------------------------------------------------------------------------
// Launch that may be scheduled while its predecessor finishes (see chain()).
template <typename... KArgs, typename... Args>
inline cudaError_t launch(void (*kernel)(KArgs...), dim3 grid, int block, size_t smem, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}
inline int32_t status_of(cudaError_t e) { return e == cudaSuccess ? PS_OK : PS_ERR_CUDA; }

int32_t launch_append(const Pool& p, int32_t layer, const ps_kv_append_t& a, int32_t* status, int nsm, cudaStream_t st);
int32_t launch_plan(const Pool& p, const Plan& plan, const Batch& b, int32_t* status, cudaStream_t st);
int32_t launch_attention(const Pool& p, const PoolMaps& maps, const Plan& plan, const Batch& b, int32_t layer, int32_t turn, const ps_kv_attention_t& a,
                         int32_t* status, cudaStream_t st);
int32_t launch_copy(const Pool& p, int32_t n, const int32_t* src, const int32_t* dst, int32_t* status, int nsm,
                    cudaStream_t st);
int32_t launch_fork(const Pool& p, const PageScratch& w, int32_t n, const int32_t* parents, const int32_t* children,
                    const int32_t* room, const ps_kv_rows_t& rows, int32_t row_pages, const int32_t* refs_in,
                    int32_t* refs_out, int32_t* status, int nsm, cudaStream_t st);
int32_t launch_release(const Pool& p, int32_t n, const int32_t* list, const ps_kv_rows_t& rows, int32_t row_pages,
                       int32_t* refs, int32_t* status, cudaStream_t st);
int32_t launch_compact(const Pool& p, const PageScratch& w, const ps_kv_rows_t& rows, const int32_t* refs_in, int32_t* tables_out, int32_t* refs_out, int32_t* counts,
                       int32_t* status, int nsm, cudaStream_t st);
int32_t launch_reorder(const Pool& p, const PageScratch& w, const ReorderScratch& o, int32_t requests, int32_t beams, const int32_t* list,
                       const int32_t* parents, int32_t grow, const ps_kv_rows_t& rows, int32_t row_pages,
                       const int32_t* refs_in, int32_t* refs_out, int32_t* status, int nsm, cudaStream_t st);
int32_t launch_layout(const Pool& p, const LayoutScratch& w, const ps_kv_layout_t& l, const ps_kv_rows_t& rows, int32_t row_pages,
                      int32_t* status, int nsm, cudaStream_t st);
// Kernel attributes (shared-memory opt-ins) and the workers of each attention list
// that the current device holds at once.
constexpr int kNarrowWarps = 4;  // of a CTA
int32_t configure_attention(const Pool& p, int nsm, int32_t workers[kLists]);

}  // namespace pskv
