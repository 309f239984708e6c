// ps_kv_attention: the wide tiles (17 to 256 query rows of one request, or of
// the requests that share a prefix), on tcgen05.
//
// The mathematics is the narrow tiles' (ps_kv_attend.cu).  One CTA an SM takes
// its part of the list of units; a unit is 128 keys.  Its warps:
//   8 softmax warps, two groups t of four, a thread a query row;
//   4 loader warps, each with a quarter of every unit's keys and values: whole
//     units by TMA, a box for a page (or half a page of 64) and 64 elements.  A
//     request's last unit, whose values past its end must read as zero, queries,
//     and pages of 2 or 4 tokens, whose boxes would not fill the 1024 bytes after
//     which the swizzle repeats, go by 16-byte asynchronous copies instead, eight
//     times the instructions and waited for by the copying threads: with them for
//     all units the loader warps took 7400 cycles a unit, the products 2350;
//   1 warp that issues the matrix instructions (3 more idle).
// A tile of more than 128 rows is two row blocks, one for each group, that use
// every unit's keys and values (pair mode).  A tile of up to 128 rows is one
// row block; the groups take its units in turn, each with a softmax of its own
// over them, joined when the tile ends (split mode).
//
// Tensor memory: scores S_t (128 columns of 32 bits; the weights P_t overwrite
// the first 64 with pairs of 16 bits) and outputs O_t (up to 128 columns).
// S_t = Q K^T reads both operands from shared memory; O_t += P_t V takes P_t
// from tensor memory.  While group t computes weights, the other group's
// products run.  The maximum that the weights refer to moves only when a score
// passes it by 2^8: O_t is rescaled rarely, and the final division makes up for
// whichever reference was used.
#include "ps_kv_attend.cuh"

namespace pskv {
namespace {

constexpr int kSoftmaxWarps = 8, kLoaderWarps = 4;
constexpr int kThreads = 512;  // four warpgroups: registers move between whole ones
constexpr int kSoftmaxRegs = 192, kOtherRegs = 64;  // 2 x 128 x (192 + 64) = 512 x 128, the launch's own
constexpr int UNIT = unit_keys(1), H = tile_rows(1);
__device__ __forceinline__ constexpr uint32_t col_s(int t) { return 128u * t; }
__device__ __forceinline__ constexpr uint32_t col_o(int t) { return 256u + 128u * t; }
// Bound of every wait: far beyond any tile's time, so it only ends a wait that
// would never end.
constexpr int kWaitLimit = 1 << 20;
constexpr float kRescale = 8.0f;

template <int DP>
struct Shape {
  static constexpr int kHalves = DP > 64 ? 2 : 1;          // 64-element halves of a row
  static constexpr int kBlock = 128 * 128 * kHalves;       // bytes of 128 rows
  static constexpr int kBuffers = DP > 64 ? 5 : 10;        // ring of key and value blocks, in turn
  static constexpr int kLag = kBuffers - 2;                // blocks in flight before the oldest is waited for
  static constexpr int kSmem = 1024 + (2 + kBuffers) * kBlock;
  static constexpr int kSteps = DP / 16;                   // k steps of Q K^T
};

struct Shared {
  uint64_t full[10], empty[10], s_full[2], p_full[2], o_full[2], q_full, q_empty, ml_full, ml_free;
  uint32_t tmem;
  float2 ml[128];  // split mode: group 1's (maximum, sum)
  int failed;
};

// ---- barriers, tensor memory ---------------------------------------------------
__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint64_t* b, int count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(b)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t* b) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(b)) : "memory");
}
__device__ __forceinline__ bool bar_test(uint64_t* b, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
      : "=r"(ok) : "r"(smem_addr(b)), "r"(parity) : "memory");
  return ok != 0;
}
// False if the wait ran out, here or in another warp.
__device__ __forceinline__ bool bar_wait(Shared* sh, uint64_t* b, uint32_t parity) {
  for (int i = 0; i < kWaitLimit; ++i) {
    if (bar_test(b, parity)) return true;
    if ((i & 255) == 255 && *(volatile int*)&sh->failed) return false;
  }
  *(volatile int*)&sh->failed = 1;
  return false;
}
// The same by a whole warp, with one answer.
__device__ __forceinline__ bool warp_wait(Shared* sh, uint64_t* b, uint32_t parity) {
  return __all_sync(0xFFFFFFFFu, bar_wait(sh, b, parity));
}
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// The commits and products below are one thread's.
__device__ __forceinline__ void tc_commit(uint64_t* b) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(b)) : "memory");
}
// d (+)= a b: both operands in shared memory, or a in tensor memory.
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile("{ .reg .pred p; setp.ne.u32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p; }" ::"r"(d),
               "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile("{ .reg .pred p; setp.ne.u32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p; }" ::"r"(d),
               "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
#define R8(x, i) "=r"(x[i]), "=r"(x[i + 1]), "=r"(x[i + 2]), "=r"(x[i + 3]), "=r"(x[i + 4]), "=r"(x[i + 5]), "=r"(x[i + 6]), "=r"(x[i + 7])
#define W8(x, i) "r"(x[i]), "r"(x[i + 1]), "r"(x[i + 2]), "r"(x[i + 3]), "r"(x[i + 4]), "r"(x[i + 5]), "r"(x[i + 6]), "r"(x[i + 7])
// 32 columns of the thread's lane.
__device__ __forceinline__ void tm_load32(uint32_t* x, uint32_t addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
      "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : R8(x, 0), R8(x, 8), R8(x, 16), R8(x, 24) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tm_load16(uint32_t* x, uint32_t addr) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : R8(x, 0), R8(x, 8) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tm_store16(uint32_t addr, const uint32_t* x) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr),
               W8(x, 0), W8(x, 8) : "memory");
}
__device__ __forceinline__ void tm_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tm_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
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
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool ok) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void to_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// Descriptor of a block of 128-byte rows with the 128-byte swizzle.  Eight rows
// are 1024 bytes; 'lead' is the distance of the second 64-element half where the
// rows are the contraction's (values), unused where they are the result's.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lead) {
  return (uint64_t)((addr >> 4) & 0x3FFF) | (uint64_t)((lead >> 4) & 0x3FFF) << 16 | (uint64_t)(1024 >> 4) << 32 |
         (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// Instruction descriptor: 32-bit sums of 16-bit products, 128 rows, n columns.
template <typename T>
__device__ __forceinline__ uint32_t instr_desc(int n, bool b_rows_contract) {
  const uint32_t type = sizeof(T) == 2 && Num<T>::kBf16 ? 1 : 0;
  return 1u << 4 | type << 7 | type << 10 | (b_rows_contract ? 1u << 16 : 0) | (uint32_t)(n >> 3) << 17 | (128u >> 4) << 24;
}

// The CTA's part of the list, one (tile, head) at a time; every role runs its own.
struct Parts {
  const Tile* tiles;
  const int64_t* ucum;
  int heads, left, tile, head, unit, nunits, count;
  Tile t;
  __device__ __forceinline__ void start(const AttendArgs& a, int64_t u0, int n, int first_tile) {
    tiles = a.plan.tiles[1];
    ucum = a.plan.ucum[1];
    heads = a.pool.kv_heads;
    left = n;
    tile = first_tile;
    t = tiles[tile];
    const int64_t b = ucum[tile];
    nunits = (int)((ucum[tile + 1] - b) / heads);
    head = (int)((u0 - b) / nunits);
    unit = (int)((u0 - b) % nunits);
    count = min(left, nunits - unit);
  }
  __device__ __forceinline__ bool next() {
    left -= count;
    if (left <= 0) return false;
    unit = 0;
    if (++head == heads) {
      head = 0;
      ++tile;
      t = tiles[tile];
      nunits = (int)((ucum[tile + 1] - ucum[tile]) / heads);
    }
    count = min(left, nunits);
    return true;
  }
  __device__ __forceinline__ bool pair() const { return t.nrows > 128; }
};

// ---- loader warps ------------------------------------------------------------------
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, uint64_t* bar, int x, int head, int token, int page,
                                         int layer) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst),
      "l"(map), "r"(x), "r"(head), "r"(token), "r"(page), "r"(layer), "r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void bar_expect(uint64_t* b, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_addr(b)), "r"(bytes) : "memory");
}

template <int DP>
struct Loader {
  using S = Shape<DP>;
  static constexpr int CH = DP / 8;                      // 16-byte words of a row that hold elements
  static constexpr int RPI = 32 / (CH <= 8 ? 8 : 16);    // rows that one copy instruction covers
  const AttendArgs& a;
  Shared* sh;
  const int lane, warp;
  const int w, sub;  // the lane's word of a row, and row of an instruction's
  uint32_t issued = 0, told = 0;  // blocks issued, blocks whose arrival was signalled

  __device__ __forceinline__ Loader(const AttendArgs& args, Shared* s)
      : a(args), sh(s), lane(threadIdx.x & 31), warp((threadIdx.x >> 5) - kSoftmaxWarps), w(lane % (32 / RPI)), sub(lane / (32 / RPI)) {}

  // 32 rows of the warp's, row r at element off (of lane r; -1: zeros).
  __device__ __forceinline__ void copy_rows(uint32_t dst, const char* base, int64_t off) const {
    const bool on = w * 8 < a.pool.head_dim;
    int64_t o[32 / RPI];
#pragma unroll
    for (int j = 0; j < 32 / RPI; ++j) o[j] = __shfl_sync(0xFFFFFFFFu, off, j * RPI + sub);
#pragma unroll
    for (int j = 0; j < 32 / RPI; ++j) {
      const int r = warp * 32 + j * RPI + sub;
      const bool ok = o[j] >= 0 && on;
      // word w of row r: half w / 8, swizzled within its 128 bytes
      if (w < CH)
        cp16(dst + (w >> 3) * (128 * 128) + r * 128 + (((w & 7) ^ (r & 7)) << 4), base + (ok ? 2 * o[j] + w * 16 : 0), ok);
    }
    cp_commit();
  }
  __device__ __forceinline__ void tell(uint32_t upto) {
    to_async_proxy();
    __syncwarp();
    for (; told < upto; ++told)
      if (lane == 0) bar_arrive(&sh->full[told % S::kBuffers]);
  }
  __device__ __forceinline__ void tell_all() {
    if (issued > told) {
      cp_wait<0>();
      tell(issued);
    }
  }
  // The next block of the ring is free.  What was copied is not held back by the wait.
  __device__ __forceinline__ bool room() {
    uint64_t* e = &sh->empty[issued % S::kBuffers];
    const uint32_t parity = ((issued / S::kBuffers) & 1) ^ 1;
    if (__all_sync(0xFFFFFFFFu, bar_test(e, parity))) return true;
    tell_all();
    return warp_wait(sh, e, parity);
  }
};

template <int DP>
__device__ __forceinline__ bool load_role(const AttendArgs& a, const PoolMaps& maps, Shared* sh, uint32_t qs, uint32_t ring, Parts ps) {
  using S = Shape<DP>;
  Loader<DP> ld(a, sh);
  const int lane = ld.lane, warp = ld.warp;
  const bool tma = maps.ok;
  // TMA: lane i issues box i % boxes of the warp's keys, half i / boxes
  const int boxes = 32 / maps.box, mybox = lane % boxes, myhalf = lane / boxes;
  const bool issues = tma && lane < boxes * S::kHalves;
  uint32_t seg = 0;
  bool more = true;
  for (; more; ++seg, more = ps.next()) {
    const Tile t = ps.t;
    const int32_t* row = a.tables + t.req * a.table_stride;
    const int64_t head_off = (int64_t)ps.head * a.pool.head_stride;
    ld.tell_all();
    // ids are looked up one unit ahead
    auto id_of = [&](int u) -> int {
      const int base = t.kv0 + (ps.unit + u) * UNIT;
      const bool whole = tma && base + UNIT <= t.kv1;
      const int key = base + warp * 32 + (whole ? mybox * maps.box : lane);
      return u < ps.count && key < t.kv1 ? __ldg(row + (key >> a.pool.page_log2)) : -1;
    };
    int page = id_of(0);
    for (int u = 0; u < ps.count; ++u) {
      const int base = t.kv0 + (ps.unit + u) * UNIT;
      const int id = page;
      page = id_of(u + 1);
      if (tma && base + UNIT <= t.kv1) {
        const int token = (base + warp * 32 + mybox * maps.box) & (a.pool.page_size - 1);
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          if (!ld.room()) return false;
          uint64_t* bar = &sh->full[ld.issued % S::kBuffers];
          if (lane == 0) bar_expect(bar, 32 * 128 * S::kHalves);
          __syncwarp();
          if (issues)
            tma_load(ring + ld.issued % S::kBuffers * S::kBlock + myhalf * (128 * 128) + (warp * 32 + mybox * maps.box) * 128,
                     kv ? &maps.v : &maps.k, bar, myhalf * 64, ps.head, token, id, a.layer);
          ++ld.issued;
          ++ld.told;
        }
      } else {
        const int key = base + warp * 32 + lane;
        int64_t off = -1;
        if (id >= 0) off = id * a.pool.page_stride + (int64_t)(key & (a.pool.page_size - 1)) * a.pool.token_stride + head_off;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          if (!ld.room()) return false;
          ld.copy_rows(ring + ld.issued % S::kBuffers * S::kBlock, kv ? a.v : a.k, off);
          ++ld.issued;
          if (ld.issued - ld.told > S::kLag) {
            cp_wait<S::kLag>();
            ld.tell(ld.issued - S::kLag);
          }
        }
      }
      if (u == 0) {  // queries, once the last tile's are read; its first keys are under way
        ld.tell_all();
        if (!warp_wait(sh, &sh->q_empty, (seg & 1) ^ 1)) return false;
        for (int blk = 0; blk < (ps.pair() ? 2 : 1); ++blk) {
          const int r = blk * 128 + warp * 32 + lane, rr = t.row0 + r;
          int64_t off = -1;
          if (r < t.nrows)
            off = (int64_t)(t.tok0 + rr / a.pool.ratio) * a.q_stride[0] +
                  (int64_t)(ps.head * a.pool.ratio + rr % a.pool.ratio) * a.q_stride[1];
          ld.copy_rows(qs + blk * S::kBlock, a.q, off);
        }
        cp_wait<0>();
        to_async_proxy();
        __syncwarp();
        if (lane == 0) bar_arrive(&sh->q_full);
      }
    }
  }
  ld.tell_all();
  return true;
}

// ---- the warp that issues the matrix instructions ------------------------------------
// One thread (the warp's first): products issued under a predicate by a whole
// warp took nearly twice as long (113 cycles against 64, 128 x 128 x 16).
template <typename T, int DP>
__device__ __forceinline__ bool mma_role(const AttendArgs& a, Shared* sh, uint32_t tmem, uint32_t qs, uint32_t ring, Parts ps) {
  using S = Shape<DP>;
  const uint32_t id_qk = instr_desc<T>(UNIT, false), id_pv = instr_desc<T>(DP, true);
  // descriptors differ in their address field alone
  const uint64_t q_desc = smem_desc(qs, 16), k_desc = smem_desc(ring, 16), v_desc = smem_desc(ring, 128 * 128);
  uint32_t p_phase = 0;  // bit t: of group t
  uint32_t k_slot = 0, k_par = 0;  // ring place of the tile's unit 0, and how often the ring has gone round (mod 2)
  // place and parity of a block 'ahead' of the tile's first
  auto slot_of = [&](uint32_t ahead, uint32_t* par) {
    const uint32_t i = k_slot + ahead;
    *par = (k_par + i / S::kBuffers) & 1;
    return i % S::kBuffers;
  };
  auto scores = [&](int t, int qblk, uint32_t slot) {
    const uint64_t q = q_desc + (uint64_t)(qblk * (S::kBlock >> 4)), k = k_desc + (uint64_t)(slot * (S::kBlock >> 4));
#pragma unroll
    for (int s = 0; s < S::kSteps; ++s) {
      constexpr int kHalf = 128 * 128 >> 4;
      const int at = (s >> 2) * kHalf + (s & 3) * 2;
      mma_ss(tmem + col_s(t), q + at, k + at, id_qk, s > 0);
    }
    tc_commit(&sh->s_full[t]);
  };
  uint32_t seg = 0;
  bool more = true;
  for (; more; ++seg, more = ps.next()) {
    const bool pair = ps.pair();
    const int n = ps.count;
    const int steps0 = pair ? n : (n + 1) / 2, steps1 = pair ? n : n / 2;
    if (!bar_wait(sh, &sh->q_full, seg & 1)) return false;
#pragma unroll 1
    for (int t = 0; t < 2; ++t) {
      if (t == 1 && steps1 == 0) continue;
      uint32_t par;
      const uint32_t kb = slot_of(pair ? 0 : 2 * t, &par);
      if (!bar_wait(sh, &sh->full[kb], par)) return false;
      tc_after();
      scores(t, pair ? t : 0, kb);
      if (!pair || t == 1) tc_commit(&sh->empty[kb]);
    }
    if (steps0 == 1) tc_commit(&sh->q_empty);
    for (int i = 0; i < steps0; ++i) {
#pragma unroll 1
      for (int t = 0; t < 2; ++t) {
        const int mine = t ? steps1 : steps0;
        if (i >= mine) continue;
        const uint32_t unit = pair ? i : 2 * i + t, step = pair ? 1 : 2;
        uint32_t vpar, kpar;
        const uint32_t vb = slot_of(2 * unit + 1, &vpar), kb = slot_of(2 * (unit + step), &kpar);
        if (!bar_wait(sh, &sh->full[vb], vpar)) return false;
        if (!bar_wait(sh, &sh->p_full[t], p_phase >> t & 1)) return false;
        p_phase ^= 1u << t;
        tc_after();
        const uint64_t v = v_desc + (uint64_t)(vb * (S::kBlock >> 4));
#pragma unroll
        for (int s = 0; s < UNIT / 16; ++s)
          mma_ts(tmem + col_o(t), tmem + col_s(t) + s * 8, v + s * (2048 >> 4), id_pv, i > 0 || s > 0);
        if (!pair || t == 1) tc_commit(&sh->empty[vb]);
        if (i + 1 < mine) {
          if (!bar_wait(sh, &sh->full[kb], kpar)) return false;
          tc_after();
          scores(t, pair ? t : 0, kb);
          if (!pair || t == 1) tc_commit(&sh->empty[kb]);
        } else {
          tc_commit(&sh->o_full[t]);
        }
      }
      if (i + 2 == steps0) tc_commit(&sh->q_empty);  // the last scores are on their way
    }
    k_slot = slot_of(2 * n, &k_par);
  }
  return true;
}

// ---- softmax warps ------------------------------------------------------------------
template <typename T, int DP>
__device__ __forceinline__ bool softmax_role(const AttendArgs& a, Shared* sh, uint32_t tmem, Parts ps, int c, int C) {
  const int warp = threadIdx.x >> 5, t = warp >> 2, lane = threadIdx.x & 31;
  const int row = (warp & 3) * 32 + lane;  // of the row block, and the tensor memory lane
  const uint32_t at = tmem + ((uint32_t)(warp & 3) << 21);
  const uint32_t s_at = at + col_s(t), o_at = at + col_o(t);
  // 2^(s sc - m): a scale of 0 or below goes into the scores
  const float sign = a.scale2 > 0 ? 1.0f : (a.scale2 < 0 ? -1.0f : 0.0f);
  const float sc = a.scale2 != 0 ? fabsf(a.scale2) : 1.0f;
  uint32_t s_phase = 0, o_mine = 0, o_other = 0, ml_phase = 0;  // o_other: group 1's, as group 0 counts it
  bool held = false;  // group 1: the last tile's O_1 and ml may still be read by group 0
  auto let_go = [&]() {
    if (!held) return true;
    held = false;
    const bool ok = warp_wait(sh, &sh->ml_free, ml_phase);
    ml_phase ^= 1;
    return ok;
  };
  bool more = true;
  for (; more; more = ps.next()) {
    const Tile tl = ps.t;
    const bool pair = ps.pair();
    const int n = ps.count;
    const int mine = pair ? n : (t == 0 ? (n + 1) / 2 : n / 2);
    const int trow = pair ? t * 128 + row : row;  // row of the tile
    const int rr = tl.row0 + trow;
    const int lim = min(tl.kv1, tl.ctx + 1 + rr / a.pool.ratio);
    float m = -INFINITY, l = 0;  // m: the scaled reference
    for (int i = 0; i < mine; ++i) {
      const int base = tl.kv0 + (ps.unit + (pair ? i : 2 * i + t)) * UNIT;
      if (!warp_wait(sh, &sh->s_full[t], s_phase)) return false;
      s_phase ^= 1;
      tc_after();
      uint32_t raw[128];
#pragma unroll
      for (int j = 0; j < 128; j += 32) tm_load32(raw + j, s_at + j);
      tm_wait_ld();
      float* s = reinterpret_cast<float*>(raw);
      if (sign != 1.0f) {
#pragma unroll
        for (int j = 0; j < 128; ++j) s[j] *= sign;
      }
      const int seen = lim - base;
      if (__any_sync(0xFFFFFFFFu, seen < UNIT)) {
#pragma unroll
        for (int j = 0; j < 128; ++j)
          if (j >= seen) s[j] = -INFINITY;
      }
      float mx[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
      for (int j = 4; j + 8 <= 128; j += 8)
#pragma unroll
        for (int x = 0; x < 4; ++x) mx[x] = max3(mx[x], s[j + 2 * x], s[j + 2 * x + 1]);
#pragma unroll
      for (int x = 0; x < 4; ++x) mx[x] = fmaxf(mx[x], s[124 + x]);
      const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * sc;
      const bool move = top > m + kRescale || m == -INFINITY;
      if (__any_sync(0xFFFFFFFFu, move)) {
        const float mn = move ? fmaxf(m, top) : m;
        const float f = m == -INFINITY ? 0.0f : ex2(m - mn);
        m = mn;
        l *= f;
        if (i > 0) {
#pragma unroll
          for (int j = 0; j < DP; j += 16) {
            uint32_t o[16];
            tm_load16(o, o_at + j);
            tm_wait_ld();
#pragma unroll
            for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * f);
            tm_store16(o_at + j, o);
          }
        }
      }
      const float ref = m == -INFINITY ? 0.0f : m;
      const uint64_t sc2 = pack2(sc, sc), ref2 = pack2(-ref, -ref);
      uint64_t sum[2] = {0, 0};
#pragma unroll
      for (int j = 0; j < 128; j += 32) {
        uint32_t p[16];
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const float2 e = unpack2(fma2(pack2(s[j + 2 * x], s[j + 2 * x + 1]), sc2, ref2));
          const float e0 = ex2(e.x), e1 = ex2(e.y);
          sum[x & 1] = add2(sum[x & 1], pack2(e0, e1));
          p[x] = Num<T>::pack(e0, e1);
        }
        tm_store16(s_at + j / 2, p);
      }
      const float2 total = unpack2(add2(sum[0], sum[1]));
      l += total.x + total.y;
      tm_wait_st();
      if (i == 0 && !let_go()) return false;
      tc_before();
      __syncwarp();
      if (lane == 0) bar_arrive(&sh->p_full[t]);
    }
    // the tile's end
    const bool whole = ps.unit == 0 && n == ps.nunits;
    float f[2] = {1.0f, 0.0f};
    if (!pair) {
      if (t == 1) {  // group 0 finishes the tile
        if (!let_go()) return false;
        sh->ml[row] = make_float2(m, l);
        __syncwarp();
        if (lane == 0) bar_arrive(&sh->ml_full);
        held = true;
        if (mine > 0) o_mine ^= 1;
        continue;
      }
      if (!warp_wait(sh, &sh->ml_full, ml_phase)) return false;
      ml_phase ^= 1;
      const float2 x = sh->ml[row];
      const float mn = fmaxf(m, x.x), ref = mn == -INFINITY ? 0.0f : mn;
      f[0] = ex2(m - ref);
      f[1] = ex2(x.x - ref);
      l = l * f[0] + x.y * f[1];
      m = mn;
    }
    if (!warp_wait(sh, &sh->o_full[t], o_mine)) return false;
    o_mine ^= 1;
    const bool both = !pair && n > 1;
    if (both && !warp_wait(sh, &sh->o_full[1], o_other)) return false;
    if (pair || n > 1) o_other ^= 1;
    tc_after();
    const bool direct = whole && tl.sidx < 0;
    const bool in = trow < tl.nrows;
    const int64_t tok = tl.tok0 + rr / a.pool.ratio;
    const int hq = ps.head * a.pool.ratio + rr % a.pool.ratio;
    const float inv = l > 0 ? 1.0f / l : (l == 0 ? 0.0f : l);
    char* op = a.out + 2 * (tok * a.out_stride[0] + (int64_t)hq * a.out_stride[1]);
    const int64_t prow = part_row<H>(tl.sidx, tl.nrows, ps.head, c, ps.unit > 0, C) + trow;
    float* po = a.plan.part_o[1] + prow * a.pool.head_dim;
#pragma unroll
    for (int j = 0; j < DP; j += 16) {
      uint32_t o[16];
      tm_load16(o, o_at + j);
      tm_wait_ld();
      float* x = reinterpret_cast<float*>(o);
      if (!pair) {
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] *= f[0];
        if (both) {
          uint32_t o1[16];
          tm_load16(o1, at + col_o(1) + j);
          tm_wait_ld();
#pragma unroll
          for (int e = 0; e < 16; ++e) x[e] += __uint_as_float(o1[e]) * f[1];
        }
      }
      if (!in) continue;
#pragma unroll
      for (int e = 0; e < 16; e += 8) {
        if (j + e >= a.pool.head_dim) continue;
        if (direct) {
          *reinterpret_cast<uint4*>(op + 2 * (j + e)) =
              make_uint4(Num<T>::pack(x[e] * inv, x[e + 1] * inv), Num<T>::pack(x[e + 2] * inv, x[e + 3] * inv),
                         Num<T>::pack(x[e + 4] * inv, x[e + 5] * inv), Num<T>::pack(x[e + 6] * inv, x[e + 7] * inv));
        } else {
          *reinterpret_cast<float4*>(po + j + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
          *reinterpret_cast<float4*>(po + j + e + 4) = make_float4(x[e + 4], x[e + 5], x[e + 6], x[e + 7]);
        }
      }
    }
    if (in) {
      if (!direct) a.plan.part_ml[1][prow] = make_float2(m, l);
      else if (a.lse) a.lse[tok * a.pool.q_heads + hq] = log_sum(m, l);
    }
    tc_before();
    if (!pair) {
      __syncwarp();
      if (lane == 0) bar_arrive(&sh->ml_free);
    }
  }
  return true;
}

template <typename T, int DP>
__global__ void __launch_bounds__(kThreads, 1) k_attend_wide(const __grid_constant__ AttendArgs a,
                                                             const __grid_constant__ PoolMaps maps) {
  using S = Shape<DP>;
  extern __shared__ char dyn[];
  __shared__ Shared sh;
  chain();
  const PlanHdr* hdr = a.plan.hdr;
  const int C = hdr->ctas[1], c = blockIdx.x;
  if (c >= C) return;
  const int64_t U = hdr->units[1], u0 = U * c / C;
  const int n = (int)(U * (c + 1) / C - u0);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t qs = (smem_addr(dyn) + 1023) & ~1023u, ring = qs + 2 * S::kBlock;
  if (warp == kSoftmaxWarps + kLoaderWarps) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&sh.tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (threadIdx.x == 0) {
    for (int b = 0; b < S::kBuffers; ++b) {
      bar_init(&sh.full[b], kLoaderWarps);
      bar_init(&sh.empty[b], 1);
    }
    for (int t = 0; t < 2; ++t) {
      bar_init(&sh.s_full[t], 1);
      bar_init(&sh.p_full[t], 4);
      bar_init(&sh.o_full[t], 1);
    }
    bar_init(&sh.q_full, kLoaderWarps);
    bar_init(&sh.q_empty, 1);
    bar_init(&sh.ml_full, 4);
    bar_init(&sh.ml_free, 4);
    sh.failed = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  tc_before();
  __syncthreads();
  tc_after();
  const uint32_t tmem = sh.tmem;
  Parts ps;
  ps.start(a, u0, n, a.plan.cta_tile[1][c]);
  bool ok = true;
  if (warp < kSoftmaxWarps) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
    ok = softmax_role<T, DP>(a, &sh, tmem, ps, c, C);
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
  }
  if (warp >= kSoftmaxWarps && warp < kSoftmaxWarps + kLoaderWarps) {
    ok = load_role<DP>(a, maps, &sh, qs, ring, ps);
    cp_wait<0>();
  } else if (warp == kSoftmaxWarps + kLoaderWarps && lane == 0) {
    ok = mma_role<T, DP>(a, &sh, tmem, qs, ring, ps);
  }
  if (!ok && lane == 0) set_error(a.status, PS_ERR_TIMEOUT);
  __syncwarp();
  tc_before();
  __syncthreads();
  tc_after();
  if (warp == kSoftmaxWarps + kLoaderWarps)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

template <typename T, int DP>
cudaError_t wide(const AttendArgs& a, const PoolMaps& m, cudaStream_t st) {
  return launch(k_attend_wide<T, DP>, dim3((unsigned)a.plan.max_ctas[1]), kThreads, Shape<DP>::kSmem, st, a, m);
}
template <typename T>
cudaError_t wide_t(const AttendArgs& a, const PoolMaps& m, cudaStream_t st) {
  const int d = a.pool.head_dim;
  return d <= 64 ? wide<T, 64>(a, m, st) : d <= 80 ? wide<T, 80>(a, m, st) : d <= 96 ? wide<T, 96>(a, m, st) : wide<T, 128>(a, m, st);
}
template <typename T, int DP>
cudaError_t configure_dp() {
  return cudaFuncSetAttribute(k_attend_wide<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<DP>::kSmem);
}
template <typename T>
cudaError_t configure_t(int d) {
  return d <= 64 ? configure_dp<T, 64>() : d <= 80 ? configure_dp<T, 80>() : d <= 96 ? configure_dp<T, 96>() : configure_dp<T, 128>();
}

}  // namespace

cudaError_t launch_wide(const AttendArgs& a, const PoolMaps& m, cudaStream_t st) {
  return a.pool.dtype == PS_KV_BF16 ? wide_t<__nv_bfloat16>(a, m, st) : wide_t<__half>(a, m, st);
}

bool make_maps(const Pool& p, PoolMaps* m) {
  m->ok = 0;
  m->box = p.page_size < 32 ? p.page_size : 32;
  if (p.page_size < 8) return false;
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult found;
  if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess ||
      found != cudaDriverEntryPointSuccess || !fn)
    return false;
  const auto encode = reinterpret_cast<decltype(&cuTensorMapEncodeTiled)>(fn);
  const cuuint64_t dims[5] = {(cuuint64_t)p.head_dim, (cuuint64_t)p.kv_heads, (cuuint64_t)p.page_size, (cuuint64_t)p.num_pages,
                              (cuuint64_t)p.num_layers};
  const int64_t stride[4] = {p.head_stride, p.token_stride, p.page_stride, p.layer_stride};
  cuuint64_t bytes[4];
  for (int i = 0; i < 4; ++i) {  // an axis of one place is never stepped over: any stride will do
    bytes[i] = dims[i + 1] > 1 ? 2 * (cuuint64_t)stride[i] : 16;
    if (bytes[i] == 0 || bytes[i] >= (1ull << 40)) return false;
  }
  const cuuint32_t box[5] = {64, 1, (cuuint32_t)m->box, 1, 1}, step[5] = {1, 1, 1, 1, 1};
  const CUtensorMapDataType type = p.dtype == PS_KV_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  for (int i = 0; i < 2; ++i)
    if (encode(i ? &m->v : &m->k, type, 5, i ? p.v : p.k, dims, bytes, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return false;
  m->ok = 1;
  return true;
}
cudaError_t configure_wide(const Pool& p) {
  return p.dtype == PS_KV_BF16 ? configure_t<__nv_bfloat16>(p.head_dim) : configure_t<__half>(p.head_dim);
}

}  // namespace pskv
