// ps_kv_attention: the wide tiles (17 to 256 query rows of one request, or of
// the requests that share a prefix), on tcgen05.
//
// The mathematics is the narrow tiles' (ps_kv_attend.cu).  One CTA an SM takes
// its part of the list of units; a unit is 128 keys.  Its warps:
//   8 softmax warps, two groups t of four, a thread a query row;
//   4 loader warps, each with a quarter of every unit's keys and values: whole
//     units by TMA, a box for 16 tokens of a page and 64 elements, and the
//     queries, a box of 64 elements of 128 rows.  A
//     request's last unit, whose values past its end must read as zero, queries
//     of which 128 rows are not whole tokens, and pages of 2 or 4 tokens, whose
//     boxes would not fill the 1024 bytes after which the swizzle repeats, go by
//     16-byte asynchronous copies instead, eight times the instructions and
//     waited for by the copying threads: with them for all units the loader
//     warps took 7400 cycles a unit, and for queries alone 3400 a tile, in
//     which the next tile's products waited;
//   2 warps that issue the matrix instructions, one for each group (2 more idle).
// A tile of more than 128 rows is two row blocks, one for each group, that use
// every unit's keys and values (pair mode).  A tile of up to 128 rows is one
// row block; the groups take its units in turn, each with a softmax of its own
// over them, joined when the tile ends (split mode).
//
// Tensor memory: scores S_t (128 columns of 32 bits; the weights P_t overwrite
// the first 64 with pairs of 16 bits) and outputs O_t (up to 128 columns).
// S_t = Q K^T reads both operands from shared memory; O_t += P_t V takes P_t
// from tensor memory.  While group t computes weights, the other group's
// products run; the first half of its weights is multiplied while it computes
// the second (prompts 324 -> 308 us).  The maximum that the weights refer to moves only when a score
// passes it by 2^8: O_t is rescaled rarely, and the final division makes up for
// whichever reference was used.
//
// Bound by the chain of a unit: 2048 cycles of products for a pair's, 2700 to
// 2800 measured, of which the groups' turns, the waits between dependent
// products and the copies' share of shared memory are the rest; with the
// exponentials and most maxima left out they are 2560.  (Weights computed with
// the old reference beside the search for the maximum were no faster: 321 us;
// the groups without turns 343.)  A tile's ends cost some four units (tile_cost).
// 7000 new bf16 tokens after 2000 to 4900 cached ones, 32 heads of 128 on 8: a
// call takes 310 us on inputs that change, 1.29 PFLOP/s of the 1.88 that a
// library's plain product reaches, and 285 to 292 on one input again, whose
// queries are in L2 (the other figures for prompts here are of that kind); 128
// requests of one token after 16384 shared ones: 52 us by itself, on the 76 SMs
// that it has there.  The compiler spills 168 bytes of stores and 292 of loads a
// thread in every variant; in which warps' code was not looked into.
#include "ps_kv_attend.cuh"

namespace pskv {
namespace {

constexpr int kSoftmaxWarps = 8, kLoaderWarps = 4;
constexpr int kThreads = 512;  // four warpgroups: registers move between whole ones
constexpr int kSoftmaxRegs = 192, kOtherRegs = 64;  // 2 x 128 x (192 + 64) = 512 x 128, the launch's own
constexpr int UNIT = unit_keys(1), H = tile_rows(1);
__device__ __forceinline__ constexpr uint32_t col_s(int t) { return 128u * t; }
__device__ __forceinline__ constexpr uint32_t col_o(int t) { return 256u + 128u * t; }
constexpr float kRescale = 8.0f;
constexpr int kEarly = 64;  // keys of a unit whose weights are announced by themselves

template <int DP>
struct Shape {
  static constexpr int kHalves = DP > 64 ? 2 : 1;          // 64-element halves of a row
  static constexpr int kBlock = 128 * 128 * kHalves;       // bytes of 128 rows
  static constexpr int kBuffers = DP > 64 ? 5 : 10;        // ring of key and value blocks, in turn
  static constexpr int kSmem = 1024 + (2 + kBuffers) * kBlock;
  static constexpr int kSteps = DP / 16;                   // k steps of Q K^T
};

struct Shared {
  uint64_t full[10], empty[10], s_full[2], p_part[2], p_full[2], o_full[2], q_full[2], q_empty[2], ml_full, ml_free, turn[2];
  uint32_t tmem;
  float2 ml[128];  // split mode: group 1's (maximum, sum)
};

// ---- barriers, tensor memory ---------------------------------------------------
// Whether a wait would succeed, without waiting (try_wait may suspend the thread for thousands
// of cycles before it answers no).
__device__ __forceinline__ bool bar_peek(uint64_t* b, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{ .reg .pred p; mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
      : "=r"(ok) : "r"(smem_addr(b)), "r"(parity) : "memory");
  return ok != 0;
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
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// Descriptor of a block of 128-byte rows with the 128-byte swizzle.  Eight rows
// are 1024 bytes; 'lead' is the distance of the second 64-element half where the
// rows are the contraction's (values), unused where they are the result's.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lead) {
  return (uint64_t)(1024 >> 4 | 1u << 14 | 2u << 29) << 32 | (lead >> 4 << 16) | addr >> 4;
}
// Instruction descriptor: 32-bit sums of 16-bit products, 128 rows, n columns.
template <typename T>
__device__ __forceinline__ uint32_t instr_desc(int n, bool b_rows_contract) {
  const uint32_t type = sizeof(T) == 2 && Num<T>::kBf16 ? 1 : 0;
  return 1u << 4 | type << 7 | type << 10 | (b_rows_contract ? 1u << 16 : 0) | (uint32_t)(n >> 3) << 17 | (128u >> 4) << 24;
}

// Two row blocks?
__device__ __forceinline__ bool is_pair(const Tile& t) { return t.nrows > 128; }

// The two blocks of queries: both are a pair's, one is a single row block's, the
// other one next time, so that a tile's queries arrive while the last one's are
// in use.  'fills' bit b: parity of block b's fills so far.
struct QueryBlocks {
  uint32_t fills = 0, turn = 0;
  __device__ __forceinline__ uint32_t first(bool pair) const { return pair ? 0 : turn; }
  __device__ __forceinline__ void next(bool pair) {
    fills ^= pair ? 3u : 1u << turn;
    if (!pair) turn ^= 1;
  }
};

// ---- loader warps ------------------------------------------------------------------
// A place in the ring of blocks, and the parity of its use.
template <int N>
struct Place {
  uint32_t slot = 0, par = 0;
  __device__ __forceinline__ Place ahead(uint32_t n) const {  // n < N
    Place p;
    p.slot = slot + n;
    p.par = par;
    if (p.slot >= N) {
      p.slot -= N;
      p.par ^= 1;
    }
    return p;
  }
  __device__ __forceinline__ Place skip(uint32_t n) const {
    Place p;
    p.slot = (slot + n) % N;
    p.par = (par + (slot + n) / N) & 1;
    return p;
  }
};

// 32 rows of the warp's, row r at element off (of lane r; -1: zeros), as one
// group of asynchronous copies.
template <int DP>
__device__ __forceinline__ void copy_rows(uint32_t dst, const char* base, int64_t off, int head_dim) {
  constexpr int CH = DP / 8;                    // 16-byte words of a row that hold elements
  constexpr int RPI = 32 / (CH <= 8 ? 8 : 16);  // rows that one copy instruction covers
  const int lane = threadIdx.x & 31, row0 = (threadIdx.x >> 5 & 3) * 32;
  const int w = lane % (32 / RPI), sub = lane / (32 / RPI);
  const bool on = w * 8 < head_dim;
#pragma unroll 4
  for (int j = 0; j < 32; j += RPI) {
    const int64_t o = __shfl_sync(0xFFFFFFFFu, off, j + sub);
    const int r = row0 + j + sub;
    const bool ok = o >= 0 && on;
    // word w of row r: half w / 8, swizzled within its 128 bytes
    if (w < CH) cp16(dst + (w >> 3) * (128 * 128) + r * 128 + (((w & 7) ^ (r & 7)) << 4), base + (ok ? 2 * o + w * 16 : 0), ok);
  }
  cp_commit();
}

template <int DP>
__device__ __forceinline__ bool load_role(const AttendArgs& a, const PoolMaps& maps, Shared* sh, uint32_t qs, uint32_t ring, Parts<1> ps) {
  using S = Shape<DP>;
  static_assert(kSoftmaxWarps % 4 == 0, "copy_rows takes the warp's place in its group");
  const int lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) - kSoftmaxWarps;
  const bool tma = maps.ok;
  // TMA: lane i issues box i % boxes of the warp's keys, half i / boxes
  const int boxes = 32 / maps.box, mybox = lane % boxes, myhalf = lane / boxes;
  const bool issues = tma && lane < boxes * S::kHalves;
  const uint32_t box_at = myhalf * (128 * 128) + (warp * 32 + mybox * maps.box) * 128;
  Place<S::kBuffers> at;       // the next block
  uint64_t* copied[2] = {nullptr, nullptr};  // blocks whose copies are under way
  auto told = [&]() {                        // wait for them and say so
    if (!copied[0]) return;
    cp_wait<0>();
    to_async_proxy();
    __syncwarp();
    if (lane == 0) bar_arrive(copied[0]);
    if (lane == 0 && copied[1]) bar_arrive(copied[1]);
    copied[0] = copied[1] = nullptr;
  };
  QueryBlocks qb;
  bool more = true;
  for (; more; more = ps.next()) {
    const Tile t = ps.t;
    const int32_t* row = a.tables + t.req * a.table_stride;
    // A unit is read whole up to here: the keys that follow a causal tile's last
    // one are the request's own, and weigh nothing (see mend_row for what is not
    // finite among them).
    const int end = t.ctx == kNoMask ? t.kv1 : a.kv_lens[t.req];
    // ids are looked up one unit ahead
    auto id_of = [&](int u) -> int {
      const int base = t.kv0 + (ps.unit + u) * UNIT;
      const bool whole = tma && base + UNIT <= end;
      const int key = base + warp * 32 + (whole ? mybox * maps.box : lane);
      return u < ps.count && key < (whole ? end : t.kv1) ? __ldg(row + (key >> a.pool.page_log2)) : -1;
    };
    int page = id_of(0);
#pragma unroll 1
    for (int u = 0; u < ps.count; ++u) {
      const int base = t.kv0 + (ps.unit + u) * UNIT;
      const bool whole = tma && base + UNIT <= end;
      const int id = page;
      page = id_of(u + 1);
      const int key = base + warp * 32 + (whole ? mybox * maps.box : lane), token = key & (a.pool.page_size - 1);
      // keys, values; with a tile's first unit under way its queries (one loop, so
      // that the copies' code is there once)
      const int jobs = u > 0 ? 2 : (is_pair(ps.t) ? 4 : 3);
#pragma unroll 1
      for (int job = 0; job < jobs; ++job) {
        const uint32_t qblk = qb.first(is_pair(ps.t)) ^ (job & 1);  // of jobs 2 and 3
        uint64_t* bar = job < 2 ? &sh->full[at.slot] : &sh->q_full[qblk];
        uint64_t* free = job < 2 ? &sh->empty[at.slot] : &sh->q_empty[qblk];
        const uint32_t parity = (job < 2 ? at.par : qb.fills >> qblk & 1) ^ 1;
        if (!__all_sync(0xFFFFFFFFu, bar_peek(free, parity))) {
          told();  // what was copied is not held back by the wait
          if (!warp_wait(free, parity)) return false;
        }
        const char* src = job == 0 ? a.k : (job == 1 ? a.v : a.q);
        uint32_t dst;
        int64_t off;
        int qtok = 0;
        if (job < 2) {
          dst = ring + at.slot * S::kBlock;
          at = at.ahead(1);
          if (whole) {
            if (lane == 0) bar_expect(bar, 32 * 128 * S::kHalves);
            __syncwarp();
            if (issues) tma_load(dst + box_at, job ? &maps.v : &maps.k, bar, myhalf * 64, ps.head, token, id);
            continue;
          }
          off = id * a.pool.page_stride + (int64_t)token * a.pool.token_stride + (int64_t)ps.head * a.pool.head_stride;
          if (id < 0) off = -1;
        } else {
          const int r = (job - 2) * 128 + warp * 32 + lane, rr = t.row0 + r;
          dst = qs + qblk * S::kBlock;
          qtok = t.tok0 + (t.row0 + (job - 2) * 128) / a.pool.ratio;
          off = (int64_t)(t.tok0 + rr / a.pool.ratio) * a.q_stride[0] +
                (int64_t)(ps.head * a.pool.ratio + rr % a.pool.ratio) * a.q_stride[1];
          if (r >= t.nrows) off = -1;
        }
        if (job >= 2 && maps.q_ok) {
          if (warp == 0) {
            if (elect()) {
              bar_expect(bar, S::kBlock);
#pragma unroll
              for (int half = 0; half < S::kHalves; ++half)
                tma_load(dst + half * (128 * 128), &maps.q, bar, half * 64, 0, ps.head, qtok);
            }
          } else if (lane == 0) {
            bar_arrive(bar);
          }
          __syncwarp();
          continue;
        }
        if (job != 3) told();
        copy_rows<DP>(dst, src, off, a.pool.head_dim);
        copied[copied[0] ? 1 : 0] = bar;
      }
      told();
      if (u == 0) qb.next(is_pair(ps.t));
    }
  }
  told();
  return true;
}

// ---- the warps that issue the matrix instructions -------------------------------------
// One warp for each group t.  Every wait between products drains the warp's queue
// of them (some 200 cycles), which the other group's products fill.  The groups
// take turns: left to themselves they fell into step, both waiting for weights
// or both for products (4500 cycles for a unit's 2048 of products).
template <typename T, int DP>
__device__ __forceinline__ bool mma_role(const AttendArgs& a, Shared* sh, int t, uint32_t tmem, uint32_t qs, uint32_t ring, Parts<1> ps) {
  using S = Shape<DP>;
  // scores are negated where the scale is negative
  const uint32_t id_qk = instr_desc<T>(UNIT, false) | (a.scale2 < 0 ? 1u << 13 : 0), id_pv = instr_desc<T>(DP, true);
  // descriptors differ in their address field alone
  const uint64_t q_desc = smem_desc(qs, 16), k_desc = smem_desc(ring, 16), v_desc = smem_desc(ring, 128 * 128);
  constexpr uint32_t kBlk = S::kBlock >> 4;
  const uint32_t s_at = tmem + col_s(t), o_at = tmem + col_o(t);
  uint32_t p_phase = 0, turn = t ^ 1;  // group 0 has the first turn
  Place<S::kBuffers> at;  // the tile's first block: unit 0's keys, then its values, unit 1's keys ...
  QueryBlocks qb;
  bool more = true;
  for (; more; more = ps.next()) {
    const bool pair = is_pair(ps.t);
    const int n = ps.count;
    const uint32_t qblk = pair ? t : qb.first(false);
    if (!warp_wait(&sh->q_full[qblk], qb.fills >> qblk & 1)) return false;
    qb.next(pair);
    const uint64_t q = q_desc + qblk * kBlk;
    // a query block's two arrivals: both of the one group of a pair, one of each otherwise
    auto release_q = [&]() {
      tc_commit(&sh->q_empty[qblk]);
      if (pair) tc_commit(&sh->q_empty[qblk]);
    };
    // A key or value block's arrivals are one of each group: a group passes over
    // the blocks that the other one alone uses, so that it has seen every use of
    // a place in the ring (a wait tells a use from the one after next, no more).
    auto pass = [&](const Place<S::kBuffers>& b) {
      if (!warp_wait(&sh->full[b.slot], b.par)) return false;
      if (elect()) bar_arrive(&sh->empty[b.slot]);
      __syncwarp();
      return true;
    };
    Place<S::kBuffers> next = at;  // the first block that this group has not seen
    const int step = pair ? 1 : 2, first = pair ? 0 : t, turns = pair ? n : (n + 1) / 2;
    // Turn i: unit u's values, then the scores of this group's next unit (turn -1
    // is the first scores alone).  The blocks' waits come before the wait for the
    // weights, where there is time; the groups' turns alternate.
#pragma unroll 1
    for (int i = -1; i < turns; ++i) {
      const int u = first + i * step;
      const bool product = i >= 0 && u < n, more_keys = u + step < n;
      const Place<S::kBuffers> vb = next;
      if (product) {
        if (!warp_wait(&sh->full[vb.slot], vb.par)) return false;
        next = next.ahead(1);
      }
      if (!pair && u + 1 >= 0 && u + 1 < n) {  // the other group's unit
        if (!pass(next) || !pass(next.ahead(1))) return false;
        next = next.ahead(2);
      }
      const Place<S::kBuffers> kb = next;
      if (more_keys) {
        if (!warp_wait(&sh->full[kb.slot], kb.par)) return false;
        next = next.ahead(1);
      }
      if (product) {
        if (!warp_wait(&sh->p_part[t], p_phase)) return false;
      }
      if (!warp_wait(&sh->turn[t], turn)) return false;
      turn ^= 1;
      const uint64_t v = v_desc + vb.slot * kBlk;
      if (product) {
        tc_after();
        if (elect()) {
#pragma unroll
          for (int s = 0; s < kEarly / 16; ++s) mma_ts(o_at, s_at + s * 8, v + s * (2048 >> 4), id_pv, i > 0 || s > 0);
        }
        __syncwarp();
        if (!warp_wait(&sh->p_full[t], p_phase)) return false;
        p_phase ^= 1;
      }
      tc_after();
      if (elect()) {
        if (product) {
#pragma unroll
          for (int s = kEarly / 16; s < UNIT / 16; ++s) mma_ts(o_at, s_at + s * 8, v + s * (2048 >> 4), id_pv, true);
        }
        if (more_keys) {
          const uint64_t k = k_desc + kb.slot * kBlk;
#pragma unroll
          for (int s = 0; s < S::kSteps; ++s) {
            const int x = (s >> 2) * (128 * 128 >> 4) + (s & 3) * 2;
            mma_ss(s_at, q + x, k + x, id_qk, s > 0);
          }
          tc_commit(&sh->s_full[t]);
        } else if (product) {
          tc_commit(&sh->o_full[t]);
        }
        bar_arrive(&sh->turn[t ^ 1]);
        if (product) tc_commit(&sh->empty[vb.slot]);
        if (more_keys) tc_commit(&sh->empty[kb.slot]);
        if (more_keys && u + 2 * step >= n) release_q();  // the last scores are on their way
      }
      __syncwarp();
    }
    if (first >= n && elect()) release_q();  // no scores at all
    __syncwarp();
    at = at.skip(2 * n);
  }
  return true;
}

// ---- softmax warps ------------------------------------------------------------------
template <typename T, int DP>
__device__ __forceinline__ bool softmax_role(const AttendArgs& a, Shared* sh, uint32_t tmem, Parts<1> ps, int c, int C) {
  const int warp = threadIdx.x >> 5, t = warp >> 2, lane = threadIdx.x & 31;
  const int row = (warp & 3) * 32 + lane;  // of the row block, and the tensor memory lane
  const uint32_t at = tmem + ((uint32_t)(warp & 3) << 21);
  const uint32_t s_at = at + col_s(t), o_at = at + col_o(t);
  // a negative scale's sign is in the scores already; at a scale of 0 the least
  // one stands for it, so that hidden scores of -infinity stay what they are
  const float sc = fmaxf(fabsf(a.scale2), 1e-30f);
  uint32_t s_phase = 0, o_mine = 0, o_other = 0, ml_phase = 0;  // o_other: group 1's, as group 0 counts it
  bool held = false;  // group 1: the last tile's O_1 and ml may still be read by group 0
  auto let_go = [&]() {
    if (!held) return true;
    held = false;
    const bool ok = warp_wait(&sh->ml_free, ml_phase);
    ml_phase ^= 1;
    return ok;
  };
  bool more = true;
  for (; more; more = ps.next()) {
    const Tile tl = ps.t;
    const bool pair = is_pair(ps.t);
    const int n = ps.count;
    const int mine = pair ? n : (t == 0 ? (n + 1) / 2 : n / 2);
    const int trow = pair ? t * 128 + row : row;  // row of the tile
    const int rr = tl.row0 + trow;
    const int lim = min(tl.kv1, tl.ctx + 1 + rr / a.pool.ratio);
    float m = -INFINITY, l = 0;  // m: the scaled reference
    for (int i = 0; i < mine; ++i) {
      const int base = tl.kv0 + (ps.unit + (pair ? i : 2 * i + t)) * UNIT;
      if (!warp_wait(&sh->s_full[t], s_phase)) return false;
      s_phase ^= 1;
      tc_after();
      uint32_t raw[128];
#pragma unroll
      for (int j = 0; j < 128; j += 32) tm_load32(raw + j, s_at + j);
      tm_wait_ld();
      float* s = reinterpret_cast<float*>(raw);
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
#pragma unroll 1
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
        if (j + 32 == kEarly || j + 32 == UNIT) {
          tm_wait_st();
          if (j + 32 == kEarly && i == 0 && !let_go()) return false;
          tc_before();
          __syncwarp();
          if (lane == 0) bar_arrive(j + 32 == kEarly ? &sh->p_part[t] : &sh->p_full[t]);
        }
      }
      const float2 total = unpack2(add2(sum[0], sum[1]));
      l += total.x + total.y;
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
      if (!warp_wait(&sh->ml_full, ml_phase)) return false;
      ml_phase ^= 1;
      const float2 x = sh->ml[row];
      const float mn = fmaxf(m, x.x), ref = mn == -INFINITY ? 0.0f : mn;
      f[0] = ex2(m - ref);
      f[1] = ex2(x.x - ref);
      l = l * f[0] + x.y * f[1];
      m = mn;
    }
    if (!warp_wait(&sh->o_full[t], o_mine)) return false;
    o_mine ^= 1;
    const bool both = !pair && n > 1;
    if (both && !warp_wait(&sh->o_full[1], o_other)) return false;
    if (pair || n > 1) o_other ^= 1;
    tc_after();
    const bool direct = whole && tl.sidx < 0;
    const bool in = trow < tl.nrows;
    const int64_t tok = tl.tok0 + rr / a.pool.ratio;
    const int hq = ps.head * a.pool.ratio + rr % a.pool.ratio;
    const float inv = l > 0 ? 1.0f / l : (l == 0 ? 0.0f : l);
    const int64_t out_at = in ? tok * a.out_stride[0] + (int64_t)hq * a.out_stride[1] : -1;
    const int64_t prow = part_row<H>(tl.sidx, tl.nrows, ps.head, c, ps.unit > 0, C) + trow;
    // where this lane writes: four lanes exchange words so that each has the
    // same 16 bytes of four rows, and they write 64 bytes of a row together
    int64_t rows_at[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) rows_at[x] = __shfl_sync(0xFFFFFFFFu, out_at, (lane & ~3) + x);
    float z = 0;
#pragma unroll 1
    for (int j = 0; j < DP; j += 32) {
      uint32_t o[32];
      tm_load32(o, o_at + j);
      tm_wait_ld();
      float* x = reinterpret_cast<float*>(o);
      if (!pair) {
#pragma unroll
        for (int e = 0; e < 32; ++e) x[e] *= f[0];
        if (both) {
          uint32_t o1[32];
          tm_load32(o1, at + col_o(1) + j);
          tm_wait_ld();
#pragma unroll
          for (int e = 0; e < 32; ++e) x[e] += __uint_as_float(o1[e]) * f[1];
        }
      }
      if (direct) {
        // (where DP is not whole times 32 the last columns are past the products' and hold anything)
#pragma unroll
        for (int e = 0; e < 32; e += 8)
          if (DP % 32 == 0 || j + e < DP) {
#pragma unroll
            for (int i = 0; i < 8; ++i) z = spoil(z, x[e + i]);
          }
        uint32_t w[4][4];
#pragma unroll
        for (int e = 0; e < 32; e += 2) w[e >> 3][(e >> 1) & 3] = Num<T>::pack(x[e] * inv, x[e + 1] * inv);
#pragma unroll
        for (int b = 1; b <= 2; b <<= 1) {
          const bool up = lane & b;
#pragma unroll
          for (int c4 = 0; c4 < 4; ++c4) {
            if (c4 & b) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t got = __shfl_xor_sync(0xFFFFFFFFu, up ? w[c4][e] : w[c4 | b][e], b);
              if (up) w[c4][e] = got;
              else w[c4 | b][e] = got;
            }
          }
        }
        const int col = j + (lane & 3) * 8;
#pragma unroll
        for (int y = 0; y < 4; ++y)
          if (rows_at[y] >= 0 && col < a.pool.head_dim)
            *reinterpret_cast<uint4*>(a.out + 2 * (rows_at[y] + col)) = make_uint4(w[y][0], w[y][1], w[y][2], w[y][3]);
      } else if (in) {
#pragma unroll
        for (int e = 0; e < 32; e += 4)
          if (j + e < a.pool.head_dim)
            a.plan.part_o[1][part_word(prow, (j + e) >> 2, a.pool.head_dim)] = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
      }
    }
    if (in) {
      if (a.causal && z != 0) ask_mend(a, 1, ps.tile, ps.head);
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
  // the plan is read before the wait, as in k_attend_narrow; the CTAs that have no
  // part wait too, since the narrow tiles' kernel counts on it
  const PlanHdr* hdr = a.plan.hdr;
  const int C = hdr->workers[1], c = blockIdx.x;
  const int64_t U = hdr->cost[1];
  Parts<1> ps;
  if (c >= C || !ps.start(a.plan, a.pool.kv_heads, c, U * c / C, U * (c + 1) / C)) {
    chain();
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t qs = (smem_addr(dyn) + 1023) & ~1023u, ring = qs + 2 * S::kBlock;
  if (warp == kSoftmaxWarps + kLoaderWarps) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&sh.tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (threadIdx.x == 0) {
    for (int b = 0; b < S::kBuffers; ++b) {
      bar_init(&sh.full[b], kLoaderWarps);
      bar_init(&sh.empty[b], 2);
    }
    for (int t = 0; t < 2; ++t) {
      bar_init(&sh.s_full[t], 1);
      bar_init(&sh.p_part[t], 4);
      bar_init(&sh.p_full[t], 4);
      bar_init(&sh.o_full[t], 1);
      bar_init(&sh.turn[t], 1);
      bar_init(&sh.q_full[t], kLoaderWarps);
      bar_init(&sh.q_empty[t], 2);
    }
    bar_init(&sh.ml_full, 4);
    bar_init(&sh.ml_free, 4);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  tc_before();
  __syncthreads();
  tc_after();
  const uint32_t tmem = sh.tmem;
  chain();
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
  } else if (warp >= kSoftmaxWarps + kLoaderWarps && warp < kSoftmaxWarps + kLoaderWarps + 2) {
    ok = mma_role<T, DP>(a, &sh, warp & 1, tmem, qs, ring, ps);
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
  return launch(k_attend_wide<T, DP>, dim3((unsigned)a.plan.max_workers[1]), kThreads, Shape<DP>::kSmem, st, a, m);
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

namespace {
struct Axis {
  int64_t size, stride;  // stride in elements
  uint32_t box;
};
bool encode_map(CUtensorMap* map, int32_t dtype, const void* base, const Axis* axes, int n) {
  static const auto encode = []() -> decltype(&cuTensorMapEncodeTiled) {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      return nullptr;
    return reinterpret_cast<decltype(&cuTensorMapEncodeTiled)>(fn);
  }();
  if (!encode) return false;
  cuuint64_t dims[5], bytes[5];
  cuuint32_t box[5], step[5];
  for (int i = 0; i < n; ++i) {
    dims[i] = (cuuint64_t)axes[i].size;
    box[i] = axes[i].box;
    step[i] = 1;
    if (i == 0) continue;
    // an axis of one place is never stepped over: any stride will do
    bytes[i - 1] = axes[i].size > 1 ? 2 * (cuuint64_t)axes[i].stride : 16;
    if (bytes[i - 1] == 0 || bytes[i - 1] >= (1ull << 40)) return false;
  }
  return encode(map, dtype == PS_KV_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, (cuuint32_t)n,
                const_cast<void*>(base), dims, bytes, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
}  // namespace

bool make_maps(const Pool& p, int32_t layer, PoolMaps* m) {
  m->ok = m->whole = m->q_ok = 0;
  m->box = p.page_size < 16 ? p.page_size : 16;
  if (p.page_size < 8) return false;
  const int parts = p.head_dim / 64;
  auto make = [&](CUtensorMap* map, void* base, const Axis* axes, int n) { return encode_map(map, p.dtype, base, axes, n); };
  const uint32_t tokens = (uint32_t)m->box;
  const Axis head = {p.kv_heads, p.head_stride, 1}, page = {p.num_pages, p.page_stride, 1},
             token = {p.page_size, p.token_stride, tokens};
  const Axis plain[4] = {{p.head_dim, 1, 64}, head, token, page};
  const Axis whole[5] = {{64, 1, 64}, token, {parts, 64, (uint32_t)parts}, head, page};
  char *k = p.k + 2 * layer * p.layer_stride, *v = p.v + 2 * layer * p.layer_stride;
  m->ok = make(&m->k, k, plain, 4) && make(&m->v, v, plain, 4);
  m->whole = m->ok && p.head_dim == 64 * parts && make(&m->whole_k, k, whole, 5) && make(&m->whole_v, v, whole, 5);
  return m->ok != 0;
}
// The queries' map, where a block of 128 rows is whole tokens.
void make_query_map(const Pool& p, const void* q, const int64_t* stride, int32_t tokens, PoolMaps* m) {
  m->q_ok = 0;
  if (p.ratio > 128 || 128 % p.ratio != 0) return;
  const Axis axes[4] = {{p.head_dim, 1, 64}, {p.ratio, stride[1], (uint32_t)p.ratio}, {p.kv_heads, p.ratio * stride[1], 1},
                        {tokens, stride[0], (uint32_t)(128 / p.ratio)}};
  m->q_ok = encode_map(&m->q, p.dtype, q, axes, 4);
}
cudaError_t configure_wide(const Pool& p) {
  return p.dtype == PS_KV_BF16 ? configure_t<__nv_bfloat16>(p.head_dim) : configure_t<__half>(p.head_dim);
}

}  // namespace pskv
