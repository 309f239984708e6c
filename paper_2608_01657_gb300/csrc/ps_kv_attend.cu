// ps_kv_attention: the narrow tiles (up to 16 query rows, mma) and the join of
// partial results.  The wide tiles are in ps_kv_attend_wide.cu.
//
// The mathematics, for one query row and the keys j that it sees:
//   t_j = scale log2(e) q k_j,  m = max t_j,  l = sum 2^(t_j - m),
//   o = sum 2^(t_j - m) v_j / l,
// kept as (m, l, sum) over a growing set of keys: a new key set's maximum m'
// scales what was there by 2^(m - max(m, m')), and two sets' (m, l, sum) join
// the same way.  m, l and the sums are in 32 bits; the weights 2^(t - m) are
// rounded to the pool's type for the product with V, as the matrix
// instructions want them.
#include "ps_kv_attend.cuh"

namespace pskv {
namespace {

constexpr int kThreads = 128;
constexpr int kWarps = kNarrowWarps;

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <typename T>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma<__nv_bfloat16>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma<__half>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void after_wide() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Shared memory of a warp: STAGES x (16 keys, 16 values), each as halves of 64
// elements, 16 rows of 128 bytes in which a 16-byte word c of row r lies at word
// c ^ (r & 7) (the copies' 128-byte swizzle), so that the eight rows of an
// ldmatrix lie in eight different bank groups.
template <int DP>
struct Shape {
  static constexpr int kHalves = DP > 64 ? 2 : 1;
  static constexpr int kBlock = kHalves * 16 * 128;  // bytes of 16 keys, or values
  static constexpr int kStages = DP <= 64 ? 6 : 3;
  static constexpr int kWarpBytes = kStages * 2 * kBlock;
  // two CTAs an SM: 113 KB each at most
  static constexpr int kSmem = kWarps * kWarpBytes + kWarps * kStages * 8;
  static_assert(2 * (kSmem + 1024) <= 228 * 1024, "two CTAs an SM");
};
// Place of word c of row r in a block.
__device__ __forceinline__ uint32_t word_at(int r, int c) { return (c >> 3) * (16 * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4); }

// Narrow tiles: decode.  Bound by HBM (a key is used by at most 16 rows).  Every
// warp is a worker of its own: it streams its keys and values, 16 at a time,
// through its own ring of stages, with no barrier (four warps to a (tile, head),
// joined where it ends, waited 3400 to 5600 cycles for one another there, two
// units' time).  The stream runs on across tiles, so that short requests do not
// drain it.  Keys and values come by TMA: a box of whole heads for 16 keys where
// heads are 64 or 128 elements, else one for every 64 elements; pages of 2 or 4
// tokens, whose boxes would not fill the 1024 bytes after which the swizzle
// repeats, by 16-byte copies.  256 requests of one token, 2.27 GB of bf16 keys
// and values: 341 us, 6.5 TB/s of the 6.8 that copies reach; one request of 700 keys: 4 us, its chain of reads.
template <typename T, int DP>
__global__ void __launch_bounds__(kThreads, 2) k_attend_narrow(const __grid_constant__ AttendArgs a,
                                                               const __grid_constant__ PoolMaps maps) {
  using S = Shape<DP>;
  constexpr int CH = DP / 8;   // 16-byte words of a row
  constexpr int KS = DP / 16;  // k steps of q k^T
  constexpr int H = tile_rows(0), UNIT = unit_keys(0);
  extern __shared__ __align__(1024) char smem[];  // the swizzle repeats after 1024 bytes
  // If the wide tiles' kernel goes before this one, it is independent of it, so
  // this one's CTAs run as soon as there is room: every CTA of that kernel has
  // waited for the work before both by then.  Its end is waited for at this
  // one's end instead, so that the join after this kernel follows both.
  // The plan and the tables are there before either wait: the kernel before this
  // one has at least waited for the plan's tiles (see k_plan_joins).
  if (a.after_wide) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const PlanHdr* hdr = a.plan.hdr;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // the first workers of all CTAs, then the second ones: few are spread over many SMs
  const int C = hdr->workers[0], c = (int)blockIdx.x < hdr->narrow_ctas ? (int)blockIdx.x + warp * hdr->narrow_ctas : C;
  const int64_t U = hdr->cost[0];
  Parts<0> ps;
  if (c >= C || !ps.start(a.plan, a.pool.kv_heads, c, U * c / C, U * (c + 1) / C)) {
    after_wide();
    return;
  }
  const uint32_t ring = smem_addr(smem) + warp * S::kWarpBytes;
  uint64_t* landed = reinterpret_cast<uint64_t*>(smem + kWarps * S::kWarpBytes) + warp * S::kStages;
  const bool tma = maps.ok;
  if (lane == 0) {
    for (int i = 0; i < S::kStages; ++i) bar_init(&landed[i], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();

  // ---- the loader: runs STAGES - 1 units ahead ----
  Parts<0> lp = ps;
  bool lmore = true;
  int lkey, lend, lkv1;      // the loader's first key, the end of its units, the end of the keys
  const int32_t* lrow;       // page ids of the request
  auto enter = [&]() {
    lkey = lp.t.kv0 + lp.unit * UNIT;
    lend = lkey + lp.count * UNIT;
    lkv1 = lp.t.kv1;
    lrow = a.tables + lp.t.req * a.table_stride;
  };
  enter();
  const char* kbase = a.k;
  const char* vbase = a.v;
  // by TMA, lane i looks up box i's page; otherwise lane i key i's
  const int boxes = maps.box == 8 ? 2 : 1;
  const int mykey = tma ? (lane == 1 && boxes == 2 ? 8 : 0) : lane & 15;  // within a unit
  // page id of this lane's key in the loader's unit, -1 past the end
  auto key_page = [&]() -> int {
    const int t = lkey + mykey;
    return t < lkv1 ? __ldg(lrow + (t >> a.pool.page_log2)) : -1;
  };
  int page = key_page();
  int lstage = 0;
  auto load_unit = [&]() {
    if (lmore) {
      const int token = (lkey + mykey) & (a.pool.page_size - 1);
      const uint32_t dst = ring + lstage * 2 * S::kBlock;
      if (tma) {
        uint64_t* bar = &landed[lstage];
        if (lkey >= lkv1) {
          // a tile without keys
        } else if (boxes == 1) {  // every lane has the one page
          if (elect()) {
            bar_expect(bar, 2 * S::kBlock);
            if (maps.whole) {
              tma_load_whole(dst, &maps.whole_k, bar, lp.head, token, page);
              tma_load_whole(dst + S::kBlock, &maps.whole_v, bar, lp.head, token, page);
            } else {
#pragma unroll
              for (int half = 0; half < S::kHalves; ++half) {
                tma_load(dst + half * (16 * 128), &maps.k, bar, half * 64, lp.head, token, page);
                tma_load(dst + S::kBlock + half * (16 * 128), &maps.v, bar, half * 64, lp.head, token, page);
              }
            }
          }
          __syncwarp();
        } else {  // two pages of 8 tokens, the second only if it has a key
          const int there = lkey + 8 < lkv1 ? 2 : 1;
#pragma unroll 1
          for (int box = 0; box < there; ++box) {
            const int id = __shfl_sync(0xFFFFFFFFu, page, box);
            if (elect()) {
              if (box == 0) bar_expect(bar, there * S::kBlock);
              const uint32_t d = dst + box * (8 * 128);
#pragma unroll
              for (int half = 0; half < S::kHalves; ++half) {
                tma_load(d + half * (16 * 128), &maps.k, bar, half * 64, lp.head, 0, id);
                tma_load(d + S::kBlock + half * (16 * 128), &maps.v, bar, half * 64, lp.head, 0, id);
              }
            }
            __syncwarp();
          }
        }
      } else {
        int64_t off = -1;
        if (page >= 0)
          off = page * a.pool.page_stride + (int64_t)token * a.pool.token_stride + lp.head * a.pool.head_stride;
#pragma unroll
        for (int j = 0; j < 16 * CH / 32; ++j) {
          const int idx = j * 32 + lane, row = idx / CH, w = idx % CH;
          const int64_t o = __shfl_sync(0xFFFFFFFFu, off, row);
          const bool ok = o >= 0 && w * 8 < a.pool.head_dim;
          const int64_t at = ok ? 2 * o + w * 16 : 0;
          const uint32_t d = dst + word_at(row, w);
          cp16(d, kbase + at, ok);
          cp16(d + S::kBlock, vbase + at, ok);
        }
      }
      lkey += UNIT;
      if (lkey == lend) {
        lmore = lp.next();
        if (lmore) enter();
      }
      if (lmore) page = key_page();
    }
    if (!tma) cp_commit();
    lstage = lstage + 1 == S::kStages ? 0 : lstage + 1;
  };
  if (!a.after_wide) chain();
#pragma unroll
  for (int s = 0; s < S::kStages - 1; ++s) load_unit();

  // ---- the consumer ----
  int stage = 0;
  uint32_t phases = 0;  // bit i: parity of stage i's next landing
  bool ok = true;
  const int g = lane >> 2, q4 = lane & 3;
  for (bool more = true; more; more = ps.next()) {
    const Tile t = ps.t;
    const int head = ps.head;
    // queries of the 16 rows, as the A operand
    uint32_t qf[KS][4];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const int r = g + 8 * hf;
      const bool in = r < t.nrows;
      const int rr = t.row0 + (in ? r : 0);
      const char* qp = a.q + 2 * ((int64_t)(t.tok0 + rr / a.pool.ratio) * a.q_stride[0] +
                                  (int64_t)(head * a.pool.ratio + rr % a.pool.ratio) * a.q_stride[1]);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int e = ks * 16 + q4 * 2;
        qf[ks][hf] = in && e < a.pool.head_dim ? *reinterpret_cast<const uint32_t*>(qp + 2 * e) : 0u;
        qf[ks][hf + 2] = in && e + 8 < a.pool.head_dim ? *reinterpret_cast<const uint32_t*>(qp + 2 * e + 16) : 0u;
      }
    }
    // the keys before lim[.] are seen by rows g and g + 8; those before lim0 by all
    const int lim0 = min(t.kv1, t.ctx + 1 + t.row0 / a.pool.ratio);
    const int lim[2] = {min(t.kv1, t.ctx + 1 + (t.row0 + g) / a.pool.ratio),
                        min(t.kv1, t.ctx + 1 + (t.row0 + g + 8) / a.pool.ratio)};
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0, 0};
    float o[DP / 8][4];
#pragma unroll
    for (int i = 0; i < DP / 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[i][j] = 0;

    const int first = ps.unit, count = ps.count;
    for (int it = 0; it < count; ++it) {
      const int base = t.kv0 + (first + it) * UNIT;
      const int keys = t.kv1 - base;
      if (!tma) {
        cp_wait<S::kStages - 2>();
      } else if (keys > 0) {
        ok = ok && bar_wait(&landed[stage], phases >> stage & 1);
        phases ^= 1u << stage;
      }
      __syncwarp();  // the unit has landed, and the stage of the one before it is read
      load_unit();
      if (keys > 0) {
        const uint32_t ks_at = ring + stage * 2 * S::kBlock, vs_at = ks_at + S::kBlock;
        if (tma && keys < 16) {  // what lies past the end must weigh nothing: zeros for the values
          for (int i = lane; i < (16 - keys) * CH; i += 32)
            asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(vs_at + word_at(keys + i / CH, i % CH)), "r"(0) : "memory");
          to_async_proxy();
          __syncwarp();
        }
        // two sums a score, of even and odd steps: half the products' latency
        float s[2][4] = {}, s1[2][4] = {};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          uint32_t b[4];
          const int row = (lane & 7) + ((lane >> 4) << 3), w = 2 * ks + ((lane >> 3) & 1);
          ldsm4(b, ks_at + word_at(row, w));
          mma<T>(ks & 1 ? s1[0] : s[0], qf[ks], b[0], b[1]);
          mma<T>(ks & 1 ? s1[1] : s[1], qf[ks], b[2], b[3]);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) s[i][j] += s1[i][j];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) s[i][j] *= a.scale2;
        if (base + 16 > lim0) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (base + i * 8 + q4 * 2 + (j & 1) >= lim[j >> 1]) s[i][j] = -INFINITY;
        }
        bool grew = false;
        float mn[2], ms[2];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          float x = fmaxf(fmaxf(s[0][2 * hf], s[0][2 * hf + 1]), fmaxf(s[1][2 * hf], s[1][2 * hf + 1]));
          x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, 1));
          x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, 2));
          mn[hf] = fmaxf(m[hf], x);
          grew = grew || mn[hf] > m[hf];
          ms[hf] = mn[hf] == -INFINITY ? 0.0f : mn[hf];
        }
        if (__any_sync(0xFFFFFFFFu, grew)) {
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const float f = ex2(m[hf] - ms[hf]);
            l[hf] *= f;
#pragma unroll
            for (int i = 0; i < DP / 8; ++i) {
              o[i][2 * hf] *= f;
              o[i][2 * hf + 1] *= f;
            }
            m[hf] = mn[hf];
          }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            s[i][j] = ex2(s[i][j] - ms[j >> 1]);
            l[j >> 1] += s[i][j];
          }
        const uint32_t pf[4] = {Num<T>::pack(s[0][0], s[0][1]), Num<T>::pack(s[0][2], s[0][3]),
                                Num<T>::pack(s[1][0], s[1][1]), Num<T>::pack(s[1][2], s[1][3])};
#pragma unroll
        for (int np = 0; np < DP / 16; ++np) {
          uint32_t b[4];
          const int row = (lane & 7) + (((lane >> 3) & 1) << 3), w = 2 * np + (lane >> 4);
          ldsm4t(b, vs_at + word_at(row, w));
          mma<T>(o[2 * np], pf, b[0], b[1]);
          mma<T>(o[2 * np + 1], pf, b[2], b[3]);
        }
      }
      stage = stage + 1 == S::kStages ? 0 : stage + 1;
    }

#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      l[hf] += __shfl_xor_sync(0xFFFFFFFFu, l[hf], 1);
      l[hf] += __shfl_xor_sync(0xFFFFFFFFu, l[hf], 2);
    }
    {
      const bool whole = first == 0 && count == ps.nunits;
      if (whole && t.sidx < 0) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const int r = g + 8 * hf;
          if (r < t.nrows) {
            const int rr = t.row0 + r;
            const int64_t tok = t.tok0 + rr / a.pool.ratio;
            const int hq = head * a.pool.ratio + rr % a.pool.ratio;
            const float inv = l[hf] > 0 ? 1.0f / l[hf] : (l[hf] == 0 ? 0.0f : l[hf]);
            char* op = a.out + 2 * (tok * a.out_stride[0] + (int64_t)hq * a.out_stride[1]);
            float z = 0;
#pragma unroll
            for (int i = 0; i < DP / 8; ++i) z = spoil(spoil(z, o[i][2 * hf]), o[i][2 * hf + 1]);
            if (a.causal && z != 0) ask_mend(a, 0, ps.tile, head);
#pragma unroll
            for (int i = 0; i < DP / 8; ++i)
              if (i * 8 < a.pool.head_dim)
                *reinterpret_cast<uint32_t*>(op + 2 * (i * 8 + q4 * 2)) =
                    Num<T>::pack(o[i][2 * hf] * inv, o[i][2 * hf + 1] * inv);
            if (a.lse && q4 == 0) a.lse[tok * a.pool.q_heads + hq] = log_sum(m[hf], l[hf]);
          }
        }
      } else {
        const int64_t prow = part_row<H>(t.sidx, t.nrows, head, c, first > 0, C);
        float2* pml = a.plan.part_ml[0] + prow;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const int r = g + 8 * hf;
          if (r < t.nrows) {
#pragma unroll
            for (int i = 0; i < DP / 8; ++i)
              if (i * 8 < a.pool.head_dim)
                reinterpret_cast<float2*>(a.plan.part_o[0] + part_word(prow + r, 2 * i + (q4 >> 1), a.pool.head_dim))[q4 & 1] =
                    make_float2(o[i][2 * hf], o[i][2 * hf + 1]);
            if (q4 == 0) pml[r] = make_float2(m[hf], l[hf]);
          }
        }
      }
    }
  }
  cp_wait<0>();
  if (!ok && lane == 0) set_error(a.status, PS_ERR_TIMEOUT);
  after_wide();
}

// ---- the join --------------------------------------------------------------------
// A warp for eight rows of a (tile, head) that has partial results, lane = row +
// 8 (word mod 4): their own tile's parts, then their group's prefix's, in workers'
// order.  Bound by the latency of its dependent reads (the entry; then each
// part's maximum, sum and outputs, written just before and so in L2; the parts'
// reads do not depend on one another).  The entries are read before the wait for
// the tiles' kernels (one request's token: 11.9 us a call with them read after
// it and the tiles' kernels reading their plan after theirs, 9.6 so).  SPLIT
// kJoinWarps: the warps of a CTA take an equal share of the parts each, for when
// there are fewer rows than warps.  256 requests' rows: 8 us.
constexpr int kJoinWords = PS_KV_MAX_HEAD_DIM / 16;  // of a lane
constexpr int kJoinWarps = 4;                         // of a CTA
struct JoinShared {
  float4 o[kJoinWarps - 1][kJoinWords][32];
  float2 ml[kJoinWarps - 1][32];
};

// Numbers that are not finite among the values of tokens that a row does not
// see.  The matrix products give those tokens the weight 0, and 0 times infinity
// is NaN: only the last tokens of a tile are hidden from some of its rows, so
// only a prompt's rows can be spoilt, and only elements that are not finite in
// the result.  Those of a row whose hidden values have such a number there, and
// whose own token's value is not NaN itself, are computed again by a warp over the keys that
// the row sees alone: a lane a key for the scores, a lane four elements for the
// sum.  None of it runs on finite data.
template <typename T>
__device__ __forceinline__ uint32_t not_finite(uint2 x) {
  const float2 a = Num<T>::unpack(x.x), b = Num<T>::unpack(x.y);
  return (spoil(0, a.x) != 0 ? 1u : 0u) | (spoil(0, a.y) != 0 ? 2u : 0u) | (spoil(0, b.x) != 0 ? 4u : 0u) |
         (spoil(0, b.y) != 0 ? 8u : 0u);
}
template <typename T>
__device__ __noinline__ void mend_row(const AttendArgs& a, int tok0, int row, int head, int lane) {
  const Pool& p = a.pool;
  const int tok = tok0 + row / p.ratio, hq = head * p.ratio + row % p.ratio;
  const int req = a.plan.tok_req[tok], q0 = a.q_offsets[req], len = a.kv_lens[req];
  const int seen = max(len - (a.q_offsets[req + 1] - q0) + tok - q0 + 1, 0);
  const bool mine = 4 * lane < p.head_dim;
  uint2* op = reinterpret_cast<uint2*>(a.out + 2 * (tok * a.out_stride[0] + hq * a.out_stride[1])) + lane;
  auto at = [&](int key) {  // element 0 of a key of this head
    const int64_t page = a.tables[req * a.table_stride + (key >> p.page_log2)];
    return 2 * (page * p.page_stride + (key & (p.page_size - 1)) * p.token_stride + head * p.head_stride);
  };
  auto value = [&](int key) { return mine ? *reinterpret_cast<const uint2*>(a.v + at(key) + 8 * lane) : make_uint2(0, 0); };
  __syncwarp();
  const uint2 was = mine ? __ldcg(op) : make_uint2(0, 0);
  uint32_t redo = not_finite<T>(was), hidden = 0;
  if (seen > 0) {
    const uint2 own = value(seen - 1);
    const float2 x = Num<T>::unpack(own.x), y = Num<T>::unpack(own.y);
    redo &= (x.x == x.x ? 1u : 0u) | (x.y == x.y ? 2u : 0u) | (y.x == y.x ? 4u : 0u) | (y.y == y.y ? 8u : 0u);
  }
  if (!__any_sync(0xFFFFFFFFu, redo)) return;
  for (int k = seen; k < min(len, seen + tile_rows(1) + unit_keys(1)); ++k) hidden |= not_finite<T>(value(k));
  redo &= hidden;
  if (!__any_sync(0xFFFFFFFFu, redo)) return;
  const char* qp = a.q + 2 * (tok * a.q_stride[0] + hq * a.q_stride[1]);
  float m = -INFINITY, l = 0;
  float4 o = make_float4(0, 0, 0, 0);
  for (int k0 = 0; k0 < seen; k0 += 32) {
    float t = -INFINITY;
    if (k0 + lane < seen) {
      const char* kp = a.k + at(k0 + lane);
      float dot = 0;
      for (int e = 0; e < p.head_dim; e += 2) {
        const float2 x = Num<T>::unpack(*reinterpret_cast<const uint32_t*>(qp + 2 * e));
        const float2 y = Num<T>::unpack(*reinterpret_cast<const uint32_t*>(kp + 2 * e));
        dot = fmaf(x.y, y.y, fmaf(x.x, y.x, dot));
      }
      t = dot * a.scale2;
    }
    float mn = t;
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) mn = fmaxf(mn, __shfl_xor_sync(0xFFFFFFFFu, mn, x));
    mn = fmaxf(mn, m);
    const float ref = mn == -INFINITY ? 0.0f : mn, f = ex2(m - ref), w = ex2(t - ref);
    m = mn;
    l = l * f + w;  // the lane's own keys
    o.x *= f, o.y *= f, o.z *= f, o.w *= f;
    for (int j = 0; j < min(32, seen - k0); ++j) {
      const float wj = __shfl_sync(0xFFFFFFFFu, w, j);
      const uint2 v = value(k0 + j);
      const float2 lo = Num<T>::unpack(v.x), hi = Num<T>::unpack(v.y);
      o.x = fmaf(wj, lo.x, o.x);
      o.y = fmaf(wj, lo.y, o.y);
      o.z = fmaf(wj, hi.x, o.z);
      o.w = fmaf(wj, hi.y, o.w);
    }
  }
#pragma unroll
  for (int x = 1; x < 32; x <<= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, x);
  const float inv = l > 0 ? 1.0f / l : (l == 0 ? 0.0f : l);
  const uint32_t lo = Num<T>::pack(o.x * inv, o.y * inv), hi = Num<T>::pack(o.z * inv, o.w * inv);
  const uint32_t keep_lo = (redo & 1 ? 0u : 0xFFFFu) | (redo & 2 ? 0u : 0xFFFF0000u);
  const uint32_t keep_hi = (redo & 4 ? 0u : 0xFFFFu) | (redo & 8 ? 0u : 0xFFFF0000u);
  if (redo) *op = make_uint2((was.x & keep_lo) | (lo & ~keep_lo), (was.y & keep_hi) | (hi & ~keep_hi));
}
// The rows of the tiles that asked for it: those that wrote their outputs themselves.
template <typename T, int LIST>
__device__ __forceinline__ void mend_tiles(const AttendArgs& a, int64_t warp, int64_t warps, int lane) {
  constexpr int W = tile_rows(LIST) / 8;  // eight rows at a time
  const int64_t n = (int64_t)a.plan.hdr->ntiles[LIST] * a.pool.kv_heads;
  for (int64_t i = warp; i < n * W; i += warps) {
    if (!__ldcg(a.plan.mend[LIST] + i / W)) continue;
    const Tile& t = a.plan.tiles[LIST][i / W / a.pool.kv_heads];
    if (t.sidx >= 0) continue;  // its rows are the join's, and its byte is not kept
    const int r0 = (int)(i % W) * 8;
    for (int r = r0; r < min(t.nrows, r0 + 8); ++r) mend_row<T>(a, t.tok0, t.row0 + r, (int)(i / W % a.pool.kv_heads), lane);
  }
}

template <typename T, int H, int SPLIT>
__device__ __forceinline__ void join_rows(const AttendArgs& a, JoinShared* sh, bool* waited, int list, int entries,
                                          int64_t item0, int64_t step, int sub, int lane) {
  const int dim = a.pool.head_dim, words = dim >> 2;
  constexpr int W = H / 8, NW = kJoinWords;  // warps of an entry
  for (int64_t it = item0; it < (int64_t)entries * W; it += step) {
    static_assert(sizeof(JoinRec) == 80, "one word a lane");
    const int word = lane < 20 ? __ldg(reinterpret_cast<const int*>(a.plan.joins[list] + it / W) + lane) : 0;
    auto field = [&](int i) { return __shfl_sync(0xFFFFFFFFu, word, i); };
    const int nrows = field(14);
    const int r = (int)(it % W) * 8 + (lane & 7), c0 = lane >> 3;
    if (r - (lane & 7) >= nrows) continue;  // the whole warp, and with SPLIT the whole CTA
    const Parts4 own = {field(0), field(1), field(2), field(3)};
    const Parts4 pa = {field(4), field(5), field(6), field(7)}, pb = {field(8), field(9), field(10), field(11)};
    const int tok0 = field(12), row0 = field(13), head = field(15);
    const int plist = field(16), pofs = field(17), psplit = field(18);
    const bool in = r < nrows;
    if (!*waited) chain();
    *waited = true;
    float m = -INFINITY, l = 0;
    float4 o[NW];
#pragma unroll
    for (int i = 0; i < NW; ++i) o[i] = make_float4(0, 0, 0, 0);
    auto take = [&](float mx, float lx, const float4 (&v)[NW]) {
      const float mn = fmaxf(m, mx), ref = mn == -INFINITY ? 0.0f : mn;
      const float f0 = ex2(m - ref), f1 = ex2(mx - ref);
#pragma unroll
      for (int i = 0; i < NW; ++i) {
        o[i].x = o[i].x * f0 + v[i].x * f1;
        o[i].y = o[i].y * f0 + v[i].y * f1;
        o[i].z = o[i].z * f0 + v[i].z * f1;
        o[i].w = o[i].w * f0 + v[i].w * f1;
      }
      l = l * f0 + lx * f1;
      m = mn;
    };
    // the parts sub, sub + SPLIT, ... of the row's own and its prefix's, as one list
    const bool second = r >= psplit;
    const Parts4 pp = {second ? pb.first : pa.first, second ? pb.second : pa.second,
                       plist < 0 ? 0 : (second ? pb.count : pa.count), second ? pb.stride : pa.stride};
    const int prow = second ? r - psplit : r + pofs, n = in ? own.count + pp.count : 0;
#pragma unroll 2
    for (int k = sub; k < n; k += SPLIT) {
      const bool mine = k < own.count;
      const int kp = k - own.count;
      const int64_t at = mine ? (k ? own.second + (int64_t)(k - 1) * own.stride : own.first) + r
                              : (kp ? pp.second + (int64_t)(kp - 1) * pp.stride : pp.first) + prow;
      const bool from = mine ? list : plist;
      const float4* po = from ? a.plan.part_o[1] : a.plan.part_o[0];
      const float2 x = __ldcg((from ? a.plan.part_ml[1] : a.plan.part_ml[0]) + at);
      float4 v[NW];
#pragma unroll
      for (int i = 0; i < NW; ++i)
        v[i] = c0 + 4 * i < words ? __ldcg(po + part_word(at, c0 + 4 * i, dim)) : make_float4(0, 0, 0, 0);
      take(x.x, x.y, v);
    }
    if (SPLIT > 1) {
      __syncthreads();
      if (sub > 0) {
        sh->ml[sub - 1][lane] = make_float2(m, l);
#pragma unroll
        for (int i = 0; i < NW; ++i) sh->o[sub - 1][i][lane] = o[i];
      }
      __syncthreads();
      if (sub > 0) continue;
      for (int x = 0; x < SPLIT - 1; ++x) {
        float4 v[NW];
#pragma unroll
        for (int i = 0; i < NW; ++i) v[i] = sh->o[x][i][lane];
        take(sh->ml[x][lane].x, sh->ml[x][lane].y, v);
      }
    }
    const int rr = row0 + r;
    const int64_t tok = tok0 + rr / a.pool.ratio;
    const int hq = head * a.pool.ratio + rr % a.pool.ratio;
    float z = 0;
    if (in) {
      const float inv = l > 0 ? 1.0f / l : (l == 0 ? 0.0f : l);
      char* op = a.out + 2 * (tok * a.out_stride[0] + (int64_t)hq * a.out_stride[1]);
#pragma unroll
      for (int i = 0; i < NW; ++i)
        if (c0 + 4 * i < words) {
          z = spoil(spoil(spoil(spoil(z, o[i].x), o[i].y), o[i].z), o[i].w);
          *reinterpret_cast<uint2*>(op + 8 * (c0 + 4 * i)) =
              make_uint2(Num<T>::pack(o[i].x * inv, o[i].y * inv), Num<T>::pack(o[i].z * inv, o[i].w * inv));
        }
      if (a.lse && c0 == 0) a.lse[tok * a.pool.q_heads + hq] = log_sum(m, l);
    }
    if (!a.causal) continue;
    for (uint32_t spoilt = __reduce_or_sync(0xFFFFFFFFu, z != 0 ? 1u << (lane & 7) : 0u); spoilt; spoilt &= spoilt - 1)
      mend_row<T>(a, tok0, row0 + (int)(it % W) * 8 + __ffs(spoilt) - 1, head, lane);
  }
}
template <typename T>
__global__ void __launch_bounds__(32 * kJoinWarps, 16 / kJoinWarps) k_attend_join(AttendArgs a) {
  __shared__ JoinShared sh;
  // the entries are the plan's: they are read before the wait for the tiles' kernels
  const int4 h = __ldcg(reinterpret_cast<const int4*>(a.plan.hdr));  // status, entries
  bool waited = false;
  if (h.x != PS_OK) {
    chain();
    if (a.fill) {
      const int words = a.pool.head_dim / 8;
      const int64_t n = (int64_t)a.num_tokens * a.pool.q_heads * words;
      for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t row = i / words;
        char* p = a.out + 2 * (row / a.pool.q_heads * a.out_stride[0] + row % a.pool.q_heads * a.out_stride[1]);
        constexpr uint32_t x = Num<T>::kNan2;
        reinterpret_cast<uint4*>(p)[i % words] = make_uint4(x, x, x, x);
      }
    }
    return;
  }
  const int lane = threadIdx.x & 31, sub = threadIdx.x >> 5;
  const int64_t warp = (int64_t)blockIdx.x * kJoinWarps + sub, warps = (int64_t)gridDim.x * kJoinWarps;
  if ((int64_t)h.y * (tile_rows(0) / 8) + (int64_t)h.z * (tile_rows(1) / 8) <= 2 * (int64_t)gridDim.x) {
    join_rows<T, tile_rows(0), kJoinWarps>(a, &sh, &waited, 0, h.y, blockIdx.x, gridDim.x, sub, lane);
    join_rows<T, tile_rows(1), kJoinWarps>(a, &sh, &waited, 1, h.z, blockIdx.x, gridDim.x, sub, lane);
  } else {
    join_rows<T, tile_rows(0), 1>(a, &sh, &waited, 0, h.y, warp, warps, 0, lane);
    join_rows<T, tile_rows(1), 1>(a, &sh, &waited, 1, h.z, warp, warps, 0, lane);
  }
  if (!waited) chain();
  if (blockIdx.x == 0 && threadIdx.x == 0) a.plan.hdr->mend[a.turn ^ 1] = 0;
  if (__ldcg(&a.plan.hdr->mend[a.turn])) {
    mend_tiles<T, 0>(a, warp, warps, lane);
    mend_tiles<T, 1>(a, warp, warps, lane);
  }
}

template <typename T, int DP>
cudaError_t narrow(const AttendArgs& a, const PoolMaps& m, cudaStream_t st) {
  return launch(k_attend_narrow<T, DP>, dim3((unsigned)(a.plan.max_workers[0] / kWarps)), kThreads, Shape<DP>::kSmem, st, a, m);
}
template <typename T>
cudaError_t narrow_t(const AttendArgs& a, const PoolMaps& m, cudaStream_t st) {
  const int d = a.pool.head_dim;
  return d <= 64 ? narrow<T, 64>(a, m, st) : d <= 80 ? narrow<T, 80>(a, m, st) : d <= 96 ? narrow<T, 96>(a, m, st) : narrow<T, 128>(a, m, st);
}
template <typename T, int DP>
cudaError_t configure_narrow(int nsm, int32_t* workers) {
  cudaError_t e = cudaFuncSetAttribute(k_attend_narrow<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<DP>::kSmem);
  int occ = 0;
  if (e == cudaSuccess)
    e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&occ, k_attend_narrow<T, DP>, kThreads, Shape<DP>::kSmem);
  *workers = nsm * (occ > 0 ? occ : 1) * kWarps;
  return e;
}
template <typename T>
cudaError_t configure_t(int d, int nsm, int32_t* workers) {
  return d <= 64 ? configure_narrow<T, 64>(nsm, workers) : d <= 80 ? configure_narrow<T, 80>(nsm, workers)
       : d <= 96 ? configure_narrow<T, 96>(nsm, workers) : configure_narrow<T, 128>(nsm, workers);
}

}  // namespace

int32_t configure_attention(const Pool& p, int nsm, int32_t workers[kLists]) {
  workers[1] = nsm;
  const cudaError_t e = configure_wide(p);
  if (e != cudaSuccess) return status_of(e);
  return status_of(p.dtype == PS_KV_BF16 ? configure_t<__nv_bfloat16>(p.head_dim, nsm, workers)
                                         : configure_t<__half>(p.head_dim, nsm, workers));
}

int32_t launch_attention(const Pool& p, const PoolMaps& maps, const Plan& plan, const Batch& b, int32_t layer,
                         int32_t turn, const ps_kv_attention_t& in, int32_t* status, cudaStream_t st) {
  AttendArgs a{};
  a.pool = p;
  a.plan = plan;
  a.k = p.k + 2 * layer * p.layer_stride;
  a.v = p.v + 2 * layer * p.layer_stride;
  a.q = (const char*)in.q;
  a.out = (char*)in.out;
  a.lse = in.lse;
  for (int i = 0; i < 2; ++i) {
    a.q_stride[i] = in.q_stride[i];
    a.out_stride[i] = in.out_stride[i];
  }
  a.tables = b.tables;
  a.table_stride = b.table_stride;
  a.q_offsets = b.q_offsets;
  a.kv_lens = b.kv_lens;
  a.causal = b.causal;
  a.turn = turn;
  a.fill = in.fill;
  a.num_tokens = b.num_tokens;
  a.status = status;
  a.scale2 = in.scale * 1.4426950408889634f;
  // no tile has more rows than the whole batch
  const bool wide = list_of(b.num_tokens * p.ratio) == 1;
  a.after_wide = wide;
  cudaError_t e = cudaSuccess;
  if (wide) {
    PoolMaps with_q = maps;
    make_query_map(p, in.q, in.q_stride, b.num_tokens, &with_q);
    e = launch_wide(a, with_q, st);
  }
  if (e == cudaSuccess) e = p.dtype == PS_KV_BF16 ? narrow_t<__nv_bfloat16>(a, maps, st) : narrow_t<__half>(a, maps, st);
  if (e != cudaSuccess) return status_of(e);
  // a CTA for every eight rows of narrow tiles, up to one full wave
  const int64_t want = (int64_t)b.num_tokens * p.kv_heads * 2, most = (int64_t)plan.max_workers[1] * (16 / kJoinWarps);
  const dim3 grid((unsigned)(want < most ? want : most));
  e = p.dtype == PS_KV_BF16 ? launch(k_attend_join<__nv_bfloat16>, grid, 32 * kJoinWarps, 0, st, a)
                            : launch(k_attend_join<__half>, grid, 32 * kJoinWarps, 0, st, a);
  return status_of(e);
}

}  // namespace pskv
