// ps_kv_append: norm of queries and keys for each head, position rotation, and
// the write of keys and values into their pages, in one pass.
#include "ps_kv_attend.cuh"

namespace pskv {
namespace {

struct AppendArgs {
  const char *q, *k, *v, *qw, *kw;
  char *qo, *pk, *pv;  // the pool's pointers at the call's layer
  const int64_t* slots;
  const int32_t* positions;
  const float* rope;
  int32_t* status;
  int64_t qs[2], ks[2], vs[2], os[2];       // strides in elements
  int64_t page_stride, token_stride, head_stride, nslots;
  int32_t T, hq, hk, dim, page_log2, rope_rows, rope_dim, fill;
  float eps;
};

// The mathematics, for one head x of D elements: r = 1 / sqrt(sum x^2 / D +
// eps), y = r x w, then for each rotated pair (a, b) -> (a cos - b sin, b cos +
// a sin).  The weights are put into the pair's four factors, so an element takes
// two products and one by r.
//
// Every element is read once and written once, so HBM is the floor; what it
// comes to lies with the instructions per element, so there are few of them.  A
// head is held by G lanes of two parts of E elements each, chosen so that a
// pair's partner is in the lane itself: of the rotated elements part i with part
// i + rope_dim / (2 E), of the rest (and of interleaved pairs) neighbours.  The
// sum of squares is a shuffle over G lanes; products and sums go two at a time.
// A warp takes 32 / G heads at once, a slice.  All tokens' slices (queries, then
// keys and values as one list of heads) are one list that is cut into equal
// parts for the resident warps; a warp keeps a token's factors in registers, and
// the next slice's loads are in flight while it works on one.
template <typename T>
__device__ __forceinline__ uint64_t wide2(uint32_t x) {
  const float2 f = Num<T>::unpack(x);
  return pack2(f.x, f.y);
}
template <typename T>
__device__ __forceinline__ uint32_t narrow2(uint64_t x) {
  const float2 f = unpack2(x);
  return Num<T>::pack(f.x, f.y);
}
__device__ __forceinline__ uint64_t swap2(uint64_t x) {
  const float2 f = unpack2(x);
  return pack2(f.y, f.x);
}

template <int E>
struct Part {
  uint32_t x[E / 2];
};
template <int E>
__device__ __forceinline__ Part<E> read_part(const char* p) {  // shared memory
  Part<E> r;
  if (E == 8) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    r.x[0] = v.x, r.x[1] = v.y, r.x[E / 2 - 2] = v.z, r.x[E / 2 - 1] = v.w;
  } else {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    r.x[0] = v.x, r.x[1] = v.y;
  }
  return r;
}
// A part into shared memory, or zeros where !ok.
template <int E>
__device__ __forceinline__ void copy_part(uint32_t dst, const char* src, bool ok) {
  if (E == 8)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(ok ? 8 : 0) : "memory");
}
template <int E>
__device__ __forceinline__ void write_part(char* p, const Part<E>& r) {
  if (E == 8) *reinterpret_cast<uint4*>(p) = make_uint4(r.x[0], r.x[1], r.x[E / 2 - 2], r.x[E / 2 - 1]);
  else *reinterpret_cast<uint2*>(p) = make_uint2(r.x[0], r.x[1]);
}

// 8191 bf16 tokens, 32 + 2 x 8 heads of 128, both norms, all rotated: 36 us, 5.7
// TB/s of the 6.8 that copies reach, with the issue slots at 70 % (293
// instructions a slice of four heads).  Loads into registers, one slice ahead:
// 50 us; 8-byte parts, two heads' loads together and 48 warps an SM: 44 us.
// Six CTAs an SM spill registers (47 us), three or six stages change nothing.
constexpr int kThreads = 128;
constexpr int kCtasPerSm = 5;
constexpr int kStages = 4;  // slices of a warp in flight or at work
struct WarpShared {
  char slice[kStages][2][32 * 16];  // parts of the lanes
  char weight[2][256];              // of queries and keys
  float row[4][128];                // rotation table rows of four tokens in a row
};

template <typename T, int E, int G, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads, kCtasPerSm) k_append(AppendArgs a) {
  chain();
  constexpr int H = 32 / G, N = E / 2;  // heads of a slice, words of a part
  const int lane = threadIdx.x % G, grp = threadIdx.x % 32 / G;
  const int parts = a.dim / E, pairs = a.rope_dim / (2 * E);
  const bool rotated = lane < pairs;
  // the lane's two parts of a head
  const int p0 = INTERLEAVED || !rotated ? 2 * lane : lane, p1 = INTERLEAVED || !rotated ? p0 + 1 : lane + pairs;
  const bool on0 = p0 < parts, on1 = p1 < parts;
  const int at0 = 2 * E * p0, at1 = 2 * E * p1;
  const float inv_dim = 1.0f / a.dim;
  __shared__ __align__(16) WarpShared shared[kThreads / 32];
  WarpShared& sh = shared[threadIdx.x / 32];

  const int nq = (a.hq + H - 1) / H, S = nq + (2 * a.hk + H - 1) / H;  // slices of a token
  const int64_t units = (int64_t)a.T * S;
  const int64_t w = (int64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32, warps = (int64_t)gridDim.x * (kThreads / 32);
  const int64_t first = units * w / warps;
  const int n = (int)(units * (w + 1) / warps - first);
  if (n <= 0) return;
  int t = (int)(first / S), s = (int)(first - (int64_t)t * S);  // of the slice at work
  int lt = t, ls = s;                                           // of the one to load

  // The weights, a row of the table and a slice, asynchronously.
  const int wl = threadIdx.x % 32;
  {
    const char* weight = wl < 16 ? a.qw : a.kw;
    const int c = wl % 16;
    cp16(smem_addr(sh.weight[wl / 16] + 16 * c), weight ? weight + 16 * c : a.q, weight && c * 8 < a.dim);
  }
  int load_pos = a.rope ? a.positions[lt] : 0;
  int load_stage = 0, load_left = n;
  bool load_row = true;
  auto load = [&]() {
    if (load_left > 0) {
      --load_left;
      if (load_row && a.rope) {  // a token's first slice here
        if (load_pos >= 0 && load_pos < a.rope_rows)
          cp16(smem_addr(sh.row[lt & 3] + 4 * wl), a.rope + (int64_t)load_pos * a.rope_dim + 4 * wl, 4 * wl < a.rope_dim);
        if (lt + 1 < a.T) load_pos = a.positions[lt + 1];
      }
      const char* p;
      bool in;
      if (ls < nq) {
        const int h = ls * H + grp;
        in = h < a.hq;
        p = a.q + 2 * (lt * a.qs[0] + h * a.qs[1]);
      } else {
        const int h = (ls - nq) * H + grp;
        in = h < 2 * a.hk;
        p = h < a.hk ? a.k + 2 * (lt * a.ks[0] + h * a.ks[1]) : a.v + 2 * (lt * a.vs[0] + (h - a.hk) * a.vs[1]);
      }
      copy_part<E>(smem_addr(sh.slice[load_stage][0] + 16 * wl), in && on0 ? p + at0 : a.q, in && on0);
      copy_part<E>(smem_addr(sh.slice[load_stage][1] + 16 * wl), in && on1 ? p + at1 : a.q, in && on1);
      load_stage = (load_stage + 1) % kStages;
      load_row = ++ls == S;
      if (load_row) {
        ls = 0;
        ++lt;
      }
    }
    cp_commit();
  };

  // A token's slot and position are read while the one before it is worked on.
  int64_t next_slot = a.slots[t];
  int next_pos = a.rope ? a.positions[t] : 0;
  bool valid = false, begun = false, fresh = true;  // fresh: no factors yet
  int64_t at = -1;  // of the token in the pool; negative: not written
  // f0 x + f1 y for the words x of a part, y their partners (the other part's, or the swapped ones)
  uint64_t f0[2][N], f1[2][N];
  auto factors = [&](const char* weight, bool has) {
    uint64_t wt[2][N], cs[2][N / 2], sn[2][N / 2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      Part<E> raw{};
      if (has && (i ? on1 : on0)) raw = read_part<E>(weight + (i ? at1 : at0));
#pragma unroll
      for (int j = 0; j < N; ++j) wt[i][j] = has ? wide2<T>(raw.x[j]) : pack2(1.0f, 1.0f);
    }
    if (!rotated) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) f0[i][j] = wt[i][j];
      return;
    }
    const float* row = sh.row[t & 3] + E * lane;
#pragma unroll
    for (int j = 0; j < E / 4; ++j) {
      const float4 c = *(reinterpret_cast<const float4*>(row) + j);
      const float4 v = *(reinterpret_cast<const float4*>(row + a.rope_dim / 2) + j);
      cs[2 * j / (N / 2)][2 * j % (N / 2)] = pack2(c.x, c.y);
      cs[(2 * j + 1) / (N / 2)][(2 * j + 1) % (N / 2)] = pack2(c.z, c.w);
      sn[2 * j / (N / 2)][2 * j % (N / 2)] = pack2(v.x, v.y);
      sn[(2 * j + 1) / (N / 2)][(2 * j + 1) % (N / 2)] = pack2(v.z, v.w);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (INTERLEAVED) {  // word j of part i is a pair: cosine i N + j
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float2 c2 = unpack2(cs[i][j / 2]), s2 = unpack2(sn[i][j / 2]), w2 = unpack2(wt[i][j]);
          const float c = j % 2 ? c2.y : c2.x, v = j % 2 ? s2.y : s2.x;
          f0[i][j] = pack2(w2.x * c, w2.y * c);
          f1[i][j] = pack2(-w2.y * v, w2.x * v);
        }
      } else {
        const uint64_t c = cs[j / (N / 2)][j % (N / 2)], v = sn[j / (N / 2)][j % (N / 2)];
        f0[0][j] = mul2(wt[0][j], c);
        f1[0][j] = mul2(wt[1][j], v) ^ 0x8000000080000000ull;
        f0[1][j] = mul2(wt[1][j], c);
        f1[1][j] = mul2(wt[0][j], v);
      }
    }
  };

  int stage = 0;
  auto work = [&]() {
    Part<E> raw[2] = {read_part<E>(sh.slice[stage][0] + 16 * wl), read_part<E>(sh.slice[stage][1] + 16 * wl)};
    stage = (stage + 1) % kStages;
    if (s == 0 || !begun) {  // a token's first slice here
      begun = true;
      const int64_t slot = next_slot;
      const int pos = next_pos;
      if (t + 1 < a.T) {
        next_slot = a.slots[t + 1];
        if (a.rope) next_pos = a.positions[t + 1];
      }
      valid = slot < a.nslots && (!a.rope || (pos >= 0 && pos < a.rope_rows));
      if (!valid && wl == 0) set_error(a.status, PS_ERR_INVALID_ARG);
      at = valid && slot >= 0 ? 2 * ((slot >> a.page_log2) * a.page_stride + (slot & ((1 << a.page_log2) - 1)) * a.token_stride) : -1;
    }
    const bool query = s < nq;
    const int h = (query ? s : s - nq) * H + grp;
    const bool value = !query && h >= a.hk;
    char* dst = nullptr;
    if (query && h < a.hq && (valid || a.fill)) dst = a.qo + 2 * (t * a.os[0] + h * a.os[1]);
    if (!query && h < 2 * a.hk && at >= 0) dst = (value ? a.pv - 2 * a.hk * a.head_stride : a.pk) + at + 2 * h * a.head_stride;
    if (!__all_sync(0xFFFFFFFFu, value)) {
      const bool weight = query ? a.qw != nullptr : a.kw != nullptr;
      if (s == 0 || s == nq || fresh) factors(sh.weight[query ? 0 : 1], weight);
      fresh = false;
      uint64_t x[2][N];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) x[i][j] = wide2<T>(raw[i].x[j]);
      uint64_t r2 = pack2(1.0f, 1.0f);
      if (weight) {
        uint64_t s2 = mul2(x[0][0], x[0][0]);
#pragma unroll
        for (int k = 1; k < 2 * N; ++k) s2 = fma2(x[k / N][k % N], x[k / N][k % N], s2);
        const float2 f = unpack2(s2);
        float ss = f.x + f.y;
#pragma unroll
        for (int o = G / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, o);
        const float r = rsqrtf(ss * inv_dim + a.eps);
        r2 = pack2(r, r);
      }
      Part<E> y[2];
#pragma unroll
      for (int j = 0; j < N; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint64_t v = mul2(x[i][j], f0[i][j]);
          if (rotated) v = fma2(INTERLEAVED ? swap2(x[i][j]) : x[1 - i][j], f1[i][j], v);
          y[i].x[j] = narrow2<T>(mul2(v, r2));
        }
      if (!value) {  // values are moved as they are (a conversion could change a NaN's bits)
        raw[0] = y[0];
        raw[1] = y[1];
      }
    }
    if (!valid && query) {
#pragma unroll
      for (int j = 0; j < N; ++j) raw[0].x[j] = raw[1].x[j] = Num<T>::kNan2;
    }
    if (dst && on0) write_part<E>(dst + at0, raw[0]);
    if (dst && on1) write_part<E>(dst + at1, raw[1]);
    if (++s == S) {
      s = 0;
      ++t;
    }
  };

#pragma unroll 1
  for (int i = 0; i < kStages - 1; ++i) load();
#pragma unroll 1
  for (int i = 0; i < n; ++i) {
    cp_wait<kStages - 2>();
    __syncwarp();  // the slice has landed, and all lanes are done with the one before it
    load();
    work();
  }
  cp_wait<0>();
}

template <typename T, int E, int G, bool I>
cudaError_t launch_g(const AppendArgs& a, int nsm, cudaStream_t st) {
  constexpr int H = 32 / G, W = kThreads / 32;
  const int64_t units = (int64_t)a.T * ((a.hq + H - 1) / H + (2 * a.hk + H - 1) / H), most = (int64_t)nsm * kCtasPerSm;
  const int64_t want = (units + W - 1) / W;
  return launch(k_append<T, E, G, I>, dim3((unsigned)(want < most ? want : most)), kThreads, 0, st, a);
}
// Parts of 8 elements (16 bytes) where the rotated half is whole times 8, else of 4
// (half the bytes an instruction: 8191 tokens took 44 us with parts of 4).
template <typename T, bool I>
cudaError_t launch_e(const AppendArgs& a, int nsm, cudaStream_t st) {
  if (a.rope_dim % 16 == 0) return a.dim <= 64 ? launch_g<T, 8, 4, I>(a, nsm, st) : launch_g<T, 8, 8, I>(a, nsm, st);
  return a.dim <= 64 ? launch_g<T, 4, 8, I>(a, nsm, st) : launch_g<T, 4, 16, I>(a, nsm, st);
}
template <typename T>
cudaError_t launch_t(const AppendArgs& a, bool interleaved, int nsm, cudaStream_t st) {
  return interleaved ? launch_e<T, true>(a, nsm, st) : launch_e<T, false>(a, nsm, st);
}

}  // namespace

int32_t launch_append(const Pool& p, int32_t layer, const ps_kv_append_t& in, int32_t* status, int nsm,
                      cudaStream_t st) {
  AppendArgs a{};
  a.q = (const char*)in.q; a.k = (const char*)in.k; a.v = (const char*)in.v;
  a.qw = (const char*)in.q_weight; a.kw = (const char*)in.k_weight;
  a.qo = (char*)in.q_out;
  a.pk = p.k + 2 * layer * p.layer_stride;
  a.pv = p.v + 2 * layer * p.layer_stride;
  a.slots = in.slots; a.positions = in.positions; a.rope = in.rope_dim > 0 ? in.rope : nullptr; a.status = status;
  for (int i = 0; i < 2; ++i) {
    a.qs[i] = in.q_stride[i]; a.ks[i] = in.k_stride[i]; a.vs[i] = in.v_stride[i]; a.os[i] = in.q_out_stride[i];
  }
  a.page_stride = p.page_stride; a.token_stride = p.token_stride; a.head_stride = p.head_stride;
  a.nslots = p.num_pages << p.page_log2;
  a.T = in.num_tokens; a.hq = p.q_heads; a.hk = p.kv_heads; a.dim = p.head_dim; a.page_log2 = p.page_log2;
  a.rope_rows = in.rope_rows; a.rope_dim = a.rope ? in.rope_dim : 0; a.eps = in.eps;
  a.fill = in.fill;
  return status_of(p.dtype == PS_KV_BF16 ? launch_t<__nv_bfloat16>(a, in.rope_interleaved != 0, nsm, st)
                                         : launch_t<__half>(a, in.rope_interleaved != 0, nsm, st));
}

}  // namespace pskv
