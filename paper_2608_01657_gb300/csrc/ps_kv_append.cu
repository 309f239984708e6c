// ps_kv_append: norm of queries and keys for each head, position rotation, and
// the write of keys and values into their pages, in one pass.
#include "ps_kv.cuh"

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
  int32_t T, hq, hk, dim, page_log2, rope_rows, rope_dim;
  float eps;
};

// The mathematics, for one head x of D elements: y = x w / sqrt(sum x^2 / D +
// eps), then for each rotated pair (a, b) -> (a cos - b sin, b cos + a sin).
//
// Every element is read once and written once, so HBM is the floor; what it
// comes to lies with the instructions per element, so there are few of them.  A
// head is held by G = 8 or 16 lanes of two quads (4 elements) each, chosen so
// that a pair's partner is in the lane itself: of the rotated part quad i with
// quad i + rope_dim / 8, of the rest (and of interleaved pairs) neighbours.  The
// sum of squares is a shuffle over G lanes; products and sums go two at a time.
// A group of lanes takes several heads of one token, whose cosines and sines
// stay in registers, U query heads' loads in flight together.
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

// Enough warps to hide the loads' latency (8191 tokens: 53 us with 8, 44 with 12).
constexpr int kCtasPerSm = 12;
template <int N>
struct Count {
  static constexpr int value = N;
};

template <typename T, int G, bool INTERLEAVED, int U>
__global__ void __launch_bounds__(128, kCtasPerSm) k_append(AppendArgs a) {
  chain();
  constexpr int kGroups = 128 / G;
  const int lane = threadIdx.x % G, grp = threadIdx.x / G;
  const bool on = lane * 8 < a.dim;
  const int pairs = a.rope_dim / 8;  // quads of half the rotated part
  const bool rotated = lane < pairs;
  // byte offsets of the lane's two quads in a head
  const int qa = INTERLEAVED || !rotated ? 2 * lane : lane;
  const int at0 = 8 * qa, at1 = 8 * (INTERLEAVED || !rotated ? qa + 1 : qa + pairs);
  const float inv_dim = 1.0f / a.dim;
  // A token's slot and position are read while the one before it is worked on.
  int64_t next_slot = blockIdx.x < a.T ? a.slots[blockIdx.x] : 0;
  int next_pos = a.rope && blockIdx.x < a.T ? a.positions[blockIdx.x] : 0;
  for (int t = blockIdx.x; t < a.T; t += gridDim.x) {
  const int64_t slot = next_slot;
  const int pos = next_pos;
  if (t + (int64_t)gridDim.x < a.T) {
    next_slot = a.slots[t + gridDim.x];
    if (a.rope) next_pos = a.positions[t + gridDim.x];
  }
  if (slot >= a.nslots || (a.rope && (pos < 0 || pos >= a.rope_rows))) {
    if (threadIdx.x == 0) set_error(a.status, PS_ERR_INVALID_ARG);
    continue;
  }
  // the pairs' cosines and sines; 1 and 0 where nothing turns
  uint64_t cs[2], sn[2];
  if (rotated) {
    const float* row = a.rope + (int64_t)pos * a.rope_dim + 4 * lane;
    const float4 c = __ldg(reinterpret_cast<const float4*>(row));
    const float4 s = __ldg(reinterpret_cast<const float4*>(row + a.rope_dim / 2));
    cs[0] = pack2(c.x, c.y); cs[1] = pack2(c.z, c.w);
    sn[0] = pack2(s.x, s.y); sn[1] = pack2(s.z, s.w);
  } else {
    cs[0] = cs[1] = pack2(1.0f, 1.0f);
    sn[0] = sn[1] = 0;
  }
  const int64_t at = slot < 0 ? 0 : 2 * ((slot >> a.page_log2) * a.page_stride +
                                         (slot & ((1 << a.page_log2) - 1)) * a.token_stride);
  // Heads grp, grp + kGroups, ... of the queries (slices [0, nq)), the keys
  // [nq, nq + nk) and the values, of which this CTA takes every gridDim.y-th.
  const int nq = (a.hq + kGroups - 1) / kGroups, nk = (a.hk + kGroups - 1) / kGroups;
  int slice = blockIdx.y;

  // norm and rotation of a slice's heads, U slices' loads at a time
  auto heads = [&](auto batch, int end, int base, int count, const char* src, int64_t src_stride, char* dst,
                   int64_t dst_stride, const char* weight, bool write) {
    constexpr int B = decltype(batch)::value;
    uint64_t w[4] = {};
    if (on && weight) {
      const uint2 w0 = __ldg(reinterpret_cast<const uint2*>(weight + at0)), w1 = __ldg(reinterpret_cast<const uint2*>(weight + at1));
      w[0] = wide2<T>(w0.x); w[1] = wide2<T>(w0.y); w[2] = wide2<T>(w1.x); w[3] = wide2<T>(w1.y);
    }
    int h = (slice - base) * kGroups + grp;
    const int step = (int)gridDim.y * kGroups;
    src += 2 * h * src_stride;
    dst += 2 * h * dst_stride;
    for (; slice < end; slice += (int)gridDim.y * B) {
      uint2 raw[B][2];
#pragma unroll
      for (int u = 0; u < B; ++u) {
        raw[u][0] = raw[u][1] = make_uint2(0, 0);
        if (h + u * step < count && on) {
          const char* p = src + 2 * u * step * src_stride;
          raw[u][0] = *reinterpret_cast<const uint2*>(p + at0);
          raw[u][1] = *reinterpret_cast<const uint2*>(p + at1);
        }
      }
#pragma unroll
      for (int u = 0; u < B; ++u) {
        // both quads, two elements at a time; x[0], x[1] pair with x[2], x[3]
        uint64_t x[4] = {wide2<T>(raw[u][0].x), wide2<T>(raw[u][0].y), wide2<T>(raw[u][1].x), wide2<T>(raw[u][1].y)};
        if (weight) {
          uint64_t s2 = mul2(x[0], x[0]);
#pragma unroll
          for (int i = 1; i < 4; ++i) s2 = fma2(x[i], x[i], s2);
          const float2 f = unpack2(s2);
          float ss = f.x + f.y;
#pragma unroll
          for (int o = G / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, o);
          const float r = rsqrtf(ss * inv_dim + a.eps);
          const uint64_t r2 = pack2(r, r);
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = mul2(mul2(x[i], r2), w[i]);
        }
        if (rotated) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (INTERLEAVED) {  // pairs (x, y) of quad i: its elements 0, 1 and 2, 3
              const float2 p = unpack2(x[2 * i]), r = unpack2(x[2 * i + 1]), c = unpack2(cs[i]), s = unpack2(sn[i]);
              x[2 * i] = pack2(p.x * c.x - p.y * s.x, p.y * c.x + p.x * s.x);
              x[2 * i + 1] = pack2(r.x * c.y - r.y * s.y, r.y * c.y + r.x * s.y);
            } else {
              const uint64_t p = x[i], r = x[i + 2];
              x[i] = fma2(r, sn[i] ^ 0x8000000080000000ull, mul2(p, cs[i]));
              x[i + 2] = fma2(p, sn[i], mul2(r, cs[i]));
            }
          }
        }
        if (h + u * step < count && on && write) {
          char* p = dst + 2 * u * step * dst_stride;
          *reinterpret_cast<uint2*>(p + at0) = make_uint2(narrow2<T>(x[0]), narrow2<T>(x[1]));
          *reinterpret_cast<uint2*>(p + at1) = make_uint2(narrow2<T>(x[2]), narrow2<T>(x[3]));
        }
      }
      h += B * step;
      src += 2 * B * step * src_stride;
      dst += 2 * B * step * dst_stride;
    }
  };
  if (slice < nq)
    heads(Count<U>{}, nq, 0, a.hq, a.q + 2 * t * a.qs[0], a.qs[1], a.qo + 2 * t * a.os[0], a.os[1], a.qw, true);
  // a batch may have stepped over slices that are not the queries'
  slice = nq > (int)blockIdx.y ? (int)blockIdx.y + (nq - (int)blockIdx.y + (int)gridDim.y - 1) / (int)gridDim.y * (int)gridDim.y
                               : (int)blockIdx.y;
  if (slice < nq + nk)
    heads(Count<1>{}, nq + nk, nq, a.hk, a.k + 2 * t * a.ks[0], a.ks[1], a.pk + at, a.head_stride, a.kw, slot >= 0);
  if (slot < 0) continue;
  // values are moved as they are (a conversion could change a NaN's bits)
  for (; slice < nq + 2 * nk; slice += gridDim.y) {
    const int h = (slice - nq - nk) * kGroups + grp;
    if (h < a.hk && on)
      *reinterpret_cast<uint4*>(a.pv + at + 2 * h * a.head_stride + 16 * lane) =
          *reinterpret_cast<const uint4*>(a.v + 2 * (t * a.vs[0] + h * a.vs[1]) + 16 * lane);
  }
  }
}

template <typename T, int G, bool I>
cudaError_t launch_g(const AppendArgs& a, int nsm, cudaStream_t st) {
  // few tokens: spread a token's heads over CTAs until the GPU has some waves;
  // otherwise the loads of two heads of a group at a time
  const int groups = 128 / G, nq = (a.hq + groups - 1) / groups, slices = nq + 2 * ((a.hk + groups - 1) / groups);
  int ny = (4 * nsm + a.T - 1) / a.T;
  ny = ny < 1 ? 1 : (ny > slices ? slices : ny);
  const dim3 grid((unsigned)(a.T < nsm * kCtasPerSm ? a.T : nsm * kCtasPerSm), (unsigned)ny);
  return nq >= 2 * ny ? launch(k_append<T, G, I, 2>, grid, 128, 0, st, a) : launch(k_append<T, G, I, 1>, grid, 128, 0, st, a);
}
template <typename T>
cudaError_t launch_t(const AppendArgs& a, bool interleaved, int nsm, cudaStream_t st) {
  if (a.dim <= 64) return interleaved ? launch_g<T, 8, true>(a, nsm, st) : launch_g<T, 8, false>(a, nsm, st);
  return interleaved ? launch_g<T, 16, true>(a, nsm, st) : launch_g<T, 16, false>(a, nsm, st);
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
  return status_of(p.dtype == PS_KV_BF16 ? launch_t<__nv_bfloat16>(a, in.rope_interleaved != 0, nsm, st)
                                         : launch_t<__half>(a, in.rope_interleaved != 0, nsm, st));
}

}  // namespace pskv
