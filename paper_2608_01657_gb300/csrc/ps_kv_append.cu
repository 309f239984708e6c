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
// Bound by HBM: every element is read once and written once.  A head's
// elements are held by G = 8 or 16 lanes, 8 elements (16 bytes) each, so the
// sum of squares is a shuffle over G lanes, and a pair's partner is either in
// the lane itself (interleaved) or rope_dim / 2 elements away.  A group of lanes
// takes several heads of one token, so that the token's cosines and sines are
// read once into registers; a CTA's blockIdx.y takes a slice of the heads
// (queries, then keys, then values).
template <typename T, int G, bool INTERLEAVED>
__global__ void __launch_bounds__(128) k_append(AppendArgs a) {
  chain();
  const int lane = threadIdx.x % G, grp = threadIdx.x / G;
  constexpr int kGroups = 128 / G;
  const int t = blockIdx.x;
  const int nheads = a.hq + 2 * a.hk;
  const int64_t slot = a.slots[t];
  const int pos = a.rope ? a.positions[t] : 0;
  if (slot >= a.nslots || (a.rope && (pos < 0 || pos >= a.rope_rows))) {
    if (threadIdx.x == 0) set_error(a.status, PS_ERR_INVALID_ARG);
    return;
  }
  const bool on = lane * 8 < a.dim;
  // Rotated elements in quarter words of four: quarter g is one of the lane's
  // two, g = 2 lane + s; without interleaving its partner is 'half' quarters
  // up or down (in the lane's other place where half is odd).
  const int half = a.rope_dim / 8;
  const bool odd = half & 1;
  // this lane's cosines and sines: of its own 8 elements, or of its 4 pairs
  constexpr int NC = INTERLEAVED ? 4 : 8;
  float cs[NC], sn[NC];
#pragma unroll
  for (int s = 0; s < NC / 4; ++s) {
    const int g = INTERLEAVED ? lane : 2 * lane + s;
    const int at = INTERLEAVED || g < half ? g : g - half;
    if (a.rope && at < half) {
      const float* row = a.rope + (int64_t)pos * a.rope_dim + 4 * at;
      const float4 c = __ldg(reinterpret_cast<const float4*>(row));
      const float4 x = __ldg(reinterpret_cast<const float4*>(row + a.rope_dim / 2));
      cs[4 * s] = c.x; cs[4 * s + 1] = c.y; cs[4 * s + 2] = c.z; cs[4 * s + 3] = c.w;
      sn[4 * s] = x.x; sn[4 * s + 1] = x.y; sn[4 * s + 2] = x.z; sn[4 * s + 3] = x.w;
    } else {  // not rotated
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        cs[4 * s + i] = 1.0f;
        sn[4 * s + i] = 0.0f;
      }
    }
  }
  const int64_t at = slot < 0 ? 0 : (slot >> a.page_log2) * a.page_stride +
                                        (slot & ((1 << a.page_log2) - 1)) * a.token_stride;
  for (int h0 = blockIdx.y * kGroups; h0 < nheads; h0 += gridDim.y * kGroups) {
    const int h = h0 + grp;
    const bool have = h < nheads;
    const int kind = h < a.hq ? 0 : (h < a.hq + a.hk ? 1 : 2);
    const int hh = kind == 0 ? h : (kind == 1 ? h - a.hq : h - a.hq - a.hk);
    uint4 raw = make_uint4(0, 0, 0, 0);
    if (have && on) {
      const char* src = kind == 0 ? a.q + 2 * (t * a.qs[0] + hh * a.qs[1])
                                  : (kind == 1 ? a.k + 2 * (t * a.ks[0] + hh * a.ks[1])
                                               : a.v + 2 * (t * a.vs[0] + hh * a.vs[1]));
      raw = *reinterpret_cast<const uint4*>(src + lane * 16);
    }
    float x[8];
    {
      const float2 f0 = Num<T>::unpack(raw.x), f1 = Num<T>::unpack(raw.y), f2 = Num<T>::unpack(raw.z),
                   f3 = Num<T>::unpack(raw.w);
      x[0] = f0.x; x[1] = f0.y; x[2] = f1.x; x[3] = f1.y; x[4] = f2.x; x[5] = f2.y; x[6] = f3.x; x[7] = f3.y;
    }
    const char* wp = kind == 0 ? a.qw : a.kw;
    if (a.qw || a.kw) {  // both shuffles and branches are uniform over the CTA
      float ss = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss += x[i] * x[i];
#pragma unroll
      for (int o = G / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, o);
      if (kind < 2 && wp && on) {
        const float r = 1.0f / sqrtf(ss / a.dim + a.eps);
        const uint4 w = __ldg(reinterpret_cast<const uint4*>(wp + lane * 16));
        const float2 f0 = Num<T>::unpack(w.x), f1 = Num<T>::unpack(w.y), f2 = Num<T>::unpack(w.z),
                     f3 = Num<T>::unpack(w.w);
        x[0] *= r * f0.x; x[1] *= r * f0.y; x[2] *= r * f1.x; x[3] *= r * f1.y;
        x[4] *= r * f2.x; x[5] *= r * f2.y; x[6] *= r * f3.x; x[7] *= r * f3.y;
      }
    }
    if (a.rope) {
      if (INTERLEAVED) {
        if (kind < 2 && lane < half) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float u = x[2 * i], w = x[2 * i + 1];
            x[2 * i] = u * cs[i % NC] - w * sn[i % NC];
            x[2 * i + 1] = w * cs[i % NC] + u * sn[i % NC];
          }
        }
      } else {
        float o[8];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const int g = 2 * lane + s;
          const int peer = g < half ? g + half : (g < 2 * half ? g - half : g);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            o[4 * s + i] = __shfl_sync(0xFFFFFFFFu, odd ? x[4 * (1 - s) + i] : x[4 * s + i], peer >> 1, G);
        }
        if (kind < 2) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int g = 2 * lane + i / 4;
            if (g < half) x[i] = x[i] * cs[i % NC] - o[i] * sn[i % NC];
            else if (g < 2 * half) x[i] = x[i] * cs[i % NC] + o[i] * sn[i % NC];
          }
        }
      }
    }
    if (!have || !on) continue;
    // values are moved as they are (a conversion could change a NaN's bits)
    if (kind < 2)
      raw = make_uint4(Num<T>::pack(x[0], x[1]), Num<T>::pack(x[2], x[3]), Num<T>::pack(x[4], x[5]),
                       Num<T>::pack(x[6], x[7]));
    char* dst;
    if (kind == 0) {
      dst = a.qo + 2 * (t * a.os[0] + hh * a.os[1]);
    } else {
      if (slot < 0) continue;
      dst = (kind == 1 ? a.pk : a.pv) + 2 * (at + hh * a.head_stride);
    }
    *reinterpret_cast<uint4*>(dst + lane * 16) = raw;
  }
}

template <typename T>
cudaError_t launch_t(const AppendArgs& a, bool interleaved, int nsm, cudaStream_t st) {
  const int groups = a.dim <= 64 ? 16 : 8;
  // few tokens: spread a token's heads over CTAs until the GPU has one wave
  const int slices = (a.hq + 2 * a.hk + groups - 1) / groups;
  int ny = (4 * nsm + a.T - 1) / a.T;
  ny = ny < 1 ? 1 : (ny > slices ? slices : ny);
  const dim3 grid((unsigned)a.T, (unsigned)ny);
  if (a.dim <= 64)
    return interleaved ? launch(k_append<T, 8, true>, grid, 128, 0, st, a) : launch(k_append<T, 8, false>, grid, 128, 0, st, a);
  return interleaved ? launch(k_append<T, 16, true>, grid, 128, 0, st, a) : launch(k_append<T, 16, false>, grid, 128, 0, st, a);
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
  a.rope_rows = in.rope_rows; a.rope_dim = in.rope_dim; a.eps = in.eps;
  return status_of(p.dtype == PS_KV_BF16 ? launch_t<__nv_bfloat16>(a, in.rope_interleaved != 0, nsm, st)
                                         : launch_t<__half>(a, in.rope_interleaved != 0, nsm, st));
}

}  // namespace pskv
