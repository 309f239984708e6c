// ps_beam_trace: sequences of tokens, back through every step's parents.
//
// A hypothesis of L steps that ends in beam b: token L - 1 is tokens[L - 1][b], then
// b <- parents[t][b] from t = L - 1 down to 1.  A chain of dependent lookups, cut into
// segments of 32 steps, one a warp: the warp holds the segment's parents and tokens a
// beam a lane, 32 registers of each, so that a lookup is a shuffle.  It first takes
// every beam at the segment's end to its ancestor before the segment, and so does it
// with the hypotheses that end inside; then a walk over the segments gives the beam in
// which each hypothesis enters each segment, and the warps go through their segments
// once more, for the tokens.  A CTA takes a request's last 16 segments at once, then
// those before them.
#include "ps_beam.cuh"

namespace psbeam {
namespace {

constexpr int kSteps = 32, kSegs = 16, kThreads = 32 * kSegs;
constexpr unsigned kAll = 0xFFFFFFFFu;

struct Args {
  ps_beam_trace_t a;
  int32_t* status;
  int32_t beams;
};

// A beam that is not there: past an end, or a parent out of range.
constexpr int kNone = -1;
__device__ __forceinline__ int look(int mine, int beam) {
  const int x = __shfl_sync(kAll, mine, beam & 31);
  return beam < 0 ? kNone : x;
}

// blockIdx.x: the request; blockIdx.y: 32 of its hypotheses, one a lane.
__global__ void __launch_bounds__(kThreads, 1) k_trace(Args g) {
  __shared__ int ancestor[kSegs][32];  // of each beam at a segment's end
  __shared__ int inside[kSegs][32];    // of the hypotheses that end in the segment
  chain();
  const ps_beam_trace_t& a = g.a;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, B = g.beams, T = a.num_steps;
  const int64_t r = blockIdx.x, R = a.num_requests;
  const int h = blockIdx.y * 32 + lane;
  const bool on = h < a.hyps;
  const int64_t at = r * a.hyps + h;
  int L = 0, last = kNone;
  if (on) {
    L = a.lengths ? a.lengths[at] : T;
    last = a.beams_of[at];
    if (L < 0 || L > T || last < -1 || last >= B) {
      if (warp == 0) set_error(g.status, PS_ERR_INVALID_ARG);
      last = kNone;
    }
    if (last < 0) L = 0;
  }
  int entry = kNone;  // the beam at the step before the segments that were done
  const int segs = (T + kSteps - 1) / kSteps;
  for (int s1 = segs; s1 > 0; s1 -= kSegs) {
    const int seg = s1 - kSegs + warp;  // warp 0 the first of these
    const int t0 = seg * kSteps;
    int parent[kSteps], token[kSteps];
    bool bad = false;
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      const int t = t0 + j;
      parent[j] = kNone;
      token[j] = -1;
      if (t >= 0 && t < T && lane < B) {
        const int64_t i = (t * R + r) * B + lane;
        parent[j] = a.parents[i];
        token[j] = a.tokens[i];
      }
    }
    int beam = lane < B ? lane : kNone, own = kNone;
    // parents that lead out of range: noticed where a hypothesis meets one, below
#pragma unroll
    for (int j = kSteps - 1; j >= 0; --j) {
      const int t = t0 + j;
      if (parent[j] < -1 || parent[j] >= B) parent[j] = -2;
      if (t < T && t > 0) {
        beam = look(parent[j], beam);
        if (t == L - 1) own = last;
        own = look(parent[j], own);
      } else if (t == 0 && t == L - 1) {
        own = last;
      }
    }
    ancestor[warp][lane] = beam;
    inside[warp][lane] = own;
    __syncthreads();
    // the beam at this warp's last step: from the segments after it
    int cur = entry;
    for (int w = kSegs - 1; w >= 0; --w) {
      const int end = (s1 - kSegs + w + 1) * kSteps;  // of segment w
      if (w == warp) {
        int b = cur;
#pragma unroll
        for (int j = kSteps - 1; j >= 0; --j) {
          const int t = t0 + j;
          if (t == L - 1) b = last;
          const int tok = look(token[j], b);
          const int up = look(parent[j], b);
          if (on && t >= 0 && t < T) {
            a.out[at * T + t] = t < L && b >= 0 ? tok : -1;
            if (t < L && t > 0 && b >= 0 && up < 0) bad = true;
          }
          if (t > 0 && t < T) b = up;
        }
      }
      // and on to the segment before it
      if (L >= end + 1) cur = cur < 0 ? cur : ancestor[w][cur];
      else if (L > end - kSteps) cur = inside[w][lane];
    }
    if (bad) set_error(g.status, PS_ERR_INVALID_ARG);
    entry = cur;
    __syncthreads();
  }
}

}  // namespace

int32_t launch_trace(const Search& s, const ps_beam_trace_t& a, int32_t* status, cudaStream_t st) {
  const Args g{a, status, s.beams};
  return status_of(launch(k_trace, dim3((unsigned)a.num_requests, (unsigned)((a.hyps + 31) / 32)), kThreads, 0, st, g));
}

}  // namespace psbeam
