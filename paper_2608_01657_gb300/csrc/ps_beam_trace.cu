// ps_beam_trace: sequences of tokens, back through every step's parents.
//
// A hypothesis of L steps that ends in beam b: token L - 1 is tokens[L - 1][b], then
// b <- parents[t][b] from t = L - 1 down to 1.  A chain of dependent lookups, each 40
// cycles in shared memory, so the steps are cut into segments and those into groups,
// and a CTA takes a request's segments at once, its parents as bytes in shared memory.
// First every beam at a segment's end is taken to its ancestor before the segment, then
// every beam at a group's end likewise, from map to map, and every hypothesis to those
// of the segment and the group in which it ends; then a thread a hypothesis goes from
// group to group; then a thread a segment and hypothesis finds the beam it begins with
// and writes the segment's path.  With segments of 32 steps and groups of 8, 2047 steps
// are 87 lookups one after another.  Beam B is none and leads to itself, so that no
// lookup asks whether there is one.  Tokens are picked from shared memory, where copies
// brought them meanwhile (gathered from global memory they took as long as all the
// rest: a sector a lane).  What does not fit into shared memory is done in rounds, from
// the last steps on.
//
// 2047 steps of 128 requests, 8 beams and 13 hypotheses take 13.9 us; their 30 MB need
// 4.6.  The parents take 3.4 (32 bytes of a step are a request's; next to one another
// they took 2.3), the maps beside the tokens' copies 2.2, groups and hypotheses 1.2,
// paths 1.9 and the output 3.0.  64 steps of 4 requests take 3.6, a launch and a chain
// of reads.
#include "ps_beam.cuh"

namespace psbeam {
namespace {

constexpr int kThreads = 1024;
constexpr int kCopiers = kThreads / 2;  // threads that fetch tokens while the others are at the maps
constexpr int kHyps = 64;          // of a CTA at most
constexpr int kBytes = 206 << 10;  // of tokens, parents and paths
constexpr int kAtOnce = 4;         // reads of a thread side by side

struct Args {
  ps_beam_trace_t a;
  int32_t* status;
  int32_t beams, hyps, steps;  // hypotheses of a CTA, steps of a round
  int32_t seg_log2, group_log2;  // steps of a segment, segments of a group
  int32_t parent_stride;  // bytes of a step's parents
  int32_t stride;       // tokens of a step in shared memory: lanes of neighbouring steps meet at most four times at a bank
  int32_t skew;         // bytes between two segments' parents, so that they lie in other banks
  int32_t path_stride;  // bytes of a hypothesis' path
  bool words;           // a step's beams are whole 16-byte words
};

// blockIdx.x: the request; blockIdx.y: 'hyps' of its hypotheses.
__global__ void __launch_bounds__(kThreads) k_trace(const __grid_constant__ Args g) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ int s_len[kHyps];
  __shared__ unsigned char s_last[kHyps], s_enter[kHyps], s_first[kHyps];
  const ps_beam_trace_t& a = g.a;
  const int tid = threadIdx.x, B = g.beams, P = g.parent_stride, T = a.num_steps, seg = 1 << g.seg_log2, group = 1 << g.group_log2;
  const int64_t r = blockIdx.x, R = a.num_requests;
  const int h0 = blockIdx.y * g.hyps, H = min(g.hyps, a.hyps - h0);
  const int most = (g.steps >> g.seg_log2) + 1;  // segments, and one to spare
  int32_t* const token = reinterpret_cast<int32_t*>(smem);              // [steps][stride]
  unsigned char* const path = smem + (size_t)g.steps * g.stride * 4;    // [H][path_stride]
  // of B beams; B is none, and leads to itself
  unsigned char* const parent = path + g.hyps * g.path_stride;          // [steps][P], see 'at'
  unsigned char* const map = parent + g.steps * P + most * g.skew;      // [segments][B + 1]
  unsigned char* const maps = map + most * (B + 1);                     // [groups][B + 1], 'map' itself where a group is a segment
  unsigned char* const entry = maps + (g.group_log2 ? most * (B + 1) : 0);  // [groups][H]
  unsigned char* const whole = g.group_log2 ? maps : map;
  auto at = [&](int t) { return t * P + (t >> g.seg_log2) * g.skew; };  // where step t's parents are
  chain();
  bool bad = false;
  if (tid < H) {
    const int64_t i = r * a.hyps + h0 + tid;
    int len = a.lengths ? a.lengths[i] : T, last = a.beams_of[i];
    if (len < 0 || len > T || last < -1 || last >= B) {
      bad = true;
      last = -1;
    }
    s_len[tid] = last < 0 ? 0 : len;
    s_last[tid] = (unsigned char)(last < 0 ? B : last);
    s_enter[tid] = (unsigned char)B;
  }
  for (int t1 = T; t1 > 0;) {
    const int t0 = t1 > g.steps ? t1 - g.steps : 0, n = t1 - t0, segs = (n + seg - 1) >> g.seg_log2;
    const int groups = (segs + group - 1) >> g.group_log2;
    const int64_t from = ((int64_t)t0 * R + r) * B;
    __syncthreads();
    // The parents.  Those of the first step are not looked at, nor are there any past the
    // last one: the beams themselves take their places.
    auto byte = [&](int p, int t, int b) { return (uint32_t)(t0 + t == 0 || t >= n ? b : (p >= 0 && p < B ? p : B)); };
    const int rows = (n + 3) & ~3;
    if (g.words) {
      const int each = B / 4;
      for (int i0 = tid; i0 < rows * each; i0 += kAtOnce * kThreads) {
        int4 p[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const int i = i0 + u * kThreads, t = i / each, w = i - t * each;
          p[u] = make_int4(0, 0, 0, 0);
          if (t < n) p[u] = *reinterpret_cast<const int4*>(a.parents + from + (int64_t)t * R * B + 4 * w);
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const int i = i0 + u * kThreads, t = i / each, b = 4 * (i - t * each);
          if (t < rows) {
            uint32_t* to = reinterpret_cast<uint32_t*>(parent + at(t) + b);
            to[0] = byte(p[u].x, t, b) | byte(p[u].y, t, b + 1) << 8 | byte(p[u].z, t, b + 2) << 16 | byte(p[u].w, t, b + 3) << 24;
            if (b + 4 == B) to[1] = B;
          }
        }
      }
    } else {
      for (int i0 = tid; i0 < rows * B; i0 += kAtOnce * kThreads) {
        int p[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const int i = i0 + u * kThreads, t = i / B;
          p[u] = t < n ? a.parents[from + (int64_t)t * R * B + (i - t * B)] : 0;
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const int i = i0 + u * kThreads, t = i / B, b = i - t * B;
          if (t < rows) {
            parent[at(t) + b] = (unsigned char)byte(p[u], t, b);
            if (b + 1 == B) parent[at(t) + B] = (unsigned char)B;
          }
        }
      }
    }
    __syncthreads();
    // From beam 'b' at step t0 + t to the one before the steps from 'down' on.
    auto back = [&](int b, int t, int down) {
      const unsigned char* p = parent + at(t);
#pragma unroll 8
      for (; t >= down; --t, p -= P) b = p[b];
      return b;
    };
    // From beam 'b' at the end of segment s to the one before the segments from 'down' on.
    auto back_segments = [&](int b, int s, int down) {
      const unsigned char* p = map + s * (B + 1);
#pragma unroll 4
      for (; s >= down; --s, p -= B + 1) b = p[b];
      return b;
    };
    if (tid < kThreads - kCopiers) {
      for (int i = tid; i < segs * B; i += kThreads - kCopiers) {
        const int s = i / B, b = i - s * B;
        if (b == 0) map[i + s + B] = (unsigned char)B;
        map[i + s] = (unsigned char)back(b, min(n, (s + 1) << g.seg_log2) - 1, s << g.seg_log2);
      }
    } else {
      const int c = kThreads - 1 - tid;
      if (c < H) {
        const int end = s_len[c] - 1 - t0;
        if (end >= 0 && end < n) s_first[c] = (unsigned char)back(s_last[c], end, end & -seg);
      }
      // the tokens, on their way
      const int W = g.words ? B / 4 : B, rise = kCopiers / W, rest = kCopiers - rise * W;
      int t = (tid - (kThreads - kCopiers)) / W, w = tid - (kThreads - kCopiers) - t * W;
#pragma unroll 4
      while (t < n) {
        const int32_t* src = a.tokens + from + (int64_t)t * R * B;
        const uint32_t to = (uint32_t)__cvta_generic_to_shared(token + t * g.stride);
        if (g.words) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + 16 * w), "l"(src + 4 * w) : "memory");
        else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to + 4 * w), "l"(src + w) : "memory");
        t += rise;
        w += rest;
        if (w >= W) w -= W, ++t;
      }
    }
    __syncthreads();
    if (g.group_log2) {
      for (int i = tid; i < groups * (B + 1); i += kThreads) {
        const int q = i / (B + 1), b = i - q * (B + 1);
        maps[i] = (unsigned char)back_segments(b, min(segs, (q + 1) << g.group_log2) - 1, q << g.group_log2);
      }
      const int c = kThreads - 1 - tid;
      if (c < H) {  // before the group in which it ends
        const int end = s_len[c] - 1 - t0, s = end >> g.seg_log2;
        if (end >= 0 && end < n) s_enter[c] = (unsigned char)back_segments(s_first[c], s - 1, s & -group);
      }
      __syncthreads();
    }
    if (tid < H) {
      const int end = s_len[tid] - 1 - t0;
      int cur = s_enter[tid], q = groups - 1;
      if (end < n) {  // it ends here, or before
        if (end < 0) cur = B;
        else if (!g.group_log2) cur = s_first[tid];
        q = end >= 0 ? (end >> g.seg_log2 >> g.group_log2) - 1 : -1;
      }
#pragma unroll 4
      for (; q >= 0; --q) {
        entry[q * H + tid] = (unsigned char)cur;
        cur = whole[q * (B + 1) + cur];
      }
      s_enter[tid] = (unsigned char)cur;
    }
    __syncthreads();
    // a segment's path, four steps a word
    for (int i = tid; i < segs * H; i += kThreads) {
      const int s = i / H, h = i - s * H, down = s << g.seg_log2, q = s >> g.group_log2, end = s_len[h] - 1 - t0, ends = end >> g.seg_log2;
      int t = (min(n, down + seg) - 1) | 3, b = B;
      if (end >= n || ends > s) {  // what it comes from: the end of the group, or its own
        const bool here = end < n && ends >> g.group_log2 == q;
        b = back_segments(here ? s_first[h] : entry[q * H + h], (here ? ends : min(segs, (q + 1) << g.group_log2)) - 1, s + 1);
      }
      uint32_t* to = reinterpret_cast<uint32_t*>(path + h * g.path_stride + t - 3);
      const unsigned char* p = parent + at(t);
      const bool ending = ends == s && end < n;  // (a step past the round may lie in its last word)
      bool some = b != B;
      for (; t >= down; t -= 4, --to) {
        uint32_t word = 0;
        if (ending && (t ^ end) >> 2 == 0) {
          some = true;
          for (int u = 0; u < 4; ++u, p -= P) {
            if (t - u == end) b = s_last[h];
            word = word << 8 | b;
            b = p[b];
          }
        } else {
#pragma unroll
          for (int u = 0; u < 4; ++u, p -= P) {
            word = word << 8 | b;
            b = p[b];
          }
        }
        *to = word;
      }
      bad = bad || (some && b == B);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    for (int t = tid; t < n; t += kThreads) {
      const unsigned char* of = path + t;
      const int32_t* pick = token + t * g.stride;
      int32_t* to = a.out + (r * a.hyps + h0) * T + t0 + t;
#pragma unroll 8
      for (int h = 0; h < H; ++h, to += T, of += g.path_stride) {
        const int b = *of;
        *to = b == B ? -1 : pick[b];
      }
    }
    t1 = t0;
  }
  if (bad) set_error(g.status, PS_ERR_INVALID_ARG);
}

}  // namespace

int32_t configure_trace() {
  return status_of(cudaFuncSetAttribute(k_trace, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes + (16 << 10)));
}

int32_t launch_trace(const Search& s, const ps_beam_trace_t& a, int32_t* status, cudaStream_t st) {
  Args g{};
  g.a = a;
  g.status = status;
  g.beams = s.beams;
  g.hyps = a.hyps < kHyps ? a.hyps : kHyps;
  // up to 128 steps: segments of about the root, without groups
  g.seg_log2 = a.num_steps <= 128 ? 3 : (a.num_steps <= 512 ? 4 : 5);
  g.group_log2 = a.num_steps <= 128 ? 0 : 3;
  const int seg = 1 << g.seg_log2;
  g.words = s.beams % 4 == 0 && ((reinterpret_cast<uintptr_t>(a.parents) | reinterpret_cast<uintptr_t>(a.tokens)) & 15) == 0;
  g.stride = !g.words ? s.beams | 1 : s.beams + (s.beams % 8 == 0 ? 4 : 0);
  g.parent_stride = s.beams + (g.words ? 4 : 1);
  g.skew = (s.beams + 3) / 4 * 4;
  const int each = 4 * g.stride + g.parent_stride + g.hyps, most = kBytes / each / seg * seg;
  g.steps = a.num_steps < most ? (a.num_steps + seg - 1) / seg * seg : most;
  g.path_stride = g.steps + 4;  // an odd number of words
  const int segs = g.steps / seg + 1;
  const size_t smem = (size_t)g.steps * each + 4 * g.hyps + (size_t)segs * (2 * s.beams + 2 + g.hyps + g.skew);
  return status_of(launch(k_trace, dim3((unsigned)a.num_requests, (unsigned)((a.hyps + g.hyps - 1) / g.hyps)), kThreads, smem, st, g));
}

}  // namespace psbeam
