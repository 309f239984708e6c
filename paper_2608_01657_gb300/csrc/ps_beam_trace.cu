// ps_beam_trace: sequences of tokens, back through every step's parents.
//
// A hypothesis of L steps that ends in beam b: token L - 1 is tokens[L - 1][b], then
// b <- parents[t][b] from t = L - 1 down to 1.  A chain of dependent lookups, so the
// steps are cut into segments and a CTA takes a request's segments at once, its parents
// as bytes in shared memory.  First every beam at a segment's end is taken to its
// ancestor before the segment, and every hypothesis to that of the segment in which it
// ends; then a thread a hypothesis goes from segment to segment; then the segments are
// gone through once more, from the beams that that gave, and the tokens are picked from
// shared memory, where copies brought them meanwhile (gathered from global memory they
// took as long as all the rest: a sector a lane).  With segments of 32 steps 2047 steps
// are 128 lookups one after another.  What does not fit into shared memory is done in
// rounds, from the last steps on.
#include "ps_beam.cuh"

namespace psbeam {
namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kHyps = 64;          // of a CTA at most
constexpr int kBytes = 206 << 10;  // of tokens, parents and paths
constexpr int kNone = 255;         // no beam

struct Args {
  ps_beam_trace_t a;
  int32_t* status;
  int32_t beams, hyps, steps, seg;  // hypotheses of a CTA, steps of a round and of a segment
  int32_t stride;                   // tokens of a step in shared memory: lanes of neighbouring steps meet at most four times at a bank
  int32_t seg_log2, skew;           // of a segment; bytes between two segments' parents, so that they lie in other banks
  bool words;                       // a step's beams are whole 16-byte words
};

// blockIdx.x: the request; blockIdx.y: 'hyps' of its hypotheses.
__global__ void __launch_bounds__(kThreads) k_trace(const __grid_constant__ Args g) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ int s_len[kHyps];
  __shared__ unsigned char s_last[kHyps], s_enter[kHyps], s_first[kHyps];
  const ps_beam_trace_t& a = g.a;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, B = g.beams, T = a.num_steps, seg = g.seg;
  const int64_t r = blockIdx.x, R = a.num_requests;
  const int h0 = blockIdx.y * g.hyps, H = min(g.hyps, a.hyps - h0);
  int32_t* const token = reinterpret_cast<int32_t*>(smem);       // [steps][stride]
  unsigned char* const parent = smem + (size_t)g.steps * g.stride * 4;      // [steps][B], see 'at'
  unsigned char* const path = parent + g.steps * B + (g.steps / seg + 1) * g.skew;  // [steps][H]
  unsigned char* const map = path + g.steps * g.hyps;            // [segments][B]
  unsigned char* const entry = map + (g.steps / seg + 1) * B;    // [segments][H]
  auto at = [&](int t) { return t * B + (t >> g.seg_log2) * g.skew; };  // where step t's parents are
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
    s_last[tid] = (unsigned char)(last < 0 ? kNone : last);
    s_enter[tid] = kNone;
  }
  for (int t1 = T; t1 > 0;) {
    const int t0 = t1 > g.steps ? t1 - g.steps : 0, n = t1 - t0, segs = (n + seg - 1) / seg;
    const int64_t from = ((int64_t)t0 * R + r) * B;
    __syncthreads();
    // the parents, and the tokens on their way
    auto byte = [&](int p) { return (uint32_t)(p >= 0 && p < B ? p : kNone); };
    if (g.words) {
      const int each = B / 4;
#pragma unroll 4
      for (int i = tid; i < n * each; i += kThreads) {
        const int t = i / each, w = i - t * each;
        const int64_t k = from + (int64_t)t * R * B + 4 * w;
        const int4 p = *reinterpret_cast<const int4*>(a.parents + k);
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(token + t * g.stride + 4 * w)),
                     "l"(a.tokens + k) : "memory");
        *reinterpret_cast<uint32_t*>(parent + at(t) + 4 * w) = byte(p.x) | byte(p.y) << 8 | byte(p.z) << 16 | byte(p.w) << 24;
      }
    } else {
#pragma unroll 4
      for (int i = tid; i < n * B; i += kThreads) {
        const int t = i / B, b = i - t * B;
        const int64_t k = from + (int64_t)t * R * B + b;
        const int p = a.parents[k];
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"((uint32_t)__cvta_generic_to_shared(token + t * g.stride + b)),
                     "l"(a.tokens + k) : "memory");
        parent[at(t) + b] = (unsigned char)byte(p);
      }
    }
    __syncthreads();
    // From beam 'b' at step t0 + t to the one before the steps from 'down' on.
    auto back = [&](int b, int t, int down) {
      if (t0 + down == 0) ++down;  // (what is before the first step is not looked at)
      const unsigned char* p = parent + at(t);
      for (; t >= down && b != kNone; --t, p -= B) b = p[b];
      return b;
    };
    for (int i = tid; i < segs * B; i += kThreads) {
      const int s = i / B, b = i - s * B;
      map[i] = (unsigned char)back(b, min(n, (s + 1) * seg) - 1, s * seg);
    }
    const int of = kThreads - 1 - tid;  // (the threads that have no part in the maps, where there are few)
    if (of < H) {
      const int end = s_len[of] - 1 - t0;
      if (end >= 0 && end < n) s_first[of] = (unsigned char)back(s_last[of], end, end / seg * seg);
    }
    __syncthreads();
    if (tid < H) {
      const int end = s_len[tid] - 1 - t0;
      int cur = s_enter[tid], s = segs - 1;
      if (end < n) {  // it ends here, or before
        cur = end >= 0 ? s_first[tid] : kNone;
        s = end >= 0 ? end / seg - 1 : -1;
      }
      for (; s >= 0; --s) {
        entry[s * H + tid] = (unsigned char)cur;
        if (cur != kNone) cur = map[s * B + cur];
      }
      s_enter[tid] = (unsigned char)cur;
    }
    __syncthreads();
    for (int i = tid; i < segs * H; i += kThreads) {
      const int s = i / H, h = i - s * H, down = s * seg, end = s_len[h] - 1 - t0;
      int t = min(n, down + seg) - 1, b = kNone;
      unsigned char* to = path + t * H + h;
      if (end > t) b = entry[i];
      for (; t > end && t >= down && b == kNone; --t, to -= H) *to = kNone;
      if (t == end) b = s_last[h];
      const unsigned char* p = parent + at(t < 0 ? 0 : t);
      for (; t >= down; --t, to -= H, p -= B) {
        *to = (unsigned char)b;
        if (b != kNone && t0 + t > 0) {
          b = p[b];
          bad = bad || b == kNone;
        }
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    for (int t = warp * 32 + lane; t < n; t += kThreads) {
      const unsigned char* of = path + t * H;
      const int32_t* pick = token + t * g.stride;
      int32_t* to = a.out + (r * a.hyps + h0) * T + t0 + t;
#pragma unroll 8
      for (int h = 0; h < H; ++h, to += T) {
        const int b = of[h];
        *to = b == kNone ? -1 : pick[b];
      }
    }
    t1 = t0;
  }
  if (bad) set_error(g.status, PS_ERR_INVALID_ARG);
}

}  // namespace

int32_t configure_trace() {
  return status_of(cudaFuncSetAttribute(k_trace, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes + (8 << 10)));
}

int32_t launch_trace(const Search& s, const ps_beam_trace_t& a, int32_t* status, cudaStream_t st) {
  Args g{};
  g.a = a;
  g.status = status;
  g.beams = s.beams;
  g.hyps = a.hyps < kHyps ? a.hyps : kHyps;
  // segments of about the root of the steps: a third of the lookups each
  g.seg_log2 = a.num_steps <= 128 ? 3 : (a.num_steps <= 512 ? 4 : 5);
  g.seg = 1 << g.seg_log2;
  g.words = s.beams % 4 == 0 && ((reinterpret_cast<uintptr_t>(a.parents) | reinterpret_cast<uintptr_t>(a.tokens)) & 15) == 0;
  g.stride = !g.words ? s.beams | 1 : s.beams + (s.beams % 8 == 0 ? 4 : 0);
  g.skew = (s.beams + 3) / 4 * 4;
  const int each = 4 * g.stride + s.beams + g.hyps, most = kBytes / each / g.seg * g.seg;
  g.steps = a.num_steps < most ? (a.num_steps + g.seg - 1) / g.seg * g.seg : most;
  const size_t smem = (size_t)g.steps * each + (size_t)(g.steps / g.seg + 1) * (s.beams + g.hyps + g.skew);
  return status_of(launch(k_trace, dim3((unsigned)a.num_requests, (unsigned)((a.hyps + g.hyps - 1) / g.hyps)), kThreads, smem, st, g));
}

}  // namespace psbeam
