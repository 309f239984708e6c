// ps_beam_select: the best continuations of a request's beams.
//
// Of a beam with score c and logits x, token v continues it with the score c + x_v
// - lse, lse = log sum_u exp x_u.  Within a beam the order is the logits', and a
// request's best are among its beams' best.  A row is read once, in words of 16
// bytes, for two things: a sum of 2^((x - ref) log2 e), whose reference rises with the
// greatest logit seen, and the 'beams' words of the greatest logits.  The row's best
// tokens are in those words: every word that comes before one of theirs (by its
// greatest logit, equal ones by place) holds a token that comes before it, too.  So
// single elements are looked at in a few words only, at the end.  Words are kept as
// whole numbers, the logit's bits in order and then the complement of the place, so
// that no two are equal.
//
// Bound by HBM.  A row is cut into parts, a CTA each, so that a few rows fill the GPU,
// too; the last CTA of a request to finish puts the parts together, in an order that
// does not depend on which one it is.
//
// A warp reads 2 KB at a time through a ring in shared memory, three of them under way
// while it works on one.  It keeps a list of 32 sorted across its lanes; what is greater than the list's
// beams-th enters a queue, 32 of which are sorted and merged at a time.
//
// Neighbours in the order of scores may be nearer than 32 bits tell: differences
// from the reference are exact or rounded once, log2 e has two parts, the lanes' sums
// are added as whole numbers of 2^-32, and scores in 64 bits.
#include "ps_beam.cuh"

namespace psbeam {
namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;
constexpr int kCtasPerSm = 6;
constexpr int kVecs = 4;                 // words of a lane and chunk
constexpr int kChunk = 32 * kVecs;       // words of a chunk
constexpr int kStages = 4;               // chunks of a warp's ring
// A warp has so many chunks at least, where there are as many.
constexpr int kLeastChunks = 2;
constexpr float kLog2e = 1.44269502f, kLog2eRest = 1.92596303e-8f;  // their sum: log2 e to 2^-48
constexpr double kLn2 = 0.693147180559945309;
constexpr unsigned kAll = 0xFFFFFFFFu;

struct Args {
  ps_beam_select_t a;
  Search s;
  int32_t* status;
  int32_t parts;  // of a row
};

// ---- elements ---------------------------------------------------------------------
// The greater, NaN if one is.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
template <typename T>
struct Elem;
template <>
struct Elem<float> {
  static constexpr int N = 4;  // of a 16-byte word
  static __device__ __forceinline__ void wide(const uint4& v, float (&x)[N]) {
    x[0] = __uint_as_float(v.x), x[1] = __uint_as_float(v.y), x[2] = __uint_as_float(v.z), x[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ uint4 narrow(const float (&x)[N]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
  static __device__ __forceinline__ uint4 none() { return make_uint4(0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u); }
  static __device__ __forceinline__ float top(const uint4& v) {
    return max_nan(max_nan(__uint_as_float(v.x), __uint_as_float(v.y)), max_nan(__uint_as_float(v.z), __uint_as_float(v.w)));
  }
  static __device__ __forceinline__ uint32_t max1(uint32_t a, uint32_t b) { return __float_as_uint(max_nan(__uint_as_float(a), __uint_as_float(b))); }
  static __device__ __forceinline__ float one(const void* p) { return *static_cast<const float*>(p); }
};
template <typename H>
struct Elem16 {
  static constexpr int N = 8;
  static __device__ __forceinline__ void wide(const uint4& v, float (&x)[N]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = pskv::Num<H>::unpack(w[i]);
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
  static __device__ __forceinline__ uint4 narrow(const float (&x)[N]) {  // of values that H holds
    return make_uint4(pskv::Num<H>::pack(x[0], x[1]), pskv::Num<H>::pack(x[2], x[3]), pskv::Num<H>::pack(x[4], x[5]),
                      pskv::Num<H>::pack(x[6], x[7]));
  }
  // The greatest, NaN if one is.
  static __device__ __forceinline__ float top(const uint4& v) {
    const float2 f = pskv::Num<H>::unpack(max1(max1(v.x, v.y), max1(v.z, v.w)));
    return max_nan(f.x, f.y);
  }
  static __device__ __forceinline__ uint32_t max1(uint32_t a, uint32_t b) {
    uint32_t r;
    if (pskv::Num<H>::kBf16) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ uint4 none() {  // -infinity
    constexpr uint32_t w = pskv::Num<H>::kBf16 ? 0xFF80FF80u : 0xFC00FC00u;
    return make_uint4(w, w, w, w);
  }
};
template <>
struct Elem<__nv_bfloat16> : Elem16<__nv_bfloat16> {
  static __device__ __forceinline__ float one(const void* p) { return __bfloat162float(*static_cast<const __nv_bfloat16*>(p)); }
};
template <>
struct Elem<__half> : Elem16<__half> {
  static __device__ __forceinline__ float one(const void* p) { return __half2float(*static_cast<const __half*>(p)); }
};
// The greatest of several words, place by place.
template <typename T, int M>
__device__ __forceinline__ uint4 greatest(const uint4 (&v)[M]) {
  uint4 m = v[0];
#pragma unroll
  for (int j = 1; j < M; ++j)
    m = make_uint4(Elem<T>::max1(m.x, v[j].x), Elem<T>::max1(m.y, v[j].y), Elem<T>::max1(m.z, v[j].z), Elem<T>::max1(m.w, v[j].w));
  return m;
}

// ---- keys ---------------------------------------------------------------------------
// The bits of x as a whole number in x's order; -0 is 0.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return (int32_t)u < 0 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t o) { return __uint_as_float((int32_t)o < 0 ? o & 0x7FFFFFFFu : ~o); }
// Of a logit and the place of its token (or of its word).
__device__ __forceinline__ uint64_t key_of(float x, int place) { return (uint64_t)ordered(x) << 32 | (uint32_t)~place; }
__device__ __forceinline__ float logit_of(uint64_t key) { return unordered((uint32_t)(key >> 32)); }
__device__ __forceinline__ int place_of(uint64_t key) { return (int)~(uint32_t)key; }
// None of -infinity is greater.
constexpr uint64_t kNoKey = 0x007FFFFFFFFFFFFFull;

__device__ __forceinline__ void exchange(uint64_t& x, int other, bool greater) {
  const uint64_t y = __shfl_xor_sync(kAll, x, other);
  x = (x > y) == greater ? x : y;
}
// 32 numbers, one a lane, from the greatest to the least.
__device__ __forceinline__ uint64_t sort32(uint64_t x, int lane) {
#pragma unroll
  for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
    for (int j = k >> 1; j > 0; j >>= 1) exchange(x, j, ((lane & j) == 0) == ((lane & k) == 0));
  return x;
}
__device__ __forceinline__ uint32_t sort32(uint32_t x, int lane) {
#pragma unroll
  for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
    for (int j = k >> 1; j > 0; j >>= 1) {
      const uint32_t y = __shfl_xor_sync(kAll, x, j);
      x = ((lane & j) == 0) == ((lane & k) == 0) ? max(x, y) : min(x, y);
    }
  return x;
}
// The 32 greatest of two such lists, as one.
__device__ __forceinline__ uint64_t merge32(uint64_t x, uint64_t y, int lane) {
  const uint64_t z = __shfl_sync(kAll, y, 31 - lane);
  x = x > z ? x : z;
#pragma unroll
  for (int j = 16; j > 0; j >>= 1) exchange(x, j, (lane & j) == 0);
  return x;
}

__device__ __forceinline__ bool ends(const Search& s, int token) {
  bool e = false;
#pragma unroll
  for (int i = 0; i < PS_BEAM_MAX_END; ++i) e = e || (i < s.num_end && s.end[i] == token);
  return e;
}

// A warp's best so far.
constexpr int kQueue = 64;
struct Best {
  uint64_t list;    // of the lane
  uint64_t floor;   // what enters is greater
  int queued;
  uint64_t* queue;  // [kQueue] of the warp
  int keep, lane;
  __device__ __forceinline__ void raise(uint64_t to) { floor = floor > to ? floor : to; }
  __device__ __forceinline__ void flush() {  // the last 32 of the queue, or all of it
    const int from = queued > 32 ? queued - 32 : 0;
    __syncwarp();
    const uint64_t q = from + lane < queued ? queue[from + lane] : 0;
    __syncwarp();
    queued = from;
    list = merge32(list, sort32(q, lane), lane);
    raise(__shfl_sync(kAll, list, keep - 1));
  }
  __device__ __forceinline__ void add(uint64_t key, bool on) {
    const unsigned m = __ballot_sync(kAll, on);
    if (on) queue[queued + __popc(m & ((1u << lane) - 1))] = key;
    queued += __popc(m);
    if (queued >= 32) flush();
  }
  // A smaller logit does not enter.
  __device__ __forceinline__ float least() const { return logit_of(floor + 1); }
};

// ---- sums -----------------------------------------------------------------------------
// exp(x) for x <= 0, the exponent in two parts; 0 below 2^-144 (where the parts are not finite at last).
__device__ __forceinline__ float exp_of(float x) {
  const float t = x * kLog2e;
  return x < -100.0f ? 0.0f : pskv::ex2(t) * (1.0f + 0.693147181f * fmaf(x, kLog2eRest, fmaf(x, kLog2e, -t)));
}
// log(u 2^-32) for u > 0, to 4e-9.  With u = 2^e m, 0.7 < m < 1.42, and f = (m - 1) /
// (m + 1): log m = 2 (f + f^3 / 3 + f^5 / 5 + ...), the first term in two parts.
__device__ __forceinline__ double log_of(uint64_t u) {
  const int lz = __clzll((long long)u);
  const uint64_t n = u << lz;
  float hi = (float)(uint32_t)(n >> 40) * 0x1p-23f, lo = (float)((uint32_t)(n >> 16) & 0xFFFFFFu) * 0x1p-47f;
  int e = 31 - lz;
  if (hi > 1.41421354f) hi *= 0.5f, lo *= 0.5f, ++e;
  const float num = hi - 1.0f, den = hi + 1.0f, den_lo = hi - (den - 1.0f) + lo;
  const float f = num / den, z = f * f;
  const float f_lo = (fmaf(-f, den, num) + lo - f * den_lo) / den;
  float p = fmaf(z, 1.0f / 13, 1.0f / 11);
  p = fmaf(p, z, 1.0f / 9);
  p = fmaf(p, z, 1.0f / 7);
  p = fmaf(p, z, 1.0f / 5);
  p = fmaf(p, z, 1.0f / 3) * z;
  return (double)e * kLn2 + ((double)(2.0f * f) + (double)(2.0f * fmaf(f, p, f_lo)));
}

// A lane's sum of exp(x - ref).
struct Sum {
  float ref, sum;
  __device__ __forceinline__ void raise(float to) {
    if (to > ref) {
      sum = ref == -INFINITY ? 0.0f : sum * pskv::ex2((ref - to) * kLog2e);
      ref = to;
    }
  }
  // What is subtracted: nothing while all are -infinity.
  __device__ __forceinline__ float base() const { return ref == -INFINITY ? 0.0f : ref; }
};
__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(kAll, x, o));
  return x;
}
__device__ __forceinline__ uint64_t warp_sum(uint64_t x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(kAll, x, o);
  return x;
}

// ---- a part of a row ------------------------------------------------------------------
// Words are counted from the row's first element on, wherever that lies in memory, so
// that a row's sum does not depend on its address: equal beams are equal to the last
// bit.  A ring slot holds aligned words.  Where the row starts 'shift' elements into
// one, a word is put together from two; elements of aligned words that are not the
// row's are not read.
constexpr int kSlot = kChunk + 1;  // with the word after the chunk's

template <typename T>
struct Row {
  static constexpr int N = Elem<T>::N;
  const T* row;
  int V, shift;
  uint4* ring;  // [kStages][kSlot] of the warp
  int lane;
  __device__ __forceinline__ void fetch_word(uint4* to, int w) const {
    const int first = w * N - shift;
    if (first >= 0 && first + N <= V) {
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(row + first) : "memory");
    } else {
      float x[N];
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = -INFINITY;
      if (first < V) {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (first + e >= 0 && first + e < V) x[e] = Elem<T>::one(row + first + e);
      }
      *to = Elem<T>::narrow(x);
    }
  }
  __device__ __forceinline__ void fetch(int c, int stage) const {
    uint4* slot = ring + stage * kSlot;
    if (c > 0 && (c + 1) * kChunk * N + N <= V) {  // all of it, and the word after it, is the row's
      const uint32_t to = (uint32_t)__cvta_generic_to_shared(slot) + lane * 16;
      const char* from = reinterpret_cast<const char*>(row - shift) + ((int64_t)c * kChunk + lane) * 16;
#pragma unroll
      for (int j = 0; j < kVecs; ++j)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + 512 * j), "l"(from + 512 * j) : "memory");
      if (shift != 0 && lane == 0)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + 512 * kVecs), "l"(from + 512 * kVecs) : "memory");
      return;
    }
#pragma unroll 1
    for (int j = 0; j < kVecs; ++j) fetch_word(slot + 32 * j + lane, c * kChunk + 32 * j + lane);
    if (shift != 0 && lane == 0) fetch_word(slot + kChunk, c * kChunk + kChunk);
  }
  __device__ __forceinline__ void take(int stage, uint4 (&v)[kVecs]) const {
    const uint4* slot = ring + stage * kSlot + lane;
#pragma unroll
    for (int j = 0; j < kVecs; ++j) v[j] = slot[32 * j];
    if (shift == 0) return;
    const int words = shift * (int)sizeof(T) / 4, bits = shift * (int)sizeof(T) % 4 * 8;
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
      const uint4 n = slot[32 * j + 1];
      uint32_t x[8] = {v[j].x, v[j].y, v[j].z, v[j].w, n.x, n.y, n.z, n.w};
      if (words & 2) {
#pragma unroll
        for (int i = 0; i < 6; ++i) x[i] = x[i + 2];
      }
      if (words & 1) {
#pragma unroll
        for (int i = 0; i < 5; ++i) x[i] = x[i + 1];
      }
      v[j] = make_uint4(__funnelshift_r(x[0], x[1], bits), __funnelshift_r(x[1], x[2], bits), __funnelshift_r(x[2], x[3], bits),
                        __funnelshift_r(x[3], x[4], bits));
    }
  }
};

template <typename T>
__device__ __forceinline__ void scan_part(const Args& g, const Row<T>& row, int part, Best& best, Sum& sum, float& most) {
  constexpr int N = Elem<T>::N;
  const int lane = row.lane, warp = threadIdx.x >> 5;
  const int words = (row.V - 1) / N + 1;
  const int chunks = (words + kChunk - 1) / kChunk;
  const int c0 = (int)((int64_t)chunks * part / g.parts) + warp, c1 = (int)((int64_t)chunks * (part + 1) / g.parts);
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) {
    if (c0 + i * kWarps < c1) row.fetch(c0 + i * kWarps, i);
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  int stage = 0, end_chunk = g.s.num_end > 0 ? 0 : 1 << 30;
  for (int c = c0; c < c1; c += kWarps) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
    __syncwarp();  // the lanes' copies are there, and all have read the slot that is filled next
    uint4 v[kVecs];
    row.take(stage, v);
    if (c + (kStages - 1) * kWarps < c1) row.fetch(c + (kStages - 1) * kWarps, stage == 0 ? kStages - 1 : stage - 1);
    asm volatile("cp.async.commit_group;" ::: "memory");
    stage = stage == kStages - 1 ? 0 : stage + 1;
    float all = Elem<T>::top(greatest<T>(v));
    most = max_nan(most, all);
    sum.raise(all);
    const float base = sum.base();
    const uint64_t minus = pskv::pack2(-base, -base), hi = pskv::pack2(kLog2e, kLog2e), lo = pskv::pack2(kLog2eRest, kLog2eRest);
    uint64_t s0 = 0, s1 = 0;
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
      float x[N];
      Elem<T>::wide(v[j], x);
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        const uint64_t d = pskv::add2(pskv::pack2(x[e], x[e + 1]), minus);
        const float2 t = pskv::unpack2(pskv::fma2(d, lo, pskv::mul2(d, hi)));
        const uint64_t p = pskv::pack2(pskv::ex2(t.x), pskv::ex2(t.y));
        if (e & 2) s1 = pskv::add2(s1, p);
        else s0 = pskv::add2(s0, p);
      }
    }
    const float2 f = pskv::unpack2(pskv::add2(s0, s1));
    sum.sum += f.x + f.y;
    const int w0 = c * kChunk + lane;
    if (c >= end_chunk) {  // an end token is among these, or one lies behind: end tokens do not count
      unsigned out = 0;
      end_chunk = 1 << 30;
      for (int i = 0; i < g.s.num_end; ++i) {
        const int word = g.s.end[i] / N, w = word - w0;
        if (w >= 0 && w < kChunk && (w & 31) == 0) out |= 1u << (w / 32 * N + g.s.end[i] % N);
        if (word / kChunk > c) end_chunk = min(end_chunk, word / kChunk);
      }
      if (out) {
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
          float x[N];
          Elem<T>::wide(v[j], x);
#pragma unroll
          for (int e = 0; e < N; ++e) x[e] = out >> (j * N + e) & 1 ? -INFINITY : x[e];
          v[j] = Elem<T>::narrow(x);
        }
        all = Elem<T>::top(greatest<T>(v));
      }
    }
    if (c == c0) {  // the beams-th of the lanes' greatest: so many words are no smaller
      const uint32_t s = __shfl_sync(kAll, sort32(ordered(all), lane), best.keep - 1);
      best.raise(((uint64_t)s << 32) - 1);
    }
    const float least = best.least();
    if (!__any_sync(kAll, all >= least)) continue;
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
      const float top = Elem<T>::top(v[j]);
      if (!__any_sync(kAll, top >= least)) continue;
      const uint64_t key = key_of(top, w0 + 32 * j);
      best.add(key, key > best.floor);
    }
  }
  while (best.queued > 0) best.flush();
}

// ---- the parts of a request -------------------------------------------------------------
// A candidate of a request: its score as a whole number in the scores' order, and its
// beam and place in the beam's list.
struct Cand {
  long long score;
  int at;  // beam 32 + place
  __device__ __forceinline__ bool before(const Cand& y) const { return score != y.score ? score > y.score : at < y.at; }
  __device__ __forceinline__ Cand shfl(int from) const { return {__shfl_sync(kAll, score, from), __shfl_sync(kAll, at, from)}; }
  __device__ __forceinline__ float value() const { return (float)__longlong_as_double(score < 0 ? score ^ 0x7FFFFFFFFFFFFFFFll : score); }
};
constexpr int kNobody = 1 << 20;  // a place after every candidate's
__device__ __forceinline__ Cand cand(double score, int at) {
  const long long b = __double_as_longlong(score + 0.0);
  return {b < 0 ? b ^ 0x7FFFFFFFFFFFFFFFll : b, at};
}
__device__ __forceinline__ Cand nobody(int lane) { return {(long long)0x8000000000000000ull, kNobody + lane}; }
__device__ __forceinline__ void exchange(Cand& x, int lane, int other, bool first) {
  const Cand y = x.shfl(lane ^ other);
  if (x.before(y) != first) x = y;
}
__device__ __forceinline__ Cand sort32(Cand x, int lane) {
#pragma unroll
  for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
    for (int j = k >> 1; j > 0; j >>= 1) exchange(x, lane, j, ((lane & j) == 0) == ((lane & k) == 0));
  return x;
}
__device__ __forceinline__ Cand merge32(Cand x, const Cand& y, int lane) {
  const Cand z = y.shfl(31 - lane);
  if (z.before(x)) x = z;
#pragma unroll
  for (int j = 16; j > 0; j >>= 1) exchange(x, lane, j, (lane & j) == 0);
  return x;
}

// The best tokens of a row, from the words that hold them.
template <typename T>
__device__ __forceinline__ uint64_t best_tokens(const Args& g, const T* row, uint64_t words, uint64_t* queue, int lane) {
  constexpr int N = Elem<T>::N, kEach = 32 / N;  // words that a warp looks at together
  const int B = g.s.beams;
  // each of the words has a token that is no smaller than the last one's
  const uint64_t last = __shfl_sync(kAll, words, B - 1);
  Best best{0, kNoKey, 0, queue, B, lane};
  if (last > kNoKey) best.raise((last >> 32 << 32) - 1);
  float x[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint64_t word = __shfl_sync(kAll, words, i * kEach + lane / N);
    const int token = place_of(word) * N + lane % N;
    x[i] = -INFINITY;
    if (i * kEach + lane / N < B && word > kNoKey && token < g.s.vocab) x[i] = Elem<T>::one(row + token);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (i * kEach >= B) break;
    const int token = place_of(__shfl_sync(kAll, words, i * kEach + lane / N)) * N + lane % N;
    const uint64_t key = key_of(x[i], token);
    best.add(key, key > best.floor && !ends(g.s, token));
  }
  while (best.queued > 0) best.flush();
  return best.list;
}

struct Joined {
  uint64_t keys[PS_BEAM_MAX_BEAMS][32];  // the beams' best tokens
  uint64_t sum[PS_BEAM_MAX_BEAMS];       // of 2^-32 exp(x - ref), 0: no candidates
  double total[PS_BEAM_MAX_BEAMS];       // its logarithm
  float score[PS_BEAM_MAX_BEAMS], ref[PS_BEAM_MAX_BEAMS];
  Cand lists[kWarps][32];
  Cand best[32];
  // The reference, which may be far from 0, is subtracted first.
  __device__ __forceinline__ double of(int b, float logit) const {
    return (double)score[b] + (((double)logit - (double)ref[b]) - total[b]);
  }
};
struct Shared {
  uint64_t queue[kWarps][kQueue];
  union {
    struct {
      uint4 ring[kWarps][kStages * kSlot];
      uint64_t lists[kWarps][32];
    } scan;
    Joined joined;
  };
  uint64_t sums[kWarps];
  float refs[kWarps];
  int bad[kWarps];
  bool last;
};

// The request's outputs, by the threads of its last CTA.
template <typename T>
__device__ __forceinline__ void finish(const Args& g, int r, uint64_t (*queue)[kQueue], Joined& s) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, B = g.s.beams, S = g.parts, E = g.s.num_end;
  const T* logits = static_cast<const T*>(g.a.logits) + r * g.a.request_stride;
  for (int b = warp; b < B; b += kWarps) {  // the beams' sums, a part a lane
    const int64_t row = (int64_t)r * B + b;
    const float c = g.a.scores[row];
    Part p{0, -INFINITY, 0};
    if (lane < S && c - c == 0) {
      const uint4 q = __ldcg(reinterpret_cast<const uint4*>(g.s.parts + row * S + lane));
      p = Part{(uint64_t)q.y << 32 | q.x, __uint_as_float(q.z), (int32_t)q.w};
    }
    const float ref = warp_max(p.ref);
    const bool bad = __any_sync(kAll, p.bad) || (c != -INFINITY && !(c - c == 0));
    if (p.ref < ref) p.sum = p.ref == -INFINITY ? 0 : __double2ull_rn((double)p.sum * (double)exp_of(p.ref - ref));
    const uint64_t sum = warp_sum(p.sum);
    if (lane == 0) {
      if (bad) set_error(g.status, PS_ERR_INVALID_ARG);
      s.score[b] = c;
      s.ref[b] = ref;
      s.sum[b] = bad ? 0 : sum;  // 0: no token may follow
    }
  }
  __syncthreads();
  if (threadIdx.x < B && s.sum[threadIdx.x] != 0) s.total[threadIdx.x] = log_of(s.sum[threadIdx.x]);
  __syncthreads();
  Cand mine = nobody(lane);
  for (int b = warp; b < B; b += kWarps) {
    if (s.sum[b] == 0) continue;
    const uint64_t* keys = g.s.keys + ((int64_t)r * B + b) * S * B + lane;
    uint64_t list = lane < B ? __ldcg(keys) : 0;
    for (int i = 1; i < S; i += 4) {
      uint64_t k[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) k[u] = lane < B && i + u < S ? __ldcg(keys + (i + u) * B) : 0;
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (i + u < S) list = merge32(list, k[u], lane);
    }
    list = best_tokens(g, logits + b * g.a.beam_stride, list, queue[warp], lane);
    s.keys[b][lane] = list;
    const Cand x = lane < B && list > kNoKey ? cand(s.of(b, logit_of(list)), b * 32 + lane) : nobody(lane);
    mine = b < kWarps ? x : merge32(mine, x, lane);
  }
  s.lists[warp][lane] = mine;
  __syncthreads();
  const int64_t to = (int64_t)r * B + lane;
  Cand last = nobody(lane);
  if (warp == 0) {
    for (int w = 1; w < kWarps && w < B; ++w) mine = merge32(mine, s.lists[w][lane], lane);
    s.best[lane] = mine;
    if (lane < B) {
      const bool on = mine.at < kNobody;
      g.a.tokens[to] = on ? place_of(s.keys[mine.at >> 5][mine.at & 31]) : -1;
      g.a.parents[to] = on ? mine.at >> 5 : -1;
      g.a.scores_out[to] = on ? mine.value() : -INFINITY;
    }
  } else if (warp == 1 && g.a.ended_tokens) {
    // the end tokens' candidates, the 32 first: 'at' is beam 32 + the end token's
    // number, and the numbers rise with the tokens
    for (int i0 = 0; i0 < B * E; i0 += 32) {
      const int i = i0 + lane, b = i / E;
      Cand x = nobody(lane);
      if (i < B * E && s.sum[b] != 0) {
        const float l = Elem<T>::one(logits + b * g.a.beam_stride + g.s.end[i % E]);
        if (l > -INFINITY) x = cand(s.of(b, l), b * 32 + i % E);
      }
      x = sort32(x, lane);
      last = i0 ? merge32(last, x, lane) : x;
    }
  }
  if (!g.a.ended_tokens) return;
  __syncthreads();
  if (warp != 1) return;
  // its place among all candidates: those of its kind before it are the lanes below
  int place = lane;
  bool on = last.at < kNobody;
  const int beam = last.at >> 5, token = on ? g.s.end[last.at & 31] : -1;
  uint64_t key = 0;
  if (on) key = key_of(Elem<T>::one(logits + beam * g.a.beam_stride + token), token);
  for (int i = 0; i < B; ++i) {
    const Cand x = s.best[i];
    bool first = x.before(last);
    if (x.score == last.score && x.at < kNobody && x.at >> 5 == beam) first = s.keys[beam][x.at & 31] > key;
    place += first;
  }
  on = on && place < B;  // (places rise with the lanes)
  if (lane < B) {
    g.a.ended_tokens[to] = on ? token : -1;
    g.a.ended_parents[to] = on ? beam : -1;
    g.a.ended_scores[to] = on ? last.value() : -INFINITY;
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads, kCtasPerSm) k_select(Args g) {
  __shared__ __align__(16) Shared sh;
  chain();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, B = g.s.beams;
  const int64_t row = blockIdx.x / g.parts;
  const int part = (int)(blockIdx.x % g.parts), r = (int)(row / B), b = (int)(row % B);
  const float c = g.a.scores[row];
  if (c - c == 0) {  // (a score that is not finite: nothing is read of the row)
    Best best{0, kNoKey, 0, sh.queue[warp], B, lane};
    Sum sum{-INFINITY, 0.0f};
    float most = -INFINITY;
    const T* from = static_cast<const T*>(g.a.logits) + r * g.a.request_stride + b * g.a.beam_stride;
    const Row<T> x{from, g.s.vocab, (int)(reinterpret_cast<uintptr_t>(from) & 15) / (int)sizeof(T), sh.scan.ring[warp], lane};
    scan_part(g, x, part, best, sum, most);
    // the lanes' and the warps' sums and lists
    const float own = warp_max(sum.ref);
    const bool bad = __any_sync(kAll, !(most < INFINITY));
    sh.scan.lists[warp][lane] = best.list;
    if (lane == 0) sh.refs[warp] = own, sh.bad[warp] = bad;
    __syncthreads();
    float ref = sh.refs[0];
    int any = sh.bad[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) ref = fmaxf(ref, sh.refs[w]), any |= sh.bad[w];
    const float scaled = sum.ref == -INFINITY ? 0.0f : sum.sum * exp_of(sum.ref - ref);
    const uint64_t total = warp_sum(__float2ull_rn(scaled * 0x1p32f));
    if (lane == 0) sh.sums[warp] = total;
    static_assert(kWarps == 4, "two rounds");
    if (warp < 2) best.list = merge32(best.list, sh.scan.lists[warp + 2][lane], lane);
    if (warp == 1) sh.scan.lists[1][lane] = best.list;
    __syncthreads();
    if (warp == 0) {
      const int64_t at = row * g.parts + part;
      best.list = merge32(best.list, sh.scan.lists[1][lane], lane);
      if (lane == 0) g.s.parts[at] = Part{sh.sums[0] + sh.sums[1] + sh.sums[2] + sh.sums[3], ref, any};
      if (lane < B) g.s.keys[at * B + lane] = best.list;
    }
  }
  // the last CTA of a request
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) {
    sh.last = atomicAdd(g.s.done + r, 1) == B * g.parts - 1;
    if (sh.last) g.s.done[r] = 0;
  }
  __syncthreads();
  if (!sh.last) return;
  __threadfence();
  finish<T>(g, r, sh.queue, sh.joined);
}

}  // namespace

int32_t launch_select(const Search& s, const ps_beam_select_t& a, int32_t* status, cudaStream_t st) {
  Args g{a, s, status, 1};
  const int64_t rows = (int64_t)a.num_requests * s.beams;
  const int64_t chunk = kChunk * (s.dtype == PS_BEAM_F32 ? 4 : 8), chunks = (s.vocab + chunk - 1) / chunk;
  int64_t parts = kSpreadCtas / rows;
  const int64_t most = (chunks + kWarps * kLeastChunks - 1) / (kWarps * kLeastChunks);
  parts = parts < most ? parts : most;
  g.parts = (int32_t)(parts < 1 ? 1 : (parts > kMaxParts ? kMaxParts : parts));
  const dim3 grid((unsigned)(rows * g.parts));
  switch (s.dtype) {
    case PS_BEAM_BF16: return status_of(launch(k_select<__nv_bfloat16>, grid, kThreads, 0, st, g));
    case PS_BEAM_F16: return status_of(launch(k_select<__half>, grid, kThreads, 0, st, g));
    default: return status_of(launch(k_select<float>, grid, kThreads, 0, st, g));
  }
}

}  // namespace psbeam
