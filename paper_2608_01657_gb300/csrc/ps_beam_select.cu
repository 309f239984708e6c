// ps_beam_select: the best continuations of a request's beams.
//
// Of a beam with score c and logits x, token v continues it with the score c + x_v
// - lse, lse = log sum_u exp x_u.  Within a beam the order is the logits', and a
// request's best are among its beams' best.  A row is read once, in runs of 128 bytes,
// for two things: a sum of 2^((x - ref) log2 e), whose reference rises with the greatest
// logit seen, and the 'beams' runs of the greatest logits.  The best tokens are in the
// best runs: every run that comes before one of theirs (by its greatest logit, equal
// ones by place) holds a token that comes before it, too, in a row as among a request's
// beams.  So single elements are looked at in a request's best runs only, at the end.
// Runs are kept as whole numbers, the logit's bits in order and then the complement of
// the place, so that no two are equal.
//
// Bound by HBM.  k_select's resident warps divide the list of all rows' chunks of 4 KB
// into equal shares.  Sums are kept for each of up to 32 parts of a row, always the
// same, so that they do not depend on the shares: equal rows have equal sums.  Rows of
// beams that are not there are left out of the list.  k_select_join puts the parts of
// a request together, a CTA each.
//
// A warp reads 4 KB at a time through a ring in shared memory, two of them under way
// while it works on one, a run a lane.  What is greater than the beams-th of its best
// enters a queue, 32 of which are looked through at a time.  A lower bound of that
// beams-th is the beams-th of the lanes' greatest logits, taken after 1, 4, 16, ... chunks.
//
// Neighbours in the order of scores may be nearer than 32 bits tell.  A term is 2^(x a -
// R), a = log2 e rounded to 32 bits and R a whole number next to the greatest x a, so that
// x a - R is rounded once and sums of other R are scaled exactly; sums are added up as
// whole numbers of 2^-32.  They are those of exp((x - R / a) a ln 2): the exponents are off
// by a ln 2 - 1 = 1.3e-8 of their size.  Scores are added in 64 bits.  R is the greatest
// product, rounded to 32 bits and then up: up to kFar, where products are told apart to a
// quarter, it is less than a quarter below that.  Rows whose greatest logit is further
// from 0 are added up again (far_sum).  Other rows' masks may be of any size: lanes and
// parts that have nothing above -2 kFar add nothing.
//
// 128 requests of 8 beams and 131072 tokens in bf16, 268 MB, take 56 us: 50 for k_select,
// which reads 5.3 TB/s at 58 % of the issue slots (45 us with the loads alone, 2 less without
// the queues, no less without the exponentials), and 6 for k_select_join.  So they do in
// f16; 64 x 8 in 32 bits take 55; 131071 tokens, whose rows begin anywhere in a word, 65;
// 64000 tokens 39 (parts of two chunks in place of one: 37, but odd ones longer); 256 single
// rows 22, of which the list of the rows that are there is 1.3; 32 x 32 beams 66.  Few rows
// are a chain of dependent steps: 8 for one row of 1000 tokens, 9.5 for 8 x 4 of 65536.
#include "ps_beam.cuh"

namespace psbeam {
namespace {

constexpr int kWarps = kWarpsPerSm, kThreads = 32 * kWarps;
// A CTA an SM, so that no SM has two while another has none, of twelve warps: with 16
// the last ones ended 10 us behind the others, and a call of 128 requests took 66 us
// instead of 57.  Registers as for 16 leave room for the next kernel's CTAs beside it.
constexpr int kRoom = 512;
// Threads of the joining kernel's CTAs: few fit beside the first kernel's CTA, many are a
// warp a beam.
constexpr int kFewThreads = 256, kManyThreads = 1024;
constexpr int kVecs = 8;                 // 16-byte words of a run
constexpr int kChunk = 32 * kVecs;       // words of a chunk, a run a lane
constexpr int kStages = 3;               // chunks of a warp's ring
constexpr float kLog2e = 1.44269502f;    // 'a'
constexpr double kLn2 = 0.693147180559945309;
constexpr float kFar = 0x1p21f;          // rows' greatest logits up to here are added up on the way
constexpr unsigned kAll = 0xFFFFFFFFu;

struct Args {
  ps_beam_select_t a;
  Search s;
  int32_t* status;
  int64_t rows;
  int32_t chunks;   // of a row
  int32_t size;     // chunks of a part
  int32_t parts;    // of a row
  int32_t slots;    // lists of a row at most
  bool compact;     // rows of beams that are not there are left out
  bool at_once;     // every part has a warp, which fetches before it knows whether the beam is there
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

// Up to this many are taken out one by one, each by two reductions (8 of them take 700
// cycles, a sort of 32 and a merge 1150).
constexpr int kOneByOne = 8;
// The 'keep' greatest of two numbers a lane, none of them equal but zeros, from the
// greatest on, one a lane; what is in the other lanes is less.
__device__ __forceinline__ uint64_t greatest_of(uint64_t a, uint64_t b, int keep, int lane) {
  if (keep > kOneByOne) return merge32(sort32(a, lane), sort32(b, lane), lane);
  uint64_t out = 0;
#pragma unroll 1
  for (int k = 0; k < keep; ++k) {
    const uint64_t m = a > b ? a : b;
    const uint32_t hi = __reduce_max_sync(kAll, (uint32_t)(m >> 32));
    const uint32_t lo = __reduce_max_sync(kAll, (uint32_t)(m >> 32) == hi ? (uint32_t)m : 0);
    const uint64_t top = (uint64_t)hi << 32 | lo;
    if (lane == k) out = top;
    if (a == top) a = 0;
    if (b == top) b = 0;
  }
  return out;
}
// The keep-th of the lanes' numbers, or a little less: the five lowest bits are cleared.
__device__ __forceinline__ uint32_t kth_of(uint32_t x, int keep, int lane) {
  x = (x & ~31u) | lane;  // no two are equal
  uint32_t end = 0;
  if (keep <= 16) {
#pragma unroll 1
    for (int k = 0; k < keep; ++k) {
      end = __reduce_max_sync(kAll, x);
      if (x == end) x = 0;
    }
  } else {  // from the other side
#pragma unroll 1
    for (int k = 32; k >= keep; --k) {
      end = __reduce_min_sync(kAll, x);
      if (x == end) x = ~0u;
    }
  }
  return end & ~31u;
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
    list = keep > kOneByOne ? merge32(list, sort32(q, lane), lane) : greatest_of(list, q, keep, lane);
    raise(__shfl_sync(kAll, list, keep - 1));
  }
  __device__ __forceinline__ void add(uint64_t key, bool on) {
    const unsigned m = __ballot_sync(kAll, on);
    if (on) queue[queued + __popc(m & ((1u << lane) - 1))] = key;
    queued += __popc(m);
    if (queued >= 32) flush();
  }
};

// ---- sums -----------------------------------------------------------------------------
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

// R of a greatest logit; -infinity where the terms are 0 in any row that is not far, whose
// greatest logit is a million above them or more.
__device__ __forceinline__ float exponent_of(float most) { return most < -2 * kFar ? -INFINITY : ceilf(most * kLog2e); }
// A lane's sum of 2^(x a - R).  (Where R is a logit's past kFar it is not looked at.)
struct Sum {
  float R, sum;
  __device__ __forceinline__ void raise(float most) {
    const float to = exponent_of(most);
    sum = R == -INFINITY ? 0.0f : sum * pskv::ex2(R - to);
    R = to;
  }
  // What is subtracted: nothing while R is -infinity, when 2^(x a) is 0.
  __device__ __forceinline__ float base() const { return R == -INFINITY ? 0.0f : R; }
};
__device__ __forceinline__ float warp_max(float x) { return unordered(__reduce_max_sync(kAll, ordered(x))); }
// Of numbers whose sum is below 2^58: a row has 2^24 terms of 2^32.25 at most.
__device__ __forceinline__ uint64_t warp_sum(uint64_t x) {
  const uint32_t lo = __reduce_add_sync(kAll, (uint32_t)x & 0x3FFFFFFu), hi = __reduce_add_sync(kAll, (uint32_t)(x >> 26));
  return ((uint64_t)hi << 26) + lo;
}

// ---- a part of a row ------------------------------------------------------------------
// Words are counted from the row's first element on, wherever that lies in memory, so
// that a row's sum does not depend on its address: equal beams are equal to the last
// bit.  A ring slot holds aligned words.  Where the row starts 'shift' elements into
// one, a word is put together from two; elements of aligned words that are not the
// row's are not read.
constexpr int kSlot = kChunk + 1;  // with the word after the chunk's
// Where word w of a chunk lies in its slot: lanes that read their runs' words, eight words
// apart, and lanes that fill neighbouring ones meet no bank twice.
__device__ __forceinline__ int place_in_slot(int w) { return w ^ (w >> 3 & 7); }

template <typename T>
__device__ __forceinline__ void fetch_word(uint4* to, const T* row, int shift, int w, int V) {
  constexpr int N = Elem<T>::N;
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
// Chunk c of a row into a slot of the ring, asynchronously.
template <typename T>
__device__ __forceinline__ void fetch_chunk(uint4* slot, const T* row, int shift, int c, int V, int lane) {
  constexpr int N = Elem<T>::N;
  if ((c > 0 || shift == 0) && (c + 1) * kChunk * N + (shift == 0 ? 0 : N) <= V) {  // all of it, and a word after it that is needed, is the row's
    const uint32_t to = (uint32_t)__cvta_generic_to_shared(slot);
    const char* from = reinterpret_cast<const char*>(row - shift) + ((int64_t)c * kChunk + lane) * 16;
#pragma unroll
    for (int j = 0; j < kVecs; ++j)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + place_in_slot(32 * j + lane) * 16), "l"(from + 512 * j) : "memory");
    if (shift != 0 && lane == 0)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + 512 * kVecs), "l"(from + 512 * kVecs) : "memory");
    return;
  }
#pragma unroll 1
  for (int j = 0; j < kVecs; ++j) fetch_word(slot + place_in_slot(32 * j + lane), row, shift, c * kChunk + 32 * j + lane, V);
  if (shift != 0 && lane == 0) fetch_word(slot + kChunk, row, shift, c * kChunk + kChunk, V);
}
// A run that begins W 32-bit words and 'bits' further on.
template <int W>
__device__ __forceinline__ void shift_run(uint4 (&v)[kVecs], const uint4& behind, int bits) {
  uint32_t x[4 * kVecs + 4];
#pragma unroll
  for (int j = 0; j <= kVecs; ++j) {
    const uint4 n = j < kVecs ? v[j < kVecs ? j : 0] : behind;
    x[4 * j] = n.x, x[4 * j + 1] = n.y, x[4 * j + 2] = n.z, x[4 * j + 3] = n.w;
  }
#pragma unroll
  for (int i = 0; i < 4 * kVecs; ++i) x[i] = __funnelshift_r(x[i + W], x[i + W + 1], bits);
#pragma unroll
  for (int j = 0; j < kVecs; ++j) v[j] = make_uint4(x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]);
}
// A lane's run of a chunk.
template <typename T>
__device__ __forceinline__ void take_run(const uint4* slot, int shift, int lane, uint4 (&v)[kVecs]) {
#pragma unroll
  for (int j = 0; j < kVecs; ++j) v[j] = slot[place_in_slot(kVecs * lane + j)];
  if (shift == 0) return;
  const int words = shift * (int)sizeof(T) / 4, bits = shift * (int)sizeof(T) % 4 * 8;
  const uint4 behind = slot[lane == 31 ? kChunk : place_in_slot(kVecs * lane + kVecs)];
  switch (words) {  // the same for all lanes
    case 0: shift_run<0>(v, behind, bits); break;
    case 1: shift_run<1>(v, behind, bits); break;
    case 2: shift_run<2>(v, behind, bits); break;
    default: shift_run<3>(v, behind, bits); break;
  }
}

// One chunk of a row.
template <typename T>
struct Scan {
  static constexpr int N = Elem<T>::N;
  Best best;
  Sum sum;
  float most;
  int end_chunk;   // no end token is in a chunk before this one
  float top;       // the lane's greatest logit of a token that ends nothing
  int seen, again; // chunks looked at, and when the lanes' greatest are looked at next
  __device__ __forceinline__ void begin_part() {
    sum = Sum{-INFINITY, 0.0f};
    most = -INFINITY;
  }
  __device__ __forceinline__ void begin_row(const Args& g) {
    best.list = 0;
    best.floor = kNoKey;
    best.queued = 0;
    top = -INFINITY;
    seen = 0;
    again = 1;
    end_chunk = g.s.num_end > 0 ? 0 : 1 << 30;
  }
  __device__ __forceinline__ void chunk(const Args& g, uint4 (&v)[kVecs], int c) {
    const int lane = best.lane;
    float all = Elem<T>::top(greatest<T>(v));
    if (all > most) sum.raise(all);
    most = max_nan(most, all);
    const float base = sum.base();
    const uint64_t minus = pskv::pack2(-base, -base), a = pskv::pack2(kLog2e, kLog2e);
    uint64_t s0 = 0, s1 = 0;
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
      float x[N];
      Elem<T>::wide(v[j], x);
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        const float2 t = pskv::unpack2(pskv::fma2(pskv::pack2(x[e], x[e + 1]), a, minus));
        const uint64_t p = pskv::pack2(pskv::ex2(t.x), pskv::ex2(t.y));
        if (e & 2) s1 = pskv::add2(s1, p);
        else s0 = pskv::add2(s0, p);
      }
    }
    const float2 f = pskv::unpack2(pskv::add2(s0, s1));
    sum.sum += f.x + f.y;
    if (c >= end_chunk) {  // an end token is among these, or one lies behind: end tokens do not count
      const int w0 = c * kChunk + kVecs * lane;
      uint64_t out = 0;
      end_chunk = 1 << 30;
      for (int i = 0; i < g.s.num_end; ++i) {
        const int word = g.s.end[i] / N, w = word - w0;
        if (w >= 0 && w < kVecs) out |= 1ull << (w * N + g.s.end[i] % N);
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
    top = fmaxf(top, all);
    if (++seen == again) {  // so many runs are no smaller
      again *= 4;
      best.raise(((uint64_t)kth_of(ordered(top), best.keep, lane) << 32) - 1);
    }
    const uint64_t key = key_of(all, c * 32 + lane);
    const bool on = key > best.floor;
    if (__any_sync(kAll, on)) best.add(key, on);
  }
};

// The rows that are looked at: all, or those whose scores are finite.
struct Live {
  uint32_t bits[kRowWords];
  int before[kRowWords + 1];  // live rows before a word's
  // Row of the live row number a, the same in all lanes.
  __device__ __forceinline__ int row(int a, int lane) const {
    int lo = 0, hi = kRowWords - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (before[mid] <= a) lo = mid;
      else hi = mid - 1;
    }
    const uint32_t m = bits[lo];
    return lo * 32 + __ffs(__ballot_sync(kAll, (m >> lane & 1) && __popc(m & ((1u << lane) - 1)) == a - before[lo])) - 1;
  }
};

// A row of the list: which one it is, where it begins, and its score, which says whether
// it is looked at.
template <typename T>
struct Open {
  const T* row;
  int i, shift;
  float score;  // looked at when it is needed: it may be on its way still
  __device__ __forceinline__ bool live() const { return score - score == 0; }
  __device__ __forceinline__ void open(const Args& g, const Live& live_rows, int number, int lane) {
    i = g.compact ? live_rows.row(number, lane) : number;
    const int r = i / g.s.beams;
    score = g.compact ? 0.0f : g.a.scores[i];
    row = static_cast<const T*>(g.a.logits) + r * g.a.request_stride + (i - r * g.s.beams) * g.a.beam_stride;
    shift = (int)(reinterpret_cast<uintptr_t>(row) & 15) / (int)sizeof(T);
  }
};

struct Shared {
  uint4 ring[kWarps][kStages * kSlot];
  uint64_t queue[kWarps][kQueue];
  Live live;
};

template <typename T>
__global__ void __launch_bounds__(kRoom, 1) k_select(const __grid_constant__ Args g) {
  extern __shared__ __align__(16) unsigned char smem[];
  Shared& sh = *reinterpret_cast<Shared*>(smem);
  chain();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, B = g.s.beams;
  int count = (int)g.rows;
  if (g.compact) {
    constexpr int kAtOnce = 8;
    const int words = (count + 31) / 32;
    for (int i0 = warp; i0 < kRowWords; i0 += kWarps * kAtOnce) {
      float c[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const int row = (i0 + u * kWarps) * 32 + lane;
        c[u] = row < g.rows ? g.a.scores[row] : -INFINITY;
      }
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const unsigned m = __ballot_sync(kAll, c[u] - c[u] == 0);
        if (lane == 0 && i0 + u * kWarps < kRowWords) sh.live.bits[i0 + u * kWarps] = m;
      }
      if (i0 + kWarps * kAtOnce - warp >= words) {  // no rows behind these
        for (int i = i0 + kWarps * kAtOnce + lane * kWarps; i < kRowWords; i += 32 * kWarps) sh.live.bits[i] = 0;
        break;
      }
    }
    __syncthreads();
    if (warp == 0) {  // four words a lane
      int n[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        n[i] = sum;
        sum += __popc(sh.live.bits[4 * lane + i]);
      }
      int incl = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(kAll, incl, o);
        if (lane >= o) incl += x;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) sh.live.before[4 * lane + i] = incl - sum + n[i];
      if (lane == 31) sh.live.before[kRowWords] = incl;
    }
    __syncthreads();
    count = sh.live.before[kRowWords];
    if (count == 0) return;
  }
  // the warp's share of the list of all parts
  const int all = gridDim.x * kWarps, w = warp * gridDim.x + blockIdx.x;  // (few shares lie on different SMs)
  const int64_t U = (int64_t)count * g.parts;
  const int C = U < all ? (int)U : all;
  if (w >= C) return;
  int64_t u0, u1;
  int slot;  // of the share's first row: workers before this one that have a share of it
  if (U <= 1 << 19) {  // w < 2^12, so that products are below 2^31
    const int n = (int)U;
    u0 = n * w / C, u1 = n * (w + 1) / C;
    slot = w - ((int)u0 / g.parts * g.parts * C + C - 1) / n;
  } else {
    u0 = U * w / C, u1 = U * (w + 1) / C;
    slot = w - pskv::worker_of(u0 / g.parts * g.parts, U, C);
  }
  int number = (int)(u0 / g.parts), chunk = (int)(u0 - (int64_t)number * g.parts) * g.size;
  const int last_number = (int)((u1 - 1) / g.parts);
  const int last_end = min((int)(u1 - (int64_t)last_number * g.parts) * g.size, g.chunks);  // chunk after the last
  uint4* const ring = sh.ring[warp];
  // the chunk to fetch next, and the one at work
  int ahead = number, ahead_chunk = chunk;
  Open<T> from;
  from.open(g, sh.live, ahead, lane);
  Open<T> at = from;
  auto fetch = [&](int stage) {
    if (ahead < last_number || (ahead == last_number && ahead_chunk < last_end)) {
      if (g.at_once || from.live()) fetch_chunk(ring + stage * kSlot, from.row, from.shift, ahead_chunk, g.s.vocab, lane);
      if (++ahead_chunk == g.chunks) {
        ahead_chunk = 0;
        if (++ahead <= last_number) from.open(g, sh.live, ahead, lane);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll 1
  for (int i = 0; i < kStages - 1; ++i) fetch(i);
  Scan<T> scan;
  scan.best.queue = sh.queue[warp];
  scan.best.keep = B;
  scan.best.lane = lane;
  scan.begin_row(g);
  scan.begin_part();
  int stage = 0, stop = min(chunk + g.size, g.chunks);
  while (true) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
    __syncwarp();  // the lanes' copies are there, and all have read the slot that is filled next
    uint4 v[kVecs];
    take_run<T>(ring + stage * kSlot, at.shift, lane, v);
    fetch(stage == 0 ? kStages - 1 : stage - 1);
    stage = stage == kStages - 1 ? 0 : stage + 1;
    if (at.live()) scan.chunk(g, v, chunk);
    if (++chunk < stop) continue;
    // the end of a part
    if (at.live()) {
      const float most = warp_max(scan.most);
      const bool bad = __any_sync(kAll, !(scan.most < INFINITY));
      const float scaled = scan.sum.R == -INFINITY ? 0.0f : scan.sum.sum * pskv::ex2(scan.sum.R - exponent_of(most));
      const uint64_t sum = warp_sum(__float2ull_rn(scaled * 0x1p32f));
      if (lane == 0) g.s.parts[(int64_t)at.i * g.parts + (chunk - 1) / g.size] = Part{sum, most, bad};
      scan.begin_part();
    }
    stop = min(chunk + g.size, g.chunks);
    if (chunk < g.chunks && !(number == last_number && chunk == last_end)) continue;
    // the end of the warp's share of the row
    if (at.live()) {
      while (scan.best.queued > 0) scan.best.flush();
      if (lane < B) g.s.keys[((int64_t)at.i * g.slots + slot) * B + lane] = scan.best.list;
      if (lane == 0 && chunk == g.chunks) g.s.lists[at.i] = slot + 1;
    }
    if (number == last_number) break;
    ++number;
    chunk = slot = 0;
    stop = min(g.size, g.chunks);
    at.open(g, sh.live, number, lane);
    scan.begin_row(g);
  }
}

// ---- the parts of a request -------------------------------------------------------------
// A candidate of a request: its score as a whole number in the scores' order, and what
// decides between equal ones.
struct Cand {
  long long score, tie;
  __device__ __forceinline__ bool before(const Cand& y) const { return score != y.score ? score > y.score : tie < y.tie; }
  __device__ __forceinline__ Cand shfl(int from) const { return {__shfl_sync(kAll, score, from), __shfl_sync(kAll, tie, from)}; }
  __device__ __forceinline__ double exact() const { return __longlong_as_double(score < 0 ? score ^ 0x7FFFFFFFFFFFFFFFll : score); }
  __device__ __forceinline__ float value() const { return (float)exact(); }
  __device__ __forceinline__ bool somebody() const { return tie < 1ll << 60; }
};
__device__ __forceinline__ Cand cand(double score, long long tie) {
  const long long b = __double_as_longlong(score + 0.0);
  return {b < 0 ? b ^ 0x7FFFFFFFFFFFFFFFll : b, tie};
}
__device__ __forceinline__ Cand nobody(int lane) { return {(long long)0x8000000000000000ull, (1ll << 60) + lane}; }
__device__ __forceinline__ Cand merge32(Cand x, const Cand& y, int lane) {
  const Cand z = y.shfl(31 - lane);
  if (z.before(x)) x = z;
#pragma unroll
  for (int j = 16; j > 0; j >>= 1) {
    const Cand o = x.shfl(lane ^ j);
    if (x.before(o) != ((lane & j) == 0)) x = o;
  }
  return x;
}

// A beam's score, the reference R / a, and the log of the sum over it.
struct Beam {
  double total, ref;
  float score;
  // The reference, which may be far from 0, is subtracted first.
  __device__ __forceinline__ double of(float logit) const { return (double)score + (((double)logit - ref) - total); }
};
// The sum of exp(x - most) of a row whose greatest logit is past kFar.  Slow, and rare:
// such rows have masks of a finite value and nothing else, or are mistakes.  A lane adds
// 2^19 terms of up to 1 at most, as whole numbers of 2^-44, so that many small ones count.
// A row of 131072 such logits takes 260 us longer, one of 5000 10.
template <typename T>
__device__ __noinline__ uint64_t far_sum(const T* row, int V, float most, int lane) {
  uint64_t sum = 0;
#pragma unroll 8
  for (int i = lane; i < V; i += 32) {
    const float d = Elem<T>::one(row + i) - most;
    sum += __float2ull_rn((d < -100.0f ? 0.0f : pskv::ex2(d * kLog2e)) * 0x1p44f);
  }
  return warp_sum((sum + (1 << 11)) >> 12);
}

// The 'keep' greatest of n numbers in any order, of which the first 64 are in a and b.
__device__ __forceinline__ uint64_t best_runs(const uint64_t* keys, uint64_t a, uint64_t b, int n, int keep, int lane) {
  uint64_t list = 0;
  for (int i = lane; i - lane < n; i += 64) {
    const uint64_t c = i + 64 < n ? keys[i + 64] : 0, d = i + 96 < n ? keys[i + 96] : 0;
    a = greatest_of(i < n ? a : 0, i + 32 < n ? b : 0, keep, lane);
    list = i == lane ? a : greatest_of(list, a, keep, lane);
    a = c, b = d;
  }
  return list;
}
// Of sorted lists of 'keep', of which the first ones (up to 'slots' may be read) are in k.
constexpr int kLists = 8;
__device__ __forceinline__ void read_lists(uint64_t (&k)[kLists], const uint64_t* keys, int from, int to, int keep, int lane) {
#pragma unroll
  for (int u = 0; u < kLists; ++u) k[u] = lane < keep && from + u < to ? keys[(from + u) * keep + lane] : 0;
}
__device__ __forceinline__ uint64_t best_lists(const uint64_t* keys, uint64_t (&k)[kLists], int lists, int keep, int lane) {
  uint64_t x = 0, y = 0;  // two chains of merges side by side
  for (int l = 0; l < lists; l += kLists) {
    if (l > 0) read_lists(k, keys, l, lists, keep, lane);
#pragma unroll
    for (int u = 0; u < kLists; u += 2) {
      if (l + u >= lists) break;
      x = merge32(x, k[u], lane);
      y = merge32(y, l + u + 1 < lists ? k[u + 1] : 0, lane);
    }
  }
  return merge32(x, y, lane);
}

// A beam's sum of 2^(x a - R), or of exp(x - most) where that is 'far', and what else is
// known of its row.
struct RowSum {
  uint64_t sum;
  float most, score;
  bool good, far;
};

// A CTA a request, of J threads, a warp a beam.  The warps put the beams' parts and lists
// together, then the best runs of all beams are found, and the tokens in those: up to
// kOneByOne beams' by counting what comes before each, more by merges of the beams' sorted
// lists, two by two.  64-bit additions are slow (an SM does two at a time): of more beams
// one warp makes the logarithms, and only those tokens are scored whose logits pass a
// bound in 32 bits.
template <typename T, int J>
__global__ void __launch_bounds__(J, J == kFewThreads ? 4 : 1) k_select_join(const __grid_constant__ Args g) {
  constexpr int N = Elem<T>::N, kTokens = kVecs * N;  // of a run
  constexpr bool kFew = J == kFewThreads;
  constexpr int kMost = kFew ? kOneByOne : PS_BEAM_MAX_BEAMS, kEnds = kMost * PS_BEAM_MAX_END;
  constexpr int kTurns = (kMost * kTokens + J - 1) / J;  // tokens of a thread
  static_assert(32 * kMost <= J && kEnds <= J && kMost <= kTokens, "a warp a beam, an end token a thread, the runs' room");
  __shared__ RowSum s_row[kMost];
  __shared__ Beam s_beam[kMost];
  __shared__ float s_least[kMost];
  __shared__ Cand s_best[kMost], s_token[kMost * kTokens], s_chosen[kMost], s_end[kEnds];
  __shared__ int s_tokens, s_ended;
  Cand* const s_run = s_token;  // the tokens come after the runs
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5, B = g.s.beams, r = blockIdx.x;
  const int E = g.a.ended_tokens ? g.s.num_end : 0;
  const T* logits = static_cast<const T*>(g.a.logits) + r * g.a.request_stride;
  const int64_t to = (int64_t)r * B;
  const int end_beam = E > 0 ? t / E : kMost, end_token = E > 0 ? g.s.end[t % E] : 0;
  if (t == 0) s_tokens = s_ended = 0;
  if (t < kMost) s_best[t] = s_chosen[t] = nobody(t);
  if (kFew && t < kMost * kMost) s_run[t] = nobody(t);
  if (kFew) __syncthreads();
  chain();
  // the end tokens' logits, on their way early
  float end_logit = -INFINITY;
  if (end_beam < B) end_logit = Elem<T>::one(logits + end_beam * g.a.beam_stride + end_token);
  uint64_t list = 0;
  auto beam_of = [](const RowSum& x) {
    Beam beam{INFINITY, 0.0, x.score};  // no candidates
    if (x.good) {
      beam.ref = x.far ? (double)x.most : (double)exponent_of(x.most) * (1.0 / (double)kLog2e);
      beam.total = log_of(x.sum);
    }
    return beam;
  };
  if (warp < B) {
    const int row = r * B + warp;
    // all that may be needed is read at once, and looked at where it is some row's of this call
    const float c = g.a.scores[row];
    const uint64_t* keys = g.s.keys + (int64_t)row * g.slots * B;
    Part p{0, -INFINITY, 0};
    if (lane < g.parts) p = g.s.parts[(int64_t)row * g.parts + lane];
    const int lists = g.s.lists[row];
    uint64_t k0 = 0, k1 = 0, k[kLists];
    if (kFew) {
      k0 = lane < g.slots * B ? keys[lane] : 0;
      k1 = lane + 32 < g.slots * B ? keys[lane + 32] : 0;
    } else {
      read_lists(k, keys, 0, g.slots, B, lane);
    }
    RowSum x{0, -INFINITY, c, false, false};
    bool bad = c != -INFINITY && !(c - c == 0);
    if (c - c == 0) {
      list = kFew ? best_runs(keys, k0, k1, lists * B, B, lane) : best_lists(keys, k, lists, B, lane);
      x.most = warp_max(p.most);
      const float R = exponent_of(x.most), down = R - exponent_of(p.most);
      x.sum = warp_sum(down < 64.0f ? p.sum >> (int)down : 0);
      bad = __any_sync(kAll, p.bad);
      x.good = !bad && x.most > -INFINITY;
      x.far = fabsf(x.most) > kFar && x.good;
      if (x.far) x.sum = far_sum(logits + warp * g.a.beam_stride, g.s.vocab, x.most, lane);
    }
    if (lane == 0 && bad) set_error(g.status, PS_ERR_INVALID_ARG);
    if (kFew) {  // eight warps' additions take no longer than another step
      const Beam beam = beam_of(x);
      if (lane == 0) s_beam[warp] = beam;
      if (lane < B && beam.total < INFINITY && list > kNoKey)
        s_run[warp * B + lane] = cand(beam.of(logit_of(list)), (long long)warp << 32 | (uint32_t)place_of(list));
    } else if (lane == 0) {
      s_row[warp] = x;
    }
  }
  __syncthreads();
  if (!kFew) {
    if (t < B) s_beam[t] = beam_of(s_row[t]);
    __syncthreads();
  }
  auto candidate = [&](int beam, bool on, float logit, uint32_t place) {
    return on && s_beam[beam].total < INFINITY ? cand(s_beam[beam].of(logit), (long long)beam << 32 | place) : nobody(t);
  };
  if (end_beam < B) s_end[t] = candidate(end_beam, end_logit > -INFINITY, end_logit, end_token);
  // x's place among n candidates, 'each' threads in a row counting a share each: in turns,
  // so that a warp reads neighbours (64 in a row each took 15 us for 256)
  auto place_among = [&](const Cand& x, const Cand* of, int n, int each) {
    int place = 0;
#pragma unroll 4
    for (int j = t % each; j < n; j += each) place += of[j].before(x);
    for (int o = 1; o < each; o <<= 1) place += __shfl_xor_sync(kAll, place, o);
    return place;
  };
  auto threads_for = [&](int n) {
    int each = 1;
    while (2 * each * n <= J && each < 16) each *= 2;
    return each;
  };
  // the best runs
  if (kFew) {
    const int each = threads_for(B * B), i = t / each;
    const Cand x = i < B * B ? s_run[i] : nobody(J);
    const int place = place_among(x, s_run, B * B, each);
    if (t % each == 0 && x.somebody() && place < B) s_best[place] = x;
  } else {
    Cand x = nobody(t);
    if (warp < B) x = candidate(warp, lane < B && list > kNoKey, logit_of(list), place_of(list));
    for (int s = 1; s < B; s <<= 1) {
      if ((warp & (2 * s - 1)) == s && warp < B) s_run[t] = x;
      __syncthreads();
      if ((warp & (2 * s - 1)) == 0 && warp + s < B) x = merge32(x, s_run[t + 32 * s], lane);
    }
    if (warp == 0 && lane < B) s_best[lane] = x;
  }
  __syncthreads();
  // the tokens of the best runs; each run has one that is no later than the last run's best
  const Cand last = s_best[B - 1];
  float logit[kTurns];
#pragma unroll
  for (int u = 0; u < kTurns; ++u) {
    const int i = t + u * J;
    logit[u] = -INFINITY;
    if (i < B * kTokens && s_best[i / kTokens].somebody()) {
      const long long run = s_best[i / kTokens].tie;
      const int64_t token = (run & 0xFFFFFFFF) * kTokens + i % kTokens;
      if (token < g.s.vocab) logit[u] = Elem<T>::one(logits + (run >> 32) * g.a.beam_stride + token);
    }
  }
  if (!kFew && t < B) {  // a logit that its beam's tokens need, or a little less
    const Beam x = s_beam[t];
    float least = -INFINITY;
    if (last.somebody() && x.total < INFINITY) {
      const double want = (last.exact() - (double)x.score) + x.total;
      least = __double2float_rd(want + x.ref - 1e-9 * (fabs(want) + fabs((double)x.score) + fabs(x.total) + fabs(x.ref)));
    }
    s_least[t] = least;
  }
  if (!kFew) __syncthreads();
#pragma unroll
  for (int u = 0; u < kTurns; ++u) {
    if (logit[u] == -INFINITY) continue;
    const int i = t + u * J;
    const long long run = s_best[i / kTokens].tie;
    const int beam = (int)(run >> 32), token = (int)(run & 0xFFFFFFFF) * kTokens + i % kTokens;
    if ((!kFew && logit[u] < s_least[beam]) || ends(g.s, token)) continue;
    const Cand y = candidate(beam, true, logit[u], token);
    if (!last.somebody() || y.score >= last.score) s_token[atomicAdd(&s_tokens, 1)] = y;
  }
  __syncthreads();
  const int n = s_tokens, each = threads_for(n);
  for (int i0 = 0; i0 < n; i0 += J / each) {
    const int i = i0 + t / each;
    const Cand x = i < n ? s_token[i] : nobody(J);
    const int place = place_among(x, s_token, n, each);
    if (t % each == 0 && x.somebody() && place < B) s_chosen[place] = x;
  }
  // an end token's place among all candidates, and among those of its kind; after the last
  // run's best it has none
  if (end_beam < B) {
    const Cand x = s_end[t];
    if (x.somebody() && (!last.somebody() || x.score >= last.score)) {
      int place = 0, others = 0;
#pragma unroll 4
      for (int j = 0; j < B * E; ++j) place += s_end[j].before(x);
#pragma unroll 4
      for (int j = 0; j < n; ++j) others += s_token[j].before(x);
      if (place + others < B) {
        atomicAdd(&s_ended, 1);
        g.a.ended_tokens[to + place] = (int)(x.tie & 0xFFFFFFFF);
        g.a.ended_parents[to + place] = (int)(x.tie >> 32);
        g.a.ended_scores[to + place] = x.value();
      }
    }
  }
  __syncthreads();
  if (t < B) {
    const Cand x = s_chosen[t];
    const bool on = x.somebody();
    g.a.tokens[to + t] = on ? (int)(x.tie & 0xFFFFFFFF) : -1;
    g.a.parents[to + t] = on ? (int)(x.tie >> 32) : -1;
    g.a.scores_out[to + t] = on ? x.value() : -INFINITY;
  }
  if (g.a.ended_tokens && t < B && t >= s_ended) {
    g.a.ended_tokens[to + t] = g.a.ended_parents[to + t] = -1;
    g.a.ended_scores[to + t] = -INFINITY;
  }
}

}  // namespace

template <typename T>
static int32_t launch_typed(const Args& g, int grid, cudaStream_t st) {
  cudaError_t e = launch(k_select<T>, dim3((unsigned)grid), kThreads, sizeof(Shared), st, g);
  if (e != cudaSuccess) return status_of(e);
  const dim3 requests((unsigned)g.a.num_requests);
  if (g.s.beams <= kOneByOne) return status_of(launch(k_select_join<T, kFewThreads>, requests, kFewThreads, 0, st, g));
  return status_of(launch(k_select_join<T, kManyThreads>, requests, kManyThreads, 0, st, g));
}

// Both kernels prefer all of an SM's memory as shared memory: where two that run after
// one another prefer different divisions, an SM has to run empty in between, and the
// CTAs that find no room meanwhile begin when others end.
template <typename T>
static cudaError_t configure_typed() {
  cudaError_t e = cudaFuncSetAttribute(k_select<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Shared));
  if (e == cudaSuccess) e = cudaFuncSetAttribute(k_select<T>, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(k_select_join<T, kFewThreads>, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(k_select_join<T, kManyThreads>, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
  return e;
}
int32_t configure_select() {
  cudaError_t e = configure_typed<__nv_bfloat16>();
  if (e == cudaSuccess) e = configure_typed<__half>();
  if (e == cudaSuccess) e = configure_typed<float>();
  return status_of(e);
}

int32_t launch_select(const Search& s, const ps_beam_select_t& a, int32_t* status, int nsm, cudaStream_t st) {
  Args g{};
  g.a = a;
  g.s = s;
  g.status = status;
  g.rows = (int64_t)a.num_requests * s.beams;
  const int64_t chunk = kChunk * (s.dtype == PS_BEAM_F32 ? 4 : 8);
  g.chunks = (int32_t)((s.vocab + chunk - 1) / chunk);
  g.size = (g.chunks + kRowParts - 1) / kRowParts;
  g.parts = (g.chunks + g.size - 1) / g.size;
  const int64_t U = g.rows * g.parts, grid = U < nsm ? U : nsm, C = U < grid * kWarps ? U : grid * kWarps;
  g.at_once = U == C;
  // where every part has a warp there is nothing to gain
  g.compact = U > C && g.rows <= 32 * kRowWords;
  const int64_t slots = g.compact ? g.parts : g.parts / (U / C) + 2;
  g.slots = (int32_t)(slots < g.parts ? slots : g.parts);
  switch (s.dtype) {
    case PS_BEAM_BF16: return launch_typed<__nv_bfloat16>(g, (int)grid, st);
    case PS_BEAM_F16: return launch_typed<__half>(g, (int)grid, st);
    default: return launch_typed<float>(g, (int)grid, st);
  }
}

}  // namespace psbeam
