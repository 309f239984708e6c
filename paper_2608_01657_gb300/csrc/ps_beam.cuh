// Internal declarations of beam search (prefixshield_beam.h).
#pragma once

#include "prefixshield_beam.h"
#include "ps_kv.cuh"

namespace psbeam {

using pskv::chain;
using pskv::launch;
using pskv::set_error;
using pskv::status_of;

// CTAs that a call's rows are spread over where they are fewer, and parts of a row at most.
constexpr int kSpreadCtas = 152 * 16;
constexpr int kMaxParts = 32;

// What one CTA found of a row: the logits' greatest, the sum of exp(x - ref) in whole
// numbers of 2^-32, and whether a logit is NaN or +infinity.
struct __align__(16) Part {
  uint64_t sum;
  float ref;
  int32_t bad;
};

struct Search {
  int32_t beams, vocab, dtype, num_end, end[PS_BEAM_MAX_END];  // the end tokens rise
  Part* parts;      // [rows * parts of a row]
  uint64_t* keys;   // [rows * parts of a row][beams]
  int32_t* done;    // [max_requests] CTAs of a request that have finished (back to 0 after each call)
};

int32_t launch_select(const Search& s, const ps_beam_select_t& a, int32_t* status, cudaStream_t st);
int32_t launch_trace(const Search& s, const ps_beam_trace_t& a, int32_t* status, cudaStream_t st);

}  // namespace psbeam
