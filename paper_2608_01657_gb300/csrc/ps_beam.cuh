// Internal declarations of beam search (prefixshield_beam.h).
#pragma once

#include "prefixshield_beam.h"
#include "ps_kv.cuh"

namespace psbeam {

using pskv::chain;
using pskv::launch;
using pskv::set_error;
using pskv::status_of;

// Parts of a row, and warps that a call's rows are divided between, at most, and rows
// of which those that are not there are left out.
constexpr int kRowParts = 32, kWarpsPerSm = 12, kRowWords = 128;
constexpr int64_t kMostWarps = (int64_t)kWarpsPerSm * pskv::kMaxSms;
// Lists of the best runs of a call's rows, one for each warp's share of a row: up to
// kRowParts of a row in a call that leaves rows out, and else two for each warp and row.
constexpr int64_t most_lists(int64_t rows) {
  const int64_t few = (rows < 32 * kRowWords ? rows : 32 * kRowWords) * kRowParts, many = 2 * (kMostWarps + rows);
  return few > many ? few : many;
}

// Of a part of a row: the sum of 2^(x a - R) in whole numbers of 2^-32, the greatest
// logit, which gives R, and whether a logit is NaN or +infinity.
struct __align__(16) Part {
  uint64_t sum;
  float most;
  int32_t bad;
};
struct Search {
  int32_t beams, vocab, dtype, num_end, end[PS_BEAM_MAX_END];  // the end tokens rise
  Part* parts;     // [rows][parts of a row]
  uint64_t* keys;  // [rows][lists of a row][beams] the best runs
  int32_t* lists;  // [rows] lists of a row
};

// Attributes of the kernels, for the current device.
int32_t configure_select();
int32_t configure_trace();
int32_t launch_select(const Search& s, const ps_beam_select_t& a, int32_t* status, int nsm, cudaStream_t st);
int32_t launch_trace(const Search& s, const ps_beam_trace_t& a, int32_t* status, cudaStream_t st);

}  // namespace psbeam
