// C ABI of beam search (declared in include/prefixshield_beam.h).
//
// Host side only: argument checks, the workspace layout and the handle.
#include <algorithm>
#include <new>

#include "ps_beam.cuh"
#include "ps_kv_overlap.cuh"

using namespace psbeam;
using pskv::Span;
using pskv::on_device;
using pskv::outputs_apart;

struct ps_beam {
  Search s;
  int32_t max_requests, dev, nsm;
};

namespace {

inline cudaStream_t as_stream(void* s) { return static_cast<cudaStream_t>(s); }
inline int64_t element_bytes(int32_t dtype) { return dtype == PS_BEAM_F32 ? 4 : 2; }

bool check_config(const ps_beam_config_t* c) {
  if (!c || c->max_requests < 1 || c->beams < 1 || c->beams > PS_BEAM_MAX_BEAMS) return false;
  if ((int64_t)c->max_requests * c->beams > (1 << 20)) return false;
  if (c->vocab < 1 || c->vocab > PS_BEAM_MAX_VOCAB) return false;
  if (c->dtype != PS_BEAM_BF16 && c->dtype != PS_BEAM_F16 && c->dtype != PS_BEAM_F32) return false;
  if (c->num_end < 0 || c->num_end > PS_BEAM_MAX_END) return false;
  for (int i = 0; i < c->num_end; ++i) {
    if (c->end_tokens[i] < 0 || c->end_tokens[i] >= c->vocab) return false;
    for (int j = 0; j < i; ++j)
      if (c->end_tokens[i] == c->end_tokens[j]) return false;
  }
  return true;
}

size_t carve(const ps_beam_config_t& c, char* base, Search* s) {
  size_t off = 0;
  auto take = [&](size_t bytes) {
    off = (off + 255) / 256 * 256;
    char* p = base ? base + off : nullptr;
    off += bytes;
    return p;
  };
  const size_t rows = (size_t)c.max_requests * c.beams;
  char* part = take(sizeof(Part) * rows * kRowParts);
  char* keys = take(8 * (size_t)most_lists((int64_t)rows) * c.beams);
  char* lists = take(4 * rows);
  if (s) {
    s->parts = reinterpret_cast<Part*>(part);
    s->keys = reinterpret_cast<uint64_t*>(keys);
    s->lists = reinterpret_cast<int32_t*>(lists);
  }
  return (off + 255) / 256 * 256;
}

}  // namespace

extern "C" {

size_t ps_beam_workspace_bytes(const ps_beam_config_t* cfg) { return check_config(cfg) ? carve(*cfg, nullptr, nullptr) : 0; }

int32_t ps_beam_create(ps_beam_t** out, const ps_beam_config_t* cfg, void* d_workspace, size_t workspace_bytes) {
  if (!out || !check_config(cfg) || !d_workspace || (reinterpret_cast<uintptr_t>(d_workspace) & 255) != 0 ||
      workspace_bytes < carve(*cfg, nullptr, nullptr))
    return PS_ERR_INVALID_ARG;
  int dev = 0, nsm = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&nsm, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return PS_ERR_CUDA;
  int32_t rc = configure_select();
  if (rc == PS_OK) rc = configure_trace();
  if (rc != PS_OK) return rc;
  ps_beam* b = new (std::nothrow) ps_beam{};
  if (!b) return PS_ERR_CUDA;
  b->max_requests = cfg->max_requests;
  b->dev = dev;
  b->nsm = nsm < pskv::kMaxSms ? nsm : pskv::kMaxSms;
  b->s.beams = cfg->beams;
  b->s.vocab = cfg->vocab;
  b->s.dtype = cfg->dtype;
  b->s.num_end = cfg->num_end;
  for (int i = 0; i < cfg->num_end; ++i) b->s.end[i] = cfg->end_tokens[i];
  std::sort(b->s.end, b->s.end + cfg->num_end);
  carve(*cfg, static_cast<char*>(d_workspace), &b->s);
  *out = b;
  return PS_OK;
}

void ps_beam_destroy(ps_beam_t* beam) { delete beam; }

int32_t ps_beam_select(ps_beam_t* beam, void* stream, const ps_beam_select_t* a, int32_t* d_status) {
  if (!beam || !a || a->num_requests < 0 || a->num_requests > beam->max_requests) return PS_ERR_INVALID_ARG;
  const int64_t R = a->num_requests, B = beam->s.beams, V = beam->s.vocab, e = element_bytes(beam->s.dtype);
  if (R == 0) return PS_OK;
  if (!a->logits || !a->scores || !a->tokens || !a->parents || !a->scores_out || a->request_stride < 0 || a->beam_stride < 0 ||
      a->request_stride > (1ll << 40) || a->beam_stride > (1ll << 40) || reinterpret_cast<uintptr_t>(a->logits) % e != 0)
    return PS_ERR_INVALID_ARG;
  if ((a->ended_tokens != nullptr) != (a->ended_parents != nullptr) || (a->ended_tokens != nullptr) != (a->ended_scores != nullptr))
    return PS_ERR_INVALID_ARG;
  const int64_t n = 4 * R * B;
  const Span spans[] = {{a->logits, e * ((R - 1) * a->request_stride + (B - 1) * a->beam_stride + V), false},
                        {a->scores == a->scores_out ? nullptr : a->scores, n, false}, {d_status, 4, false},
                        {a->tokens, n, true}, {a->parents, n, true}, {a->scores_out, n, true},
                        {a->ended_tokens, n, true}, {a->ended_parents, n, true}, {a->ended_scores, n, true}};
  if (!outputs_apart(spans) || !on_device(beam->dev)) return PS_ERR_INVALID_ARG;
  return launch_select(beam->s, *a, d_status, beam->nsm, as_stream(stream));
}

int32_t ps_beam_trace(ps_beam_t* beam, void* stream, const ps_beam_trace_t* a, int32_t* d_status) {
  if (!beam || !a || a->num_requests < 0 || a->num_requests > beam->max_requests || a->num_steps < 0 ||
      a->num_steps > (1 << 24) || a->hyps < 0 || a->hyps > (1 << 16))
    return PS_ERR_INVALID_ARG;
  const int64_t R = a->num_requests, B = beam->s.beams, T = a->num_steps, N = a->hyps;
  if (R == 0 || T == 0 || N == 0) return PS_OK;
  if (!a->tokens || !a->parents || !a->beams_of || !a->out) return PS_ERR_INVALID_ARG;
  const Span spans[] = {{a->tokens, 4 * T * R * B, false}, {a->parents, 4 * T * R * B, false}, {a->beams_of, 4 * R * N, false},
                        {a->lengths, 4 * R * N, false}, {d_status, 4, false}, {a->out, 4 * R * N * T, true}};
  if (!outputs_apart(spans) || !on_device(beam->dev)) return PS_ERR_INVALID_ARG;
  return launch_trace(beam->s, *a, d_status, as_stream(stream));
}

}  // extern "C"
