/*
 * prefixshield_beam.h -- C ABI of beam search over the requests whose keys and
 * values lie in KV pages (prefixshield_kv.h):
 *   ps_beam_select   the best continuations of each request's beams over beams
 *                    and vocabulary, from the step's logits;
 *   ps_beam_trace    sequences of tokens, back through every step's parents.
 * Between the two, ps_kv_reorder() makes the beams' pages follow their parents.
 * With one beam the selection is the likeliest token and its log-probability.
 *
 * Conventions are prefixshield_kv.h's: d_* pointers and those inside structures
 * are device pointers, every buffer is the caller's, calls are enqueued on a
 * stream and return a status, what only the device can see wrong is reported in
 * *d_status (NULL: not reported).  A handle is not thread-safe; its calls must be
 * issued in order on one stream (or with equivalent ordering), with the device
 * current that it was made on (refused otherwise).
 */
#ifndef PREFIXSHIELD_BEAM_H
#define PREFIXSHIELD_BEAM_H

#include "prefixshield.h"

#ifdef __cplusplus
extern "C" {
#endif

#define PS_BEAM_MAX_BEAMS 32
#define PS_BEAM_MAX_END 8
#define PS_BEAM_MAX_VOCAB (1 << 24)

/* Element types of the logits. */
typedef enum { PS_BEAM_BF16 = 0, PS_BEAM_F16 = 1, PS_BEAM_F32 = 2 } ps_beam_dtype_t;

typedef struct {
  int32_t max_requests;                 /* of one call; max_requests * beams is at most 2^20 */
  int32_t beams;                        /* of a request: 1..PS_BEAM_MAX_BEAMS */
  int32_t vocab;                        /* tokens: 1..PS_BEAM_MAX_VOCAB */
  int32_t dtype;                        /* ps_beam_dtype_t */
  int32_t num_end;                      /* 0..PS_BEAM_MAX_END */
  int32_t end_tokens[PS_BEAM_MAX_END];  /* the tokens that end a sequence: distinct, 0..vocab - 1 */
  int32_t pad0;
} ps_beam_config_t;

typedef struct ps_beam ps_beam_t;

/* Bytes of device workspace a handle needs (256-byte aligned base required), or 0
 * if the configuration is invalid.  With n = max_requests * beams rows: partial
 * results, 516 n bytes, and lists of 8 * beams bytes, the greater of 32 min(n, 4096)
 * and 2 n + 3840 of them. */
size_t ps_beam_workspace_bytes(const ps_beam_config_t* cfg);

/* Create a handle on the current device.  The workspace, which need not be cleared,
 * must stay allocated and untouched until ps_beam_destroy(). */
int32_t ps_beam_create(ps_beam_t** out, const ps_beam_config_t* cfg, void* d_workspace, size_t workspace_bytes);

/* Free the host-side handle.  The workspace is the caller's to free. */
void ps_beam_destroy(ps_beam_t* beam);

/* One step.  Beam b of request r has the score c = scores[r * beams + b] (the sum
 * of its tokens' log-probabilities; -infinity: there is no such beam, whatever its
 * logits are) and the logits x[v] = logits[r * request_stride + b *
 * beam_stride + v].  Continuing it with token v has the score
 *   c + x[v] - log sum_u exp x[u],
 * the sum in 32 bits at least, the score in 64, rounded once.  A logit of
 * -infinity is a token that cannot follow.  Candidates are ordered by score, equal
 * ones by beam, then by token, the lowest first.  (Logits of one beam that differ by
 * less than 64 bits hold beside the score, such as 1e-20 and 2e-20 where it is -5,
 * are in either order.)  Of each request
 *   tokens, parents, scores_out  [beams] are the first candidates whose tokens end
 *     nothing, and the beams (0..beams - 1) that they continue;
 *   ended_tokens, ended_parents, ended_scores  [beams] (all three or none) are the
 *     end tokens among the first 'beams' candidates of all kinds.
 * Where there are fewer, token and parent are -1 and the score is -infinity.
 * scores_out may be scores; otherwise outputs lie on no input and on no other
 * output (refused).  The same call gives the same bits.  A beam whose score, or
 * one of whose logits, is NaN or +infinity sets *d_status to PS_ERR_INVALID_ARG
 * and has no candidates. */
typedef struct {
  const void* logits;
  const float* scores;
  int32_t* tokens;
  int32_t* parents;
  float* scores_out;
  int32_t* ended_tokens;
  int32_t* ended_parents;
  float* ended_scores;
  int64_t request_stride, beam_stride; /* elements, not negative */
  int32_t num_requests;                /* 0..max_requests */
  int32_t pad0;
} ps_beam_select_t;
int32_t ps_beam_select(ps_beam_t* beam, void* stream, const ps_beam_select_t* a, int32_t* d_status);

/* Sequences of num_requests requests over num_steps steps: tokens and parents
 * [num_steps][num_requests][beams] are what every step's selection gave.
 * Hypothesis h (of 'hyps') of request r ends at step L - 1, L =
 * lengths[r * hyps + h] (NULL: num_steps), in beam b = beams_of[r * hyps + h]:
 * out[(r * hyps + h) * num_steps + t] is the token of step t on its way, for t < L,
 * and -1 from L on.  b = -1: no hypothesis, all -1.  (One that ended at step s with
 * parent p has L = s and beam p; its end token is not among these.)  A beam, a
 * length or a parent out of range sets *d_status to PS_ERR_INVALID_ARG, and the
 * tokens that it would have led to are -1.  out lies on no input (refused). */
typedef struct {
  const int32_t* tokens;
  const int32_t* parents;
  const int32_t* beams_of;
  const int32_t* lengths;
  int32_t* out;
  int32_t num_steps;    /* 0..2^24 */
  int32_t num_requests; /* 0..max_requests */
  int32_t hyps;         /* 0..2^16 */
  int32_t pad0;
} ps_beam_trace_t;
int32_t ps_beam_trace(ps_beam_t* beam, void* stream, const ps_beam_trace_t* a, int32_t* d_status);

#ifdef __cplusplus
}
#endif

#endif /* PREFIXSHIELD_BEAM_H */
