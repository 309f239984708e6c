"""Beam search over the requests whose keys and values lie in KV pages.

``BeamSearch`` wraps the C ABI of ``include/prefixshield_beam.h``: ``select``
picks the best continuations of every request's beams over beams and vocabulary,
``trace`` follows the steps' parents back to sequences of tokens.  Between two
steps, ``kv.KVPool.reorder`` makes the beams' pages follow their parents.  With
one beam, ``select`` is the likeliest token and its log-probability.  Calls are
enqueued on ``stream`` (default: the current one) and do not synchronize, as
``kv.KVPool``'s are.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional, Sequence

import torch

from . import binding as B
from .kv import Handle, _addresses, _fit, _need

_DTYPES = {torch.bfloat16: B.PS_BEAM_BF16, torch.float16: B.PS_BEAM_F16, torch.float32: B.PS_BEAM_F32}


class Selection(NamedTuple):
    """A step's outcome, [requests, beams] each; -1 and -infinity where there is none."""
    tokens: torch.Tensor                   # int32
    parents: torch.Tensor                  # int32, the beams that they continue
    scores: torch.Tensor                   # float32
    ended_tokens: Optional[torch.Tensor]   # int32, end tokens among the first candidates
    ended_parents: Optional[torch.Tensor]  # int32
    ended_scores: Optional[torch.Tensor]   # float32


class _MadeSelection(Selection):
    """A selection that ``BeamSearch.select`` made: ``made`` has the search, the requests
    and the addresses, so that its tensors are checked once, as long as their memory is
    the same.  (``_replace`` makes one without.)"""


class BeamSearch(Handle):
    """Beam searches on the current CUDA device: at most ``max_requests`` requests
    of ``beams`` beams each, over logits of ``vocab`` tokens in ``dtype`` (bfloat16,
    float16 or float32).  A beam that takes one of ``end_tokens`` ends."""

    _destroy, _what = "ps_beam_destroy", "a call of the beam search"

    def __init__(self, max_requests: int, beams: int, vocab: int, dtype=torch.bfloat16, end_tokens: Sequence[int] = (), stream=None):
        L = B.load()
        end_tokens = [int(t) for t in end_tokens]
        _need(dtype in _DTYPES, "logits are bfloat16, float16 or float32")
        _need(len(end_tokens) <= B.PS_BEAM_MAX_END, f"at most {B.PS_BEAM_MAX_END} end tokens")
        self.max_requests, self.beams, self.vocab, self.dtype = int(max_requests), int(beams), int(vocab), dtype
        self.end_tokens = tuple(end_tokens)
        _fit("beam search", self.max_requests, self.beams, self.vocab, *end_tokens)
        self.device = torch.device("cuda", torch.cuda.current_device())
        c = B.PsBeamConfig(max_requests=self.max_requests, beams=self.beams, vocab=self.vocab, dtype=_DTYPES[dtype],
                           num_end=len(end_tokens))
        for i, t in enumerate(end_tokens):
            c.end_tokens[i] = t
        nbytes = L.ps_beam_workspace_bytes(C.byref(c))
        _need(nbytes > 0, "invalid beam search configuration")
        with B._on_stream(stream, self.device):
            self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
        h = C.c_void_p()
        self._raise("ps_beam_create", L.ps_beam_create(C.byref(h), C.byref(c), self.workspace.data_ptr(), nbytes))
        self._h = h
        self._kept = (self.workspace, self.status)
        self._begin(stream)
        self._select_args, self._trace_args = B.PsBeamSelect(), B.PsBeamTrace()
        self._select_ref, self._trace_ref = C.byref(self._select_args), C.byref(self._trace_args)

    def _of(self, t, dtype, shape, name: str):
        if t.shape != shape or t.dtype is not dtype or t.get_device() != self._index or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous {dtype} {list(shape)} on {self.device}")
        return t.data_ptr()

    def select(self, logits, scores, out: Optional[Selection] = None, ended: bool = True, stream=None) -> Selection:
        """The best continuations of a step.  ``logits`` [requests, beams, vocab] (rows
        contiguous), ``scores`` [requests, beams] float32: the sums of the beams'
        log-probabilities, -infinity where there is no beam (in a first step, all but
        one).  A candidate's score is its beam's plus the token's log-probability.  Of
        the candidates that end nothing the first ``beams`` go on; with ``ended`` the
        end tokens among the first ``beams`` of all come separately.  ``out``: an
        earlier selection to write to; its scores may be ``scores``.  A beam whose
        score or logits are NaN or +infinity is reported and has no candidates."""
        a = self._select_args
        sh, st = logits.shape, logits.stride()
        if len(sh) != 3 or sh[1] != self.beams or sh[2] != self.vocab or logits.dtype is not self.dtype or (
                logits.get_device() != self._index) or (st[2] != 1 and self.vocab > 1):
            raise ValueError(f"logits must be {self.dtype} [requests, {self.beams}, {self.vocab}] on {self.device}, rows contiguous")
        R = sh[0]
        if R >> 31:
            _fit("select", R)
        shape, i32, f32 = (R, self.beams), torch.int32, torch.float32
        a.logits = logits.data_ptr()
        a.request_stride, a.beam_stride = st[0], st[1]
        a.scores = self._of(scores, f32, shape, "scores")
        if out is None:
            made = lambda dtype: B._made(shape, dtype, self.device, stream)  # noqa: E731
            out = _MadeSelection(made(i32), made(i32), made(f32), *((made(i32), made(i32), made(f32)) if ended else (None, None, None)))
            out.made = (self, R, *_addresses(out))
        known = getattr(out, "made", None)
        if known is not None and known[0] is self and known[1] == R and known[2:] == _addresses(out):
            a.tokens, a.parents, a.scores_out, a.ended_tokens, a.ended_parents, a.ended_scores = known[2:]
        else:
            a.tokens = self._of(out.tokens, i32, shape, "out.tokens")
            a.parents = self._of(out.parents, i32, shape, "out.parents")
            a.scores_out = self._of(out.scores, f32, shape, "out.scores")
            a.ended_tokens = None if out.ended_tokens is None else self._of(out.ended_tokens, i32, shape, "out.ended_tokens")
            a.ended_parents = None if out.ended_parents is None else self._of(out.ended_parents, i32, shape, "out.ended_parents")
            a.ended_scores = None if out.ended_scores is None else self._of(out.ended_scores, f32, shape, "out.ended_scores")
        a.num_requests = R
        raw = self._stream(stream)
        rc = self._lib.ps_beam_select(self._h, raw, self._select_ref, self._status)
        if rc:
            self._raise("ps_beam_select", rc)
        if stream is not None:
            self._record(raw, logits, scores, *out)
        return out

    def trace(self, tokens, parents, beams, lengths=None, out=None, stream=None):
        """Sequences of tokens [requests, hypotheses, steps], int32.  ``tokens`` and
        ``parents`` [steps, requests, beams] are what every step's selection gave;
        hypothesis h of request r ends in beam ``beams[r, h]`` (-1: there is none)
        after ``lengths[r, h]`` steps (None: all), and is -1 from there on."""
        a = self._trace_args
        i32 = torch.int32
        sh, of = tokens.shape, beams.shape
        if len(sh) != 3 or sh[2] != self.beams or len(of) != 2 or of[0] != sh[1]:
            raise ValueError(f"tokens must be [steps, requests, {self.beams}], beams [requests, hypotheses]")
        T, R, _ = sh
        N = of[1]
        if T >> 31 or R >> 31 or N >> 31:
            _fit("trace", T, R, N)
        a.tokens = self._of(tokens, i32, sh, "tokens")
        a.parents = self._of(parents, i32, sh, "parents")
        a.beams_of = self._of(beams, i32, of, "beams")
        a.lengths = None if lengths is None else self._of(lengths, i32, of, "lengths")
        if out is None:
            out = B._made((R, N, T), i32, self.device, stream)
        a.out = self._of(out, i32, (R, N, T), "out")
        a.num_steps, a.num_requests, a.hyps = T, R, N
        raw = self._stream(stream)
        rc = self._lib.ps_beam_trace(self._h, raw, self._trace_ref, self._status)
        if rc:
            self._raise("ps_beam_trace", rc)
        if stream is not None:
            self._record(raw, tokens, parents, beams, lengths, out)
        return out
