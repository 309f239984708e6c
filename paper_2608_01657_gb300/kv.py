"""The operators on the KV pages whose block ids the prefix cache hands out.

``KVPool`` wraps one pool of keys and values and the C ABI of
``include/prefixshield_kv.h``: laying a batch out (offsets, lengths, tables,
positions, slots), appending tokens (norms of queries and keys, rotation, page
write), attention over the pages with shared prefixes read once, copying,
forking, freeing and compacting pages, and the beam step of a search's rows.  As in ``binding``,
arguments are marshalled here and all work runs in the library's CUDA kernels;
torch provides device memory and streams.  Calls are enqueued on ``stream``
(default: the current one) and do not synchronize; what a call that names its
stream is given may be dropped once the call returns, and so may a plan's
tensors once the next plan is made, and the pool; errors that only the device
can see are reported in the int32 tensor ``pool.status``, which is sticky until
``check()``.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional

import torch

from . import binding as B

_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _fit(name: str, *sizes: int):
    """The library's sizes have 32 bits, and what is greater would come to it as another number."""
    for n in sizes:
        if not -1 << 31 <= n < 1 << 31:
            raise ValueError(f"{name}: {n} is out of range")


class Handle:
    """What the wrappers of the library's handles share: ``status`` (a sticky int32
    word of the device's errors), the streams that the handle's memory is used on,
    and checks of arrays.  A subclass sets ``device``, ``workspace``, ``status``
    and ``_kept``, the tensors that outlive its calls, and calls ``_begin``."""

    _h = None
    _destroy = ""               # entry point that frees the handle
    _what = "a call on the pool"

    def _begin(self, stream):
        self._index = self.device.index
        self._used = {}  # streams that the handle's memory is recorded on
        self._lib = B.load()
        self._status = self.status.data_ptr()
        self._stream(stream)

    def close(self):
        if getattr(self, "_h", None):
            getattr(B.load(), self._destroy)(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @staticmethod
    def _raise(name: str, rc: int):
        if rc != B.PS_OK:
            raise RuntimeError(f"{name} failed: {B.load().ps_status_string(rc).decode()} ({rc})")

    def check(self):
        """Raise if a call's device work reported an error; clears it (synchronizes:
        the device, if calls were made on other streams than the current one)."""
        elsewhere = any(raw != _raw_stream(self._index) for raw in self._used)
        if elsewhere:
            torch.cuda.synchronize(self.device)
        rc = int(self.status.item())
        if rc != B.PS_OK:
            self.status.zero_()
            if elsewhere:  # before the next call on another stream
                torch.cuda.synchronize(self.device)
            self._raise(self._what, rc)

    # -- argument checks ---------------------------------------------------
    def _stream(self, stream):
        """The raw handle of a call's stream.  What the handle keeps (the pool, the
        workspace, the status) is recorded on each stream that it is used on, so
        that its memory outlives the work there."""
        raw = _raw_stream(self._index) if stream is None else B._stream_ptr(stream)
        if raw not in self._used:
            self._used[raw] = B._stream_object(raw, self.device)
            self._record(raw, *self._kept)
        return raw

    def _record(self, raw, *tensors):
        for t in tensors:
            if t is not None:
                t.record_stream(self._used[raw])

    def _array(self, t, dtype, name: str, n: Optional[int] = None):
        sh = t.shape
        if len(sh) != 1 or t.dtype is not dtype or t.get_device() != self._index or not t.is_contiguous() or (
                n is not None and sh[0] != n):
            raise ValueError(f"{name} must be a contiguous {dtype} array" + ("" if n is None else f" of {n}"))
        return t.data_ptr()


def _addresses(tensors):
    return tuple([0 if t is None else t.data_ptr() for t in tensors])


class Layout(NamedTuple):
    """A batch's arrays, as ``append`` and ``plan`` take them."""
    q_offsets: torch.Tensor                # int32 [requests + 1]
    kv_lens: torch.Tensor                  # int32 [requests]
    tables: torch.Tensor                   # int32 [requests, pages]
    positions: torch.Tensor                # int32 [tokens]
    slots: torch.Tensor                    # int64 [tokens]
    group_offsets: Optional[torch.Tensor]  # int32 [requests + 1]


class _MadeLayout(Layout):
    """A layout that ``KVPool.layout`` made: ``made`` has the pool, the sizes and the
    addresses, so that its tensors are checked once, as long as their memory is the
    same.  (``_replace`` makes one without.)"""


class KVPool(Handle):
    """One paged pool of keys and values on the current CUDA device.

    ``k`` and ``v`` are tensors [layers, pages, page_size, kv_heads, head_dim]
    with the same strides, the innermost one 1 (a head-major pool is passed as
    its transposed view).  Page ids below ``first_page`` are the prefix
    cache's block ids, the others private pages of running requests.  The
    references count private pages alone: a later step of the cache may evict a
    block that a row still names, so no step runs while rows name cached pages,
    or the pages that it evicts are copied to private ones before its appends."""

    _destroy = "ps_kv_destroy"

    def __init__(self, k, v, num_q_heads: int, first_page: int = 0, max_requests: int = 1, max_tokens: int = 1,
                 max_row_pages: int = 1, stream=None):
        L = B.load()
        _need(k.dim() == 5 and k.shape == v.shape and k.stride() == v.stride() and k.dtype == v.dtype,
              "k and v must be alike: [layers, pages, page_size, kv_heads, head_dim]")
        _need(k.is_cuda and v.device == k.device and k.device.index == torch.cuda.current_device(),
              "k and v must be on the current CUDA device")
        _need(k.dtype in (torch.bfloat16, torch.float16), "a pool is bfloat16 or float16")
        _need(k.stride(4) == 1, "the innermost stride must be 1")
        self.k, self.v, self.dtype, self.device = k, v, k.dtype, k.device
        self.layers, self.pages, self.page_size, self.kv_heads, self.head_dim = (int(x) for x in k.shape)
        self.q_heads, self.first_page = int(num_q_heads), int(first_page)
        self.max_requests, self.max_tokens, self.max_row_pages = int(max_requests), int(max_tokens), int(max_row_pages)
        c = B.PsKvConfig(k=k.data_ptr(), v=v.data_ptr(), num_pages=self.pages, first_page=self.first_page,
                         layer_stride=k.stride(0), page_stride=k.stride(1), token_stride=k.stride(2),
                         head_stride=k.stride(3), num_layers=self.layers, page_size=self.page_size,
                         num_kv_heads=self.kv_heads, num_q_heads=self.q_heads, head_dim=self.head_dim,
                         dtype=B.PS_KV_BF16 if k.dtype == torch.bfloat16 else B.PS_KV_F16,
                         max_requests=self.max_requests, max_tokens=self.max_tokens, max_row_pages=self.max_row_pages)
        nbytes = L.ps_kv_workspace_bytes(C.byref(c))
        _need(nbytes > 0, "invalid pool configuration")
        with B._on_stream(stream, self.device):
            self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
        h = C.c_void_p()
        self._raise("ps_kv_create", L.ps_kv_create(C.byref(h), C.byref(c), self.workspace.data_ptr(), nbytes,
                                                   B._stream_ptr(stream)))
        self._h = h
        self._batch = None
        self._batch_used = set()  # streams that the plan's memory is recorded on
        self._kept = (self.k, self.v, self.workspace, self.status)
        self._begin(stream)
        # argument structures and entry points of the calls that a decode step
        # makes for every layer; their fields are filled in anew each time
        self._append_args, self._attention_args = B.PsKvAppend(), B.PsKvAttention()
        self._append_ref, self._attention_ref = C.byref(self._append_args), C.byref(self._attention_args)
        self._rows_args = B.PsKvRows()
        self._rows_ref = C.byref(self._rows_args)
        self._layout_args = B.PsKvLayout()
        self._layout_ref = C.byref(self._layout_args)
        self._private = max(0, self.pages - self.first_page)
        self._append_strides = [getattr(self._append_args, n) for n in ("q_stride", "k_stride", "v_stride", "q_out_stride")]
        self._attention_strides = [getattr(self._attention_args, n) for n in ("q_stride", "out_stride")]

    def _heads(self, t, tokens: int, heads: int, name: str, strides):
        """Checks [tokens, heads, head_dim]; its strides go to ``strides``."""
        if t.shape != (tokens, heads, self.head_dim) or t.dtype is not self.dtype or t.get_device() != self._index:
            raise ValueError(f"{name} must be {self.dtype} [{tokens}, {heads}, {self.head_dim}] on {self.device}")
        s0, s1, s2 = t.stride()
        # an axis of one element is never stepped over: its stride may be any number
        strides[0] = s0 = s0 if tokens > 1 else 0
        strides[1] = s1 = s1 if heads > 1 else 0
        p = t.data_ptr()
        if s2 != 1 or (s0 | s1) & 7 or p & 15:
            raise ValueError(f"{name}: heads must be contiguous, on 16-byte boundaries")
        return p

    def _table(self, t, name: str):
        sh = t.shape
        if len(sh) != 2 or t.dtype is not torch.int32 or t.get_device() != self._index or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous int32 [rows, pages] tensor")
        return sh

    # -- one layer's new tokens ----------------------------------------------
    def append(self, layer: int, q, k, v, slots, positions=None, rope=None, interleaved: bool = False, q_weight=None,
               k_weight=None, eps: float = 1e-6, q_out=None, stream=None):
        """Norm (with ``q_weight`` / ``k_weight``) and rotation (with ``rope``
        [rows, rope_dim] float32: cosines, then sines) of the new tokens'
        queries and keys; keys and values go to ``slots`` (page * page_size +
        offset, int64; negative: not written).  Returns the queries, NaN where a
        token was left out and ``q_out`` not given."""
        a, st = self._append_args, self._append_strides
        T = q.shape[0]
        a.fill = q_out is None
        if q_out is None:
            q_out = B._made((T, self.q_heads, self.head_dim), self.dtype, self.device, stream)
        a.q = self._heads(q, T, self.q_heads, "q", st[0])
        a.k = self._heads(k, T, self.kv_heads, "k", st[1])
        a.v = self._heads(v, T, self.kv_heads, "v", st[2])
        a.q_out = self._heads(q_out, T, self.q_heads, "q_out", st[3])
        a.slots = self._array(slots, torch.int64, "slots", T)
        if rope is not None:
            if positions is None:
                raise ValueError("a rotation needs positions")
            if len(rope.shape) != 2 or rope.dtype is not torch.float32 or not rope.is_contiguous() or rope.device != self.device:
                raise ValueError("rope must be a contiguous float32 [rows, rope_dim] table")
            a.positions = self._array(positions, torch.int32, "positions", T)
            a.rope = rope.data_ptr()
            a.rope_rows, a.rope_dim = rope.shape
            a.rope_interleaved = 1 if interleaved else 0
        else:
            a.positions = a.rope = None
            a.rope_dim = 0
        a.q_weight = None if q_weight is None else self._array(q_weight, self.dtype, "q_weight", self.head_dim)
        a.k_weight = None if k_weight is None else self._array(k_weight, self.dtype, "k_weight", self.head_dim)
        a.eps, a.num_tokens = eps, T
        raw = self._stream(stream)
        rc = self._lib.ps_kv_append(self._h, raw, layer, self._append_ref, self._status)
        if rc:
            self._raise("ps_kv_append", rc)
        if stream is not None:
            self._record(raw, q, k, v, slots, positions, rope, q_weight, k_weight, q_out)
        return q_out

    # -- a batch's arrays ------------------------------------------------------
    def layout(self, rows, tables, lens, held, num_tokens: int, counts=None, starts=None, written=None, pad: bool = False,
               groups: bool = True, out: Optional[Layout] = None, stream=None) -> Layout:
        """Where the new tokens of a batch go.  Request i is row ``rows[i]`` (None:
        row i) of ``tables`` / ``lens`` / ``held`` and has ``counts[i]`` (None: one)
        new tokens after its first ``starts[i]`` (None: the row's lens); tokens at
        positions below ``written[i]`` get slot -1.  The rest of ``num_tokens`` has
        slot -1, too, and with ``pad`` belongs to one more request without keys, so
        that the layout of a captured graph can be planned whatever the counts are.
        ``groups``: with the runs of requests that may share a prefix.  ``out``: an
        earlier layout of the same shape to write to.  A batch with a request out
        of range, or more tokens than ``num_tokens``, is left out whole: every slot
        is -1, and a plan of it is refused."""
        a = self._layout_args
        r = self._rows(tables, lens, held)
        width = self._rows_args.table_stride
        n = tables.shape[0] if rows is None else rows.shape[0]
        T, all_ = int(num_tokens), n + bool(pad)
        if T >> 31 or n >> 31:
            _fit("layout", n, T)
        i32 = torch.int32
        a.rows = None if rows is None else self._array(rows, i32, "rows")
        a.counts = None if counts is None else self._array(counts, i32, "counts", n)
        a.starts = None if starts is None else self._array(starts, i32, "starts", n)
        a.written = None if written is None else self._array(written, i32, "written", n)
        if out is None:
            made = lambda *shape, dtype=i32: B._made(shape, dtype, self.device, stream)  # noqa: E731
            out = _MadeLayout(made(all_ + 1), made(all_), made(all_, width), made(T), made(T, dtype=torch.int64),
                              made(all_ + 1) if groups else None)
            out.made = (self, all_, width, T, *_addresses(out))
        known = getattr(out, "made", None)
        if known is not None and known[0] is self and known[1:4] == (all_, width, T) and known[4:] == _addresses(out):
            a.q_offsets, a.kv_lens, a.tables, a.positions, a.slots, a.group_offsets = known[4:]
        else:
            self._table(out.tables, "out.tables")
            if out.tables.shape[0] != all_ or out.tables.shape[1] != width:
                raise ValueError(f"out.tables must be [{all_}, {width}]")
            a.q_offsets = self._array(out.q_offsets, i32, "out.q_offsets", all_ + 1)
            a.kv_lens = self._array(out.kv_lens, i32, "out.kv_lens", all_)
            a.tables = out.tables.data_ptr()
            a.positions = self._array(out.positions, i32, "out.positions", T)
            a.slots = self._array(out.slots, torch.int64, "out.slots", T)
            a.group_offsets = None if out.group_offsets is None else self._array(out.group_offsets, i32, "out.group_offsets", all_ + 1)
        a.num_requests, a.num_tokens, a.pad = n, T, 1 if pad else 0
        raw = self._stream(stream)
        rc = self._lib.ps_kv_layout(self._h, raw, r, self._layout_ref, self._status)
        if rc:
            self._raise("ps_kv_layout", rc)
        if stream is not None:
            self._record(raw, rows, tables, lens, held, counts, starts, written, *out)
        return out

    # -- attention -------------------------------------------------------------
    def plan(self, q_offsets, kv_lens, tables, num_tokens: int, group_offsets=None, causal: bool = True, stream=None):
        """Plan the attention of a batch (one plan serves every layer).
        Request i's queries are the tokens q_offsets[i]..q_offsets[i+1], the
        last of its kv_lens[i]; ``group_offsets`` divides the requests into
        runs of neighbours that may share a prefix.  The tensors must stay
        unchanged while the plan is used."""
        R = int(kv_lens.shape[0])
        self._table(tables, "tables")
        _need(int(tables.shape[0]) >= R, "tables must have a row for each request")
        b = B.PsKvBatch(q_offsets=self._array(q_offsets, torch.int32, "q_offsets", R + 1),
                        kv_lens=self._array(kv_lens, torch.int32, "kv_lens"), tables=tables.data_ptr(),
                        table_stride=int(tables.shape[1]), num_requests=R, num_tokens=int(num_tokens), causal=int(causal))
        if group_offsets is not None:
            b.group_offsets, b.num_groups = self._array(group_offsets, torch.int32, "group_offsets"), int(group_offsets.shape[0]) - 1
        self._batch = None
        raw = self._stream(stream)
        self._raise("ps_kv_plan", self._lib.ps_kv_plan(self._h, raw, C.byref(b), self._status))
        # alive while the plan is, and after it until the work on the streams that use it is done
        self._batch = (q_offsets, kv_lens, tables, group_offsets, int(num_tokens))
        self._batch_used = {raw}
        self._record(raw, *self._batch[:4])

    def attention(self, layer: int, q, scale: float, out=None, lse=None, stream=None):
        """softmax(scale q k^T) v of one layer for the planned batch.  ``lse``
        (optional, float32 [tokens, q_heads]) receives the scores' log-sum-exp.
        If the plan was found bad, nothing is written; an output that was not
        given is NaN then."""
        if self._batch is None:
            raise ValueError("attention needs a plan")
        T = self._batch[4]
        a, st = self._attention_args, self._attention_strides
        a.fill = out is None
        if out is None:
            out = B._made((T, self.q_heads, self.head_dim), self.dtype, self.device, stream)
        a.q = self._heads(q, T, self.q_heads, "q", st[0])
        a.out = self._heads(out, T, self.q_heads, "out", st[1])
        a.scale = scale
        if lse is not None:
            if lse.shape != (T, self.q_heads) or lse.dtype is not torch.float32 or not lse.is_contiguous() or lse.device != self.device:
                raise ValueError("lse must be contiguous float32 [tokens, q_heads]")
            a.lse = lse.data_ptr()
        else:
            a.lse = None
        raw = self._stream(stream)
        if raw not in self._batch_used:
            self._batch_used.add(raw)
            self._record(raw, *self._batch[:4])
        rc = self._lib.ps_kv_attention(self._h, raw, layer, self._attention_ref, self._status)
        if rc:
            self._raise("ps_kv_attention", rc)
        if stream is not None:
            self._record(raw, q, out, lse)
        return out

    # -- pages -------------------------------------------------------------------
    def copy(self, src, dst, stream=None):
        """Copy whole pages src[i] -> dst[i], all layers."""
        n, raw = src.shape[0], self._stream(stream)
        rc = self._lib.ps_kv_copy(self._h, raw, n, self._array(src, torch.int32, "src"),
                                  self._array(dst, torch.int32, "dst", n), self._status)
        if rc:
            self._raise("ps_kv_copy", rc)
        if stream is not None:
            self._record(raw, src, dst)

    def _rows(self, tables, lens, held):
        """Fills in the structure of the rows; returns the reference to pass."""
        n, width = self._table(tables, "tables")
        r = self._rows_args
        r.num_rows, r.table_stride = n, width
        r.tables = tables.data_ptr()
        r.lens = None if lens is None else self._array(lens, torch.int32, "lens", n)
        r.held = self._array(held, torch.int32, "held", n)
        return self._rows_ref

    def _refs(self, refs, name="refs"):
        return self._array(refs, torch.int32, name, self._private)

    def fork(self, parents, children, room, tables, lens, held, refs, refs_out=None, stream=None):
        """Rows ``children`` become continuations of rows ``parents`` with
        pages for ``room`` tokens: in place (parent == child), new (parent -1)
        or a fork that shares the full pages and copies the partial one."""
        n, raw = parents.shape[0], self._stream(stream)
        rows, before = self._rows(tables, lens, held), self._refs(refs)
        rc = self._lib.ps_kv_fork(
            self._h, raw, n, self._array(parents, torch.int32, "parents"),
            self._array(children, torch.int32, "children", n), self._array(room, torch.int32, "room", n), rows,
            before, before if refs_out is None else self._refs(refs_out, "refs_out"), self._status)
        if rc:
            self._raise("ps_kv_fork", rc)
        if stream is not None:
            self._record(raw, parents, children, room, tables, lens, held, refs, refs_out)

    def reorder(self, rows, parents, tables, lens, held, refs, grow: int = 1, refs_out=None, stream=None):
        """A beam step: ``rows`` [requests, beams] become continuations of their
        requests' beams ``parents`` [requests, beams] (-1: an empty row), with
        pages for ``grow`` more tokens than those have.  Full pages are shared, a
        beam's first continuation takes over its partly filled page, the others
        copy it; what no beam continues is freed."""
        sh = rows.shape
        if len(sh) != 2 or sh != parents.shape:
            raise ValueError("rows and parents must be [requests, beams]")
        (n, beams), raw = sh, self._stream(stream)
        _fit("reorder", n, beams, grow)
        for t, name in ((rows, "rows"), (parents, "parents")):
            if t.dtype is not torch.int32 or t.get_device() != self._index or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous int32 [requests, beams] tensor")
        r, before = self._rows(tables, lens, held), self._refs(refs)
        rc = self._lib.ps_kv_reorder(self._h, raw, n, beams, rows.data_ptr(), parents.data_ptr(), grow, r, before,
                                     before if refs_out is None else self._refs(refs_out, "refs_out"), self._status)
        if rc:
            self._raise("ps_kv_reorder", rc)
        if stream is not None:
            self._record(raw, rows, parents, tables, lens, held, refs, refs_out)

    def release(self, rows, tables, lens, held, refs, stream=None):
        """Free the pages that ``rows`` hold."""
        r, raw = self._rows(tables, lens, held), self._stream(stream)
        rc = self._lib.ps_kv_release(self._h, raw, rows.shape[0], self._array(rows, torch.int32, "rows"), r,
                                     self._refs(refs), self._status)
        if rc:
            self._raise("ps_kv_release", rc)
        if stream is not None:
            self._record(raw, rows, tables, lens, held, refs)

    def compact(self, tables, held, refs, tables_out=None, refs_out=None, counts=None, stream=None):
        """Move the private pages in use to the lowest ids.  Returns the int32
        tensor (pages in use, pages moved)."""
        r, before = self._rows(tables, None, held), self._refs(refs)
        if counts is None:
            counts = B._made(2, torch.int32, self.device, stream)
        tables_out = tables if tables_out is None else tables_out
        self._table(tables_out, "tables_out")
        _need(tables_out.shape == tables.shape, "tables_out must be shaped as tables")
        raw = self._stream(stream)
        rc = self._lib.ps_kv_compact(
            self._h, raw, r, before, tables_out.data_ptr(),
            before if refs_out is None else self._refs(refs_out, "refs_out"), self._array(counts, torch.int32, "counts", 2),
            self._status)
        if rc:
            self._raise("ps_kv_compact", rc)
        if stream is not None:
            self._record(raw, tables, held, refs, tables_out, refs_out, counts)
        return counts
