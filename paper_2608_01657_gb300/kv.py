"""The operators on the KV pages whose block ids the prefix cache hands out.

``KVPool`` wraps one pool of keys and values and the C ABI of
``include/prefixshield_kv.h``: appending tokens (norms of queries and keys,
rotation, page write), attention over the pages with shared prefixes read once,
and copying, forking, freeing and compacting pages.  As in ``binding``,
arguments are marshalled here and all work runs in the library's CUDA kernels;
torch provides device memory and streams.  Calls are enqueued on ``stream``
(default: the current one) and do not synchronize; errors that only the device
can see are reported in the int32 tensor ``pool.status``, which is sticky until
``check()``.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional

from . import binding as B


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


class KVPool:
    """One paged pool of keys and values on the current CUDA device.

    ``k`` and ``v`` are tensors [layers, pages, page_size, kv_heads, head_dim]
    with the same strides, the innermost one 1 (a head-major pool is passed as
    its transposed view).  Page ids below ``first_page`` are the prefix
    cache's block ids, the others private pages of running requests."""

    def __init__(self, k, v, num_q_heads: int, first_page: int = 0, max_requests: int = 1, max_tokens: int = 1,
                 max_row_pages: int = 1, stream=None):
        import torch
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
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
        h = C.c_void_p()
        self._raise("ps_kv_create", L.ps_kv_create(C.byref(h), C.byref(c), self.workspace.data_ptr(), nbytes,
                                                   B._stream_ptr(stream)))
        self._h = h
        self._batch = None

    def close(self):
        if getattr(self, "_h", None):
            B.load().ps_kv_destroy(self._h)
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
        """Raise if a call's device work reported an error; clears it (synchronizes)."""
        rc = int(self.status.item())
        if rc != B.PS_OK:
            self.status.zero_()
            self._raise("a call on the pool", rc)

    # -- argument checks ---------------------------------------------------
    def _heads(self, t, heads: int, name: str, tokens: Optional[int] = None):
        _need(t.dim() == 3 and t.shape[1] == heads and t.shape[2] == self.head_dim and t.dtype == self.dtype
              and t.device == self.device, f"{name} must be {self.dtype} [tokens, {heads}, {self.head_dim}]")
        _need(tokens is None or t.shape[0] == tokens, f"{name} must have {tokens} tokens")
        # an axis of one element is never stepped over: its stride may be any number
        s = [t.stride(i) if t.shape[i] > 1 else 0 for i in (0, 1)]
        _need((t.stride(2) == 1 or self.head_dim == 1) and s[0] % 8 == 0 and s[1] % 8 == 0 and t.data_ptr() % 16 == 0,
              f"{name}: heads must be contiguous, on 16-byte boundaries")
        return (C.c_int64 * 2)(*s)

    def _array(self, t, dtype, name: str, n: Optional[int] = None):
        _need(t.dim() == 1 and t.dtype == dtype and t.device == self.device and t.is_contiguous()
              and (n is None or t.shape[0] == n), f"{name} must be a contiguous {dtype} array" +
              ("" if n is None else f" of {n}"))
        return t.data_ptr()

    def _table(self, t, name: str):
        import torch
        _need(t.dim() == 2 and t.dtype == torch.int32 and t.device == self.device and t.is_contiguous(),
              f"{name} must be a contiguous int32 [rows, pages] tensor")

    # -- one layer's new tokens ----------------------------------------------
    def append(self, layer: int, q, k, v, slots, positions=None, rope=None, interleaved: bool = False, q_weight=None,
               k_weight=None, eps: float = 1e-6, q_out=None, stream=None):
        """Norm (with ``q_weight`` / ``k_weight``) and rotation (with ``rope``
        [rows, rope_dim] float32: cosines, then sines) of the new tokens'
        queries and keys; keys and values go to ``slots`` (page * page_size +
        offset, int64; negative: not written).  Returns the queries."""
        import torch
        T = int(q.shape[0])
        a = B.PsKvAppend(q_stride=self._heads(q, self.q_heads, "q"), k_stride=self._heads(k, self.kv_heads, "k", T),
                         v_stride=self._heads(v, self.kv_heads, "v", T))
        if q_out is None:
            q_out = torch.empty(T, self.q_heads, self.head_dim, dtype=self.dtype, device=self.device)
        a.q_out_stride = self._heads(q_out, self.q_heads, "q_out", T)
        a.q, a.k, a.v, a.q_out = q.data_ptr(), k.data_ptr(), v.data_ptr(), q_out.data_ptr()
        a.slots = self._array(slots, torch.int64, "slots", T)
        if rope is not None:
            _need(positions is not None, "a rotation needs positions")
            _need(rope.dim() == 2 and rope.dtype == torch.float32 and rope.is_contiguous() and rope.device == self.device,
                  "rope must be a contiguous float32 [rows, rope_dim] table")
            a.positions = self._array(positions, torch.int32, "positions", T)
            a.rope, a.rope_rows, a.rope_dim = rope.data_ptr(), int(rope.shape[0]), int(rope.shape[1])
            a.rope_interleaved = int(interleaved)
        if q_weight is not None:
            a.q_weight = self._array(q_weight, self.dtype, "q_weight", self.head_dim)
        if k_weight is not None:
            a.k_weight = self._array(k_weight, self.dtype, "k_weight", self.head_dim)
        a.eps, a.num_tokens = eps, T
        self._raise("ps_kv_append", B.load().ps_kv_append(self._h, B._stream_ptr(stream), int(layer), C.byref(a),
                                                          self.status.data_ptr()))
        return q_out

    # -- attention -------------------------------------------------------------
    def plan(self, q_offsets, kv_lens, tables, num_tokens: int, group_offsets=None, causal: bool = True, stream=None):
        """Plan the attention of a batch (one plan serves every layer).
        Request i's queries are the tokens q_offsets[i]..q_offsets[i+1], the
        last of its kv_lens[i]; ``group_offsets`` divides the requests into
        runs of neighbours that may share a prefix.  The tensors must stay
        unchanged while the plan is used."""
        import torch
        R = int(kv_lens.shape[0])
        self._table(tables, "tables")
        _need(tables.shape[0] >= R, "tables must have a row for each request")
        b = B.PsKvBatch(q_offsets=self._array(q_offsets, torch.int32, "q_offsets", R + 1),
                        kv_lens=self._array(kv_lens, torch.int32, "kv_lens"), tables=tables.data_ptr(),
                        table_stride=int(tables.shape[1]), num_requests=R, num_tokens=int(num_tokens), causal=int(causal))
        if group_offsets is not None:
            b.group_offsets, b.num_groups = self._array(group_offsets, torch.int32, "group_offsets"), int(group_offsets.shape[0]) - 1
        self._batch = None
        self._raise("ps_kv_plan", B.load().ps_kv_plan(self._h, B._stream_ptr(stream), C.byref(b), self.status.data_ptr()))
        self._batch = (q_offsets, kv_lens, tables, group_offsets, int(num_tokens))  # alive while the plan is

    def attention(self, layer: int, q, scale: float, out=None, lse=None, stream=None):
        """softmax(scale q k^T) v of one layer for the planned batch.  ``lse``
        (optional, float32 [tokens, q_heads]) receives the scores' log-sum-exp."""
        import torch
        _need(self._batch is not None, "attention needs a plan")
        T = self._batch[4]
        if out is None:
            out = torch.empty(T, self.q_heads, self.head_dim, dtype=self.dtype, device=self.device)
        a = B.PsKvAttention(q=q.data_ptr(), out=out.data_ptr(), q_stride=self._heads(q, self.q_heads, "q", T),
                            out_stride=self._heads(out, self.q_heads, "out", T), scale=scale)
        if lse is not None:
            _need(lse.dtype == torch.float32 and tuple(lse.shape) == (T, self.q_heads) and lse.is_contiguous()
                  and lse.device == self.device, "lse must be contiguous float32 [tokens, q_heads]")
            a.lse = lse.data_ptr()
        self._raise("ps_kv_attention", B.load().ps_kv_attention(self._h, B._stream_ptr(stream), int(layer), C.byref(a),
                                                                self.status.data_ptr()))
        return out

    # -- pages -------------------------------------------------------------------
    def copy(self, src, dst, stream=None):
        """Copy whole pages src[i] -> dst[i], all layers."""
        import torch
        n = int(src.shape[0])
        self._raise("ps_kv_copy", B.load().ps_kv_copy(
            self._h, B._stream_ptr(stream), n, self._array(src, torch.int32, "src"),
            self._array(dst, torch.int32, "dst", n), self.status.data_ptr()))

    def _rows(self, tables, lens, held):
        import torch
        self._table(tables, "tables")
        n = int(tables.shape[0])
        return B.PsKvRows(tables=tables.data_ptr(), lens=None if lens is None else self._array(lens, torch.int32, "lens", n),
                          held=self._array(held, torch.int32, "held", n), table_stride=int(tables.shape[1]), num_rows=n)

    def _refs(self, refs, name="refs"):
        import torch
        return self._array(refs, torch.int32, name, max(0, self.pages - self.first_page))

    def fork(self, parents, children, room, tables, lens, held, refs, refs_out=None, stream=None):
        """Rows ``children`` become continuations of rows ``parents`` with
        pages for ``room`` tokens: in place (parent == child), new (parent -1)
        or a fork that shares the full pages and copies the partial one."""
        import torch
        n = int(parents.shape[0])
        rows = self._rows(tables, lens, held)
        self._raise("ps_kv_fork", B.load().ps_kv_fork(
            self._h, B._stream_ptr(stream), n, self._array(parents, torch.int32, "parents"),
            self._array(children, torch.int32, "children", n), self._array(room, torch.int32, "room", n), C.byref(rows),
            self._refs(refs), self._refs(refs if refs_out is None else refs_out, "refs_out"), self.status.data_ptr()))

    def release(self, rows, tables, lens, held, refs, stream=None):
        """Free the pages that ``rows`` hold."""
        import torch
        r = self._rows(tables, lens, held)
        self._raise("ps_kv_release", B.load().ps_kv_release(
            self._h, B._stream_ptr(stream), int(rows.shape[0]), self._array(rows, torch.int32, "rows"), C.byref(r),
            self._refs(refs), self.status.data_ptr()))

    def compact(self, tables, held, refs, tables_out=None, refs_out=None, counts=None, stream=None):
        """Move the private pages in use to the lowest ids.  Returns the int32
        tensor (pages in use, pages moved)."""
        import torch
        r = self._rows(tables, None, held)
        if counts is None:
            counts = torch.empty(2, dtype=torch.int32, device=self.device)
        tables_out = tables if tables_out is None else tables_out
        self._table(tables_out, "tables_out")
        _need(tables_out.shape == tables.shape, "tables_out must be shaped as tables")
        self._raise("ps_kv_compact", B.load().ps_kv_compact(
            self._h, B._stream_ptr(stream), C.byref(r), self._refs(refs), tables_out.data_ptr(),
            self._refs(refs if refs_out is None else refs_out, "refs_out"), self._array(counts, torch.int32, "counts", 2),
            self.status.data_ptr()))
        return counts
