"""Paged caches with torch tensors as device memory, over the ``kvev_paged_*`` entry points.

:class:`PagePool` keeps a stack of free pages and the requests' block table: ``tables`` and ``release``
are a scheduler step.  :class:`PagedCache` is one layer's pages under such a table: ``write`` the new
tokens' rows, ``attention`` over them, ``gather`` whole prompts for ``Plan.evict_prefill``.  Lengths,
tables and slots stay on the device throughout.  Argument checks raise ``ValueError`` (shapes, types)
or ``KvevError`` (what the library refuses).  Calls run on the current stream or on ``stream``, and what
they return as new tensors is allocated on that stream: other streams wait for it and keep it
(``record_stream``) as they do with any tensor of torch's.

These are calls of a few microseconds on the device, made for every layer of every token: the checks
and the calls themselves are in the extension module ``kvev_paged_bind`` (``csrc/paged_bind.cpp``).
"""
from __future__ import annotations

import contextlib
import ctypes as C
import importlib.util
import os

import torch

from . import kvev

_DTYPES = {torch.bfloat16: kvev.BF16, torch.float16: kvev.FP16}
_I32 = torch.int32
_bind_module = None


def _bind():
    """The extension module (loaded once).  Raises if it is missing."""
    global _bind_module
    if _bind_module is None:
        kvev.load()
        path = os.path.join(os.path.dirname(kvev.LIB_PATH), "kvev_paged_bind.so")
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: build it with __graft_entry__.build()")
        spec = importlib.util.spec_from_file_location("kvev_paged_bind", path)
        m = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(m)
        _bind_module = m
    return _bind_module


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


# Scratch of the attention calls made on a stream, (device, stream) -> (pointer, bytes, tensor): calls on a stream
# follow one another, whatever layer they are for, so they share it.
_workspaces: dict = {}
# Scratch of the calls that a capture on the stream records, (device, stream) -> (capture's id, the same).  A graph's
# replays follow neither the stream's calls nor other graphs, so each capture has scratch of its own, from the
# graph's memory pool, whose counts the graph itself zeroes before its first attention.  Only the last capture's is
# kept: after a capture its memory is the graph's.
_captured: dict = {}


def _scratch(device: int, stream: int):
    n = kvev.kvev_paged_attention_workspace(1, 1, 128)  # what the largest call needs
    with torch.cuda.device(device), torch.cuda.stream(torch.cuda.ExternalStream(stream, device=device)):
        t = torch.empty(n, dtype=torch.uint8, device="cuda")
        t[:kvev.PAGED_SYNC_BYTES].zero_()
    return t.data_ptr(), n, t


def _workspace(device: int, stream: int, capture: int):
    if capture:
        held = _captured.get((device, stream))
        if held is None or held[0] != capture:
            held = _captured[device, stream] = (capture, _scratch(device, stream))
        return held[1]
    ws = _workspaces.get((device, stream))
    if ws is None:
        ws = _workspaces[device, stream] = _scratch(device, stream)
    return ws


def _given(ws, device: int):
    _need(isinstance(ws, torch.Tensor) and ws.is_cuda and ws.get_device() == device and ws.is_contiguous(),
          "workspace: a contiguous tensor on the cache's GPU")
    return ws.data_ptr(), ws.numel() * ws.element_size()


_here = contextlib.nullcontext()


def _on(stream):
    """Outputs made for a call belong to its stream: what the current one left in their memory may still be in use there."""
    return _here if stream is None else torch.cuda.stream(stream)


def _table(block_table) -> int:
    _need(block_table.dim() == 2 and block_table.is_cuda and block_table.dtype is _I32 and block_table.is_contiguous(),
          "block_table: contiguous int32 [requests][pages] on a GPU")
    return block_table.data_ptr()


def _strides(t) -> tuple:
    """Element strides; that of a dimension of one element, which means nothing, as if it were contiguous."""
    shape, st = t.shape, t.stride()
    if 1 in shape:
        st, full = list(st), 1
        for i in range(len(shape) - 1, -1, -1):
            if shape[i] == 1:
                st[i] = full
            full = shape[i] * st[i]
    return st


class PagePool:
    """Free pages and the block table of up to ``block_table.shape[0]`` requests.

    ``free`` is the stack's memory, int32 [num_pages]; ``free_count`` (int32 [1], on the device) its
    height.  Without them the pool starts full, pages 0, 1, ... given out in that order.  With ``free`` alone
    its own count starts at 0, none free: for programs that hand a count to each call."""

    def __init__(self, num_pages: int, page_size: int, block_table, free=None, free_count=None):
        dev = block_table.device
        if free is None:
            free = torch.arange(num_pages - 1, -1, -1, dtype=_I32, device=dev)
            free_count = torch.full((1,), num_pages, dtype=_I32, device=dev) if free_count is None else free_count
        self.num_pages, self.page_size = num_pages, page_size
        self.block_table, self._table = block_table, _table(block_table)
        self.max_requests, self.max_pages = block_table.shape
        _need(free.dtype is _I32 and free.is_contiguous() and free.numel() == num_pages and free.device == dev,
              "free: contiguous int32 [num_pages] beside the block table")
        self.free = free
        state = torch.zeros(2, dtype=_I32, device=dev)
        self.free_count = state[:1] if free_count is None else free_count
        self.device_status = state[1:]
        self._call = (page_size, num_pages, free.data_ptr(), self._table, self.max_requests, self.max_pages,
                      self.device_status.data_ptr(), dev.index or 0)
        self._lib = _bind()

    def tables(self, lens, new_lens, T: int, *, kv_lens=None, cu=None, slots=None, positions=None, granted=None,
               free_count=None, free_count_out=None, stream=None):
        """Pages for the new tokens, and where each goes: (kv_lens, cu, slots, positions, granted).
        T: rows of the new tokens' tensors.  By default the pool's count is updated in place and the
        outputs are new tensors; ``kv_lens=lens`` updates the lengths in place."""
        if kv_lens is None or cu is None or slots is None or positions is None or granted is None:
            B = lens.numel()
            e = lambda t, n: torch.empty(n, dtype=_I32, device=lens.device) if t is None else t
            with _on(stream):
                kv_lens, cu, slots, positions, granted = e(kv_lens, B), e(cu, B + 1), e(slots, T), e(positions, T), e(granted, B)
        if free_count is None:
            free_count = self.free_count
        rc = self._lib.tables(*self._call, None if stream is None else stream.cuda_stream, lens, new_lens, T, kv_lens, cu, slots,
                              positions, granted, free_count, free_count if free_count_out is None else free_count_out)
        if rc:
            raise kvev.KvevError(rc, "kvev_paged_tables")
        return kv_lens, cu, slots, positions, granted

    def release(self, lens, done, *, lens_out=None, free_count=None, free_count_out=None, stream=None):
        """The pages of requests with done != 0 go back; returns the lengths, 0 for those (by default
        ``lens`` itself and the pool's count are updated in place)."""
        if lens_out is None:
            lens_out = lens
        if free_count is None:
            free_count = self.free_count
        rc = self._lib.release(*self._call, None if stream is None else stream.cuda_stream, lens, done, lens_out, free_count,
                               free_count if free_count_out is None else free_count_out)
        if rc:
            raise kvev.KvevError(rc, "kvev_paged_release")
        return lens_out


class PagedCache:
    """One layer's pages: K and V viewed as [num_pages][page_size][H_kv][d] (bf16 or fp16, equal strides, d
    contiguous; a transposed view of [num_pages][H_kv][page_size][d] will do), under a block table."""

    def __init__(self, K, V, block_table):
        _need(K.dim() == 4 and K.shape == V.shape and _strides(K) == _strides(V) and K.stride(3) == V.stride(3) == 1,
              "K, V: [num_pages][page_size][H_kv][d] of equal strides, d contiguous")
        _need(K.dtype in _DTYPES and K.dtype is V.dtype, "K, V: bfloat16 or float16")
        _need(K.is_cuda and V.is_cuda, "K, V: CUDA tensors")
        self.K, self.V, self.block_table, self._table = K, V, block_table, _table(block_table)
        self.max_requests, self.max_pages = block_table.shape
        pages, page, self.H_kv, self.d = K.shape
        self.dtype = K.dtype
        self.desc = kvev.PagedCacheDesc(K.data_ptr(), V.data_ptr(), *_strides(K)[:3], pages, page, self.H_kv, self.d,
                                        _DTYPES[K.dtype])
        self._device = K.device.index or 0
        _need(block_table.device == K.device == V.device, "K, V and block_table: one GPU")
        self.device_status = torch.zeros(1, dtype=_I32, device=K.device)
        self._call = (C.addressof(self.desc), self._table, self.max_requests, self.max_pages, self.device_status.data_ptr(),
                      self._device)
        self._lib = _bind()

    @classmethod
    def empty(cls, num_pages, page_size, H_kv, d, block_table, dtype=torch.bfloat16, heads_first=False):
        """A layer's pages in new memory: [page][H_kv][d] each, or [H_kv][page][d] with heads_first."""
        shape = (2, num_pages, H_kv, page_size, d) if heads_first else (2, num_pages, page_size, H_kv, d)
        x = torch.empty(shape, dtype=dtype, device=block_table.device)
        K, V = x.transpose(2, 3) if heads_first else x
        return cls(K, V, block_table)

    def write(self, k, v, slots, stream=None):
        """k, v [T][H_kv][d] of equal strides into the slots (int32 [T], negative: left out)."""
        rc = self._lib.write(*self._call, None if stream is None else stream.cuda_stream, k, v, slots)
        if rc:
            raise kvev.KvevError(rc, "kvev_paged_write")

    def workspace(self, H_q: int | None = None, stream=None):
        """The scratch that attention calls on a stream use, made at the first of them or here: all layers' calls
        on a stream share one, whatever their heads (H_q is not needed).  While the stream is being captured, the
        capture's own."""
        return _workspace(self._device, *self._lib.stream(self._device, None if stream is None else stream.cuda_stream))[2]

    def attention(self, q, cu, kv_lens, *, scale=0.0, window=0, out=None, lse=None, workspace=None, stream=None):
        """Causal attention of the new tokens' queries q [T][H_q][d] (request s: rows cu[s]..cu[s+1], the last of
        its kv_lens[s] positions).  lse: fp32 [T][H_q] for the rows' log-sum-exp.  Returns out.

        Graphs captured with ``torch.cuda.graph`` may be replayed in any order, beside one another and beside other
        calls (graphs that share a memory pool one after another, as torch has it).  A graph captured by other means needs a ``workspace`` that it keeps
        (``kvev.kvev_paged_attention_workspace`` bytes, 256-byte aligned, the first ``kvev.PAGED_SYNC_BYTES`` zero
        before its first use)."""
        if out is None:
            with _on(stream):
                out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        at, capture = self._lib.stream(self._device, None if stream is None else stream.cuda_stream)
        ws = _workspace(self._device, at, capture) if workspace is None else _given(workspace, self._device)
        rc = self._lib.attention(*self._call, at, q, cu, kv_lens, out, lse, scale, window, ws[0], ws[1])
        if rc:
            raise kvev.KvevError(rc, "kvev_paged_attention")
        return out

    def gather(self, lens, out_K, out_V, stream=None):
        """The first lens[s] tokens of every request into out_K, out_V [B][H_kv][S_cap][d] (contiguous)."""
        rc = self._lib.gather(*self._call, None if stream is None else stream.cuda_stream, lens, out_K, out_V)
        if rc:
            raise kvev.KvevError(rc, "kvev_paged_gather")

    def status(self) -> int:
        """Waits for the GPU, whatever the calls' streams, then reads and clears the device status word (0: every
        call so far was in order)."""
        torch.cuda.synchronize(self._device)
        v = int(self.device_status.item())
        if v:
            self.device_status.zero_()
            if v & 1:  # a wait ran out: the pieces counted so far would be counted again (a graph zeroes its own)
                for (device, _), ws in _workspaces.items():
                    if device == self._device:
                        ws[2][:kvev.PAGED_SYNC_BYTES].zero_()
            torch.cuda.synchronize(self._device)
        return v
