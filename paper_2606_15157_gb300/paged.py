"""Paged caches with torch tensors as device memory, over the ``kvev_paged_*`` entry points.

:class:`PagePool` keeps a stack of free pages and the requests' block table: ``tables`` and ``release``
are a scheduler step.  :class:`PagedCache` is one layer's pages under such a table: ``write`` the new
tokens' rows, ``attention`` over them, ``gather`` whole prompts for ``Plan.evict_prefill``.  Lengths,
tables and slots stay on the device throughout.  Argument checks raise ``ValueError`` (shapes, types)
or ``KvevError`` (what the library refuses).
"""
from __future__ import annotations

import ctypes as C

import torch

from . import kvev

_DTYPES = {torch.bfloat16: kvev.BF16, torch.float16: kvev.FP16}


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _int32(t, n: int | None, what: str):
    """Device pointer of a contiguous int32 CUDA tensor of n elements (any number: None)."""
    if t.dtype is not torch.int32 or not t.is_cuda or not t.is_contiguous() or (n is not None and t.numel() != n):
        raise ValueError(f"{what}: a contiguous int32 CUDA tensor" + (f" of {n} elements" if n is not None else ""))
    return t.data_ptr()


def _stride(t, i: int) -> int:
    """Element stride of dimension i (that of a dimension of one element means nothing: the row size)."""
    return t.stride(i) if t.shape[i] != 1 else t.shape[-1] * (t.shape[-2] if i < t.dim() - 2 else 1)


def _same_layout(a, b) -> bool:
    return a.shape == b.shape and all(_stride(a, i) == _stride(b, i) for i in range(a.dim() - 1))


def _stream(stream) -> int:
    return torch.cuda.current_stream().cuda_stream if stream is None else stream.cuda_stream


def _table(block_table):
    _need(block_table.dim() == 2, "block_table: [requests][pages]")
    return _int32(block_table, None, "block_table")


class PagePool:
    """Free pages and the block table of up to ``block_table.shape[0]`` requests.

    ``free`` is the stack's memory, int32 [num_pages]; ``free_count`` (int32 [1], on the device) its
    height.  Without them the pool starts full, pages 0, 1, ... given out in that order."""

    def __init__(self, num_pages: int, page_size: int, block_table, free=None, free_count=None):
        dev = block_table.device
        if free is None:
            free = torch.arange(num_pages - 1, -1, -1, dtype=torch.int32, device=dev)
            free_count = torch.full((1,), num_pages, dtype=torch.int32, device=dev) if free_count is None else free_count
        self.num_pages, self.page_size = num_pages, page_size
        self.block_table, self._table = block_table, _table(block_table)
        self.free, self._free = free, _int32(free, num_pages, "free")
        self.free_count = torch.zeros(1, dtype=torch.int32, device=dev) if free_count is None else free_count
        self.device_status = torch.zeros(1, dtype=torch.int32, device=dev)

    def tables(self, lens, new_lens, T: int, *, kv_lens=None, cu=None, slots=None, positions=None, granted=None,
               free_count=None, free_count_out=None, stream=None):
        """Pages for the new tokens, and where each goes: (kv_lens, cu, slots, positions, granted).
        T: rows of the new tokens' tensors.  By default the pool's count is updated in place and the
        outputs are new tensors; ``kv_lens=lens`` updates the lengths in place."""
        B, dev = lens.numel(), lens.device
        _need(B <= self.block_table.shape[0], "more requests than the block table has rows")
        e = lambda t, n: torch.empty(n, dtype=torch.int32, device=dev) if t is None else t
        kv_lens, cu, slots, positions, granted = e(kv_lens, B), e(cu, B + 1), e(slots, T), e(positions, T), e(granted, B)
        free_count = self.free_count if free_count is None else free_count
        free_count_out = free_count if free_count_out is None else free_count_out
        kvev._check(kvev.kvev_paged_tables(
            _int32(lens, B, "lens"), _int32(new_lens, B, "new_lens"), B, self.page_size, self.num_pages, self._free,
            _int32(free_count, 1, "free_count"), self._table, self.block_table.shape[1], T, _int32(kv_lens, B, "kv_lens"),
            _int32(cu, B + 1, "cu"), _int32(slots, T, "slots"), _int32(positions, T, "positions"),
            _int32(granted, B, "granted"), _int32(free_count_out, 1, "free_count_out"), self.device_status.data_ptr(),
            _stream(stream)), "kvev_paged_tables")
        return kv_lens, cu, slots, positions, granted

    def release(self, lens, done, *, lens_out=None, free_count=None, free_count_out=None, stream=None):
        """The pages of requests with done != 0 go back; returns the lengths, 0 for those (by default
        ``lens`` itself and the pool's count are updated in place)."""
        B = lens.numel()
        _need(B <= self.block_table.shape[0], "more requests than the block table has rows")
        lens_out = lens if lens_out is None else lens_out
        free_count = self.free_count if free_count is None else free_count
        free_count_out = free_count if free_count_out is None else free_count_out
        kvev._check(kvev.kvev_paged_release(
            _int32(lens, B, "lens"), _int32(done, B, "done"), B, self.page_size, self.num_pages, self._table,
            self.block_table.shape[1], self._free, _int32(free_count, 1, "free_count"), _int32(lens_out, B, "lens_out"),
            _int32(free_count_out, 1, "free_count_out"), self.device_status.data_ptr(), _stream(stream)),
            "kvev_paged_release")
        return lens_out


class PagedCache:
    """One layer's pages: K and V viewed as [num_pages][page_size][H_kv][d] (bf16 or fp16, equal strides, d
    contiguous; a transposed view of [num_pages][H_kv][page_size][d] will do), under a block table."""

    def __init__(self, K, V, block_table):
        _need(K.dim() == 4 and V.dim() == 4 and _same_layout(K, V) and K.stride(3) == V.stride(3) == 1,
              "K, V: [num_pages][page_size][H_kv][d] of equal strides, d contiguous")
        _need(K.dtype in _DTYPES and K.dtype == V.dtype, "K, V: bfloat16 or float16")
        _need(K.is_cuda and V.is_cuda, "K, V: CUDA tensors")
        self.K, self.V, self.block_table, self._table = K, V, block_table, _table(block_table)
        pages, page, self.H_kv, self.d = K.shape
        self.desc = kvev.PagedCacheDesc(K.data_ptr(), V.data_ptr(), _stride(K, 0), _stride(K, 1), _stride(K, 2), pages, page,
                                        self.H_kv, self.d, _DTYPES[K.dtype])
        self._desc = C.addressof(self.desc)
        self.device_status = torch.zeros(1, dtype=torch.int32, device=K.device)
        self._status = self.device_status.data_ptr()
        self._workspaces = {}

    @classmethod
    def empty(cls, num_pages, page_size, H_kv, d, block_table, dtype=torch.bfloat16, heads_first=False):
        """A layer's pages in new memory: [page][H_kv][d] each, or [H_kv][page][d] with heads_first."""
        shape = (2, num_pages, H_kv, page_size, d) if heads_first else (2, num_pages, page_size, H_kv, d)
        x = torch.empty(shape, dtype=dtype, device=block_table.device)
        K, V = x.transpose(2, 3) if heads_first else x
        return cls(K, V, block_table)

    def _rows(self, t, H, what):
        _need(t.dim() == 3 and t.shape[1] == H and t.shape[2] == self.d and t.dtype is self.K.dtype and t.stride(2) == 1,
              f"{what}: [tokens][{H}][{self.d}] of the cache's type, d contiguous")
        return t.data_ptr()

    def write(self, k, v, slots, stream=None):
        """k, v [T][H_kv][d] of equal strides into the slots (int32 [T], negative: left out)."""
        T = k.shape[0]
        _need(k.dim() == 3 and _same_layout(k, v), "k, v: equal shapes and strides")
        kvev._check(kvev.kvev_paged_write(self._desc, self._rows(k, self.H_kv, "k"), self._rows(v, self.H_kv, "v"),
                                          _stride(k, 0), _stride(k, 1), _int32(slots, T, "slots"), T, self._status,
                                          _stream(stream)), "kvev_paged_write")

    def workspace(self, H_q, stream=None):
        """The scratch of attention calls on a stream (one per stream: overlapping calls may not share it)."""
        at = _stream(stream)
        ws = self._workspaces.get((H_q, at))
        if ws is None:
            n = kvev.kvev_paged_attention_workspace(H_q, self.H_kv, self.d)
            ws = self._workspaces[H_q, at] = torch.zeros(n, dtype=torch.uint8, device=self.K.device)
        return ws

    def attention(self, q, cu, kv_lens, *, scale=0.0, window=0, out=None, lse=None, workspace=None, stream=None):
        """Causal attention of the new tokens' queries q [T][H_q][d] (request s: rows cu[s]..cu[s+1], the last of
        its kv_lens[s] positions).  lse: fp32 [T][H_q] for the rows' log-sum-exp.  Returns out."""
        T, H_q = q.shape[0], q.shape[1]
        B = kv_lens.numel()
        _need(B <= self.block_table.shape[0], "more requests than the block table has rows")
        out = torch.empty((T, H_q, self.d), dtype=q.dtype, device=q.device) if out is None else out
        _need(out.shape == q.shape, "out: q's shape")
        _need(lse is None or (lse.dtype is torch.float32 and lse.is_contiguous() and lse.shape == (T, H_q)),
              "lse: contiguous float32 [T][H_q]")
        ws = self.workspace(H_q, stream) if workspace is None else workspace
        kvev._check(kvev.kvev_paged_attention(
            self._desc, self._rows(q, H_q, "q"), _stride(q, 0), _stride(q, 1), _int32(cu, B + 1, "cu"),
            _int32(kv_lens, B, "kv_lens"), self._table, self.block_table.shape[1], B, T, H_q, scale, window,
            self._rows(out, H_q, "out"), _stride(out, 0), _stride(out, 1), None if lse is None else lse.data_ptr(),
            ws.data_ptr(), ws.numel(), self._status, _stream(stream)), "kvev_paged_attention")
        return out

    def gather(self, lens, out_K, out_V, stream=None):
        """The first lens[s] tokens of every request into out_K, out_V [B][H_kv][S_cap][d] (contiguous)."""
        B, S_cap = lens.numel(), out_K.shape[2]
        for t in (out_K, out_V):
            _need(t.shape == (B, self.H_kv, S_cap, self.d) and t.is_contiguous() and t.dtype is self.K.dtype,
                  f"out_K, out_V: contiguous [{B}][{self.H_kv}][S_cap][{self.d}] of the cache's type")
        _need(B <= self.block_table.shape[0], "more requests than the block table has rows")
        kvev._check(kvev.kvev_paged_gather(self._desc, self._table, self.block_table.shape[1], _int32(lens, B, "lens"), B,
                                           S_cap, out_K.data_ptr(), out_V.data_ptr(), self._status, _stream(stream)),
                    "kvev_paged_gather")

    def status(self) -> int:
        """Synchronises, reads and clears the device status word (0: every call so far was in order)."""
        v = int(self.device_status.item())
        if v:
            self.device_status.zero_()
        return v
