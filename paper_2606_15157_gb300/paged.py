"""Paged caches with torch tensors as device memory, over the ``kvev_paged_*`` entry points.

:class:`PagePool` keeps a stack of free pages and the requests' block table: ``tables`` and ``release``
are a scheduler step.  :class:`PagedCache` is one layer's pages under such a table: ``write`` the new
tokens' rows, ``attention`` over them, ``gather`` whole prompts for ``Plan.evict_prefill``.  Lengths,
tables and slots stay on the device throughout.  Argument checks raise ``ValueError`` (shapes, types)
or ``KvevError`` (what the library refuses).

These are calls of a few microseconds on the device, made for every layer of every token: the checks
here are a handful of attribute reads, the stream is read as a number.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import kvev

_DTYPES = {torch.bfloat16: kvev.BF16, torch.float16: kvev.FP16}
_I32 = torch.int32


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _int32(t, n: int, what: str) -> int:
    """Device pointer of a contiguous int32 tensor of n elements."""
    if t.dtype is not _I32 or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{what}: a contiguous int32 tensor of {n} elements")
    return t.data_ptr()


# The current stream of a device as a number; torch.cuda.current_stream() makes an object first (2.8 us).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda device: torch.cuda.current_stream(device).cuda_stream)


# Scratch of the attention calls on a stream, (device, stream) -> (pointer, bytes, tensor): calls on a stream
# follow one another, whatever layer they are for, so they share it.
_workspaces: dict = {}


def _workspace(device: int, stream: int):
    ws = _workspaces.get((device, stream))
    if ws is None:
        n = kvev.kvev_paged_attention_workspace(1, 1, 128)  # what the largest call needs
        with torch.cuda.device(device), torch.cuda.stream(torch.cuda.ExternalStream(stream, device=device)):
            t = torch.empty(n, dtype=torch.uint8, device="cuda")
            t[:kvev.PAGED_SYNC_BYTES].zero_()
        ws = _workspaces[device, stream] = (t.data_ptr(), n, t)
    return ws


def _table(block_table) -> int:
    _need(block_table.dim() == 2 and block_table.is_cuda, "block_table: int32 [requests][pages] on a GPU")
    return _int32(block_table, block_table.numel(), "block_table")


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
    height.  Without them the pool starts full, pages 0, 1, ... given out in that order."""

    def __init__(self, num_pages: int, page_size: int, block_table, free=None, free_count=None):
        dev = block_table.device
        if free is None:
            free = torch.arange(num_pages - 1, -1, -1, dtype=_I32, device=dev)
            free_count = torch.full((1,), num_pages, dtype=_I32, device=dev) if free_count is None else free_count
        self.num_pages, self.page_size = num_pages, page_size
        self.block_table, self._table = block_table, _table(block_table)
        self.max_requests, self.max_pages = block_table.shape
        self.free, self._free = free, _int32(free, num_pages, "free")
        state = torch.zeros(2, dtype=_I32, device=dev)
        self.free_count = state[:1] if free_count is None else free_count
        self.device_status = state[1:]
        self._status, self._device = self.device_status.data_ptr(), dev.index or 0

    def tables(self, lens, new_lens, T: int, *, kv_lens=None, cu=None, slots=None, positions=None, granted=None,
               free_count=None, free_count_out=None, stream=None):
        """Pages for the new tokens, and where each goes: (kv_lens, cu, slots, positions, granted).
        T: rows of the new tokens' tensors.  By default the pool's count is updated in place and the
        outputs are new tensors; ``kv_lens=lens`` updates the lengths in place."""
        B = lens.numel()
        if B > self.max_requests:
            raise ValueError("more requests than the block table has rows")
        if kv_lens is None or cu is None or slots is None or positions is None or granted is None:
            e = lambda t, n: torch.empty(n, dtype=_I32, device=lens.device) if t is None else t
            kv_lens, cu, slots, positions, granted = e(kv_lens, B), e(cu, B + 1), e(slots, T), e(positions, T), e(granted, B)
        if free_count is None:
            free_count = self.free_count
        if free_count_out is None:
            free_count_out = free_count
        rc = kvev.load().kvev_paged_tables(
            _int32(lens, B, "lens"), _int32(new_lens, B, "new_lens"), B, self.page_size, self.num_pages, self._free,
            _int32(free_count, 1, "free_count"), self._table, self.max_pages, T, _int32(kv_lens, B, "kv_lens"),
            _int32(cu, B + 1, "cu"), _int32(slots, T, "slots"), _int32(positions, T, "positions"),
            _int32(granted, B, "granted"), _int32(free_count_out, 1, "free_count_out"), self._status,
            _raw_stream(self._device) if stream is None else stream.cuda_stream)
        if rc:
            raise kvev.KvevError(rc, "kvev_paged_tables")
        return kv_lens, cu, slots, positions, granted

    def release(self, lens, done, *, lens_out=None, free_count=None, free_count_out=None, stream=None):
        """The pages of requests with done != 0 go back; returns the lengths, 0 for those (by default
        ``lens`` itself and the pool's count are updated in place)."""
        B = lens.numel()
        if B > self.max_requests:
            raise ValueError("more requests than the block table has rows")
        if lens_out is None:
            lens_out = lens
        if free_count is None:
            free_count = self.free_count
        if free_count_out is None:
            free_count_out = free_count
        rc = kvev.load().kvev_paged_release(
            _int32(lens, B, "lens"), _int32(done, B, "done"), B, self.page_size, self.num_pages, self._table, self.max_pages,
            self._free, _int32(free_count, 1, "free_count"), _int32(lens_out, B, "lens_out"),
            _int32(free_count_out, 1, "free_count_out"), self._status,
            _raw_stream(self._device) if stream is None else stream.cuda_stream)
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
        self._desc, self._device = C.addressof(self.desc), K.device.index or 0
        self.device_status = torch.zeros(1, dtype=_I32, device=K.device)
        self._status = self.device_status.data_ptr()

    @classmethod
    def empty(cls, num_pages, page_size, H_kv, d, block_table, dtype=torch.bfloat16, heads_first=False):
        """A layer's pages in new memory: [page][H_kv][d] each, or [H_kv][page][d] with heads_first."""
        shape = (2, num_pages, H_kv, page_size, d) if heads_first else (2, num_pages, page_size, H_kv, d)
        x = torch.empty(shape, dtype=dtype, device=block_table.device)
        K, V = x.transpose(2, 3) if heads_first else x
        return cls(K, V, block_table)

    def _rows(self, t, shape, what) -> tuple:
        """(token stride, head stride) of [T][H][d] rows of the cache's type."""
        if len(shape) != 3 or t.dtype is not self.dtype or shape[2] != self.d:
            raise ValueError(f"{what}: [tokens][heads][{self.d}] of the cache's type")
        st = _strides(t)
        if st[2] != 1:
            raise ValueError(f"{what}: the last dimension is contiguous")
        return st

    def write(self, k, v, slots, stream=None):
        """k, v [T][H_kv][d] of equal strides into the slots (int32 [T], negative: left out)."""
        shape = k.shape
        st = self._rows(k, shape, "k")
        if shape[1] != self.H_kv or v.shape != shape or self._rows(v, shape, "v") != st:
            raise ValueError(f"k, v: [tokens][{self.H_kv}][{self.d}] of equal strides")
        rc = kvev.load().kvev_paged_write(
            self._desc, k.data_ptr(), v.data_ptr(), st[0], st[1], _int32(slots, shape[0], "slots"), shape[0], self._status,
            _raw_stream(self._device) if stream is None else stream.cuda_stream)
        if rc:
            raise kvev.KvevError(rc, "kvev_paged_write")

    def workspace(self, H_q: int | None = None, stream=None):
        """The scratch that attention calls on a stream use, made at the first of them (before a capture of
        the stream, let one call or this one make it): all layers' calls on a stream share one."""
        return _workspace(self._device, _raw_stream(self._device) if stream is None else stream.cuda_stream)[2]

    def attention(self, q, cu, kv_lens, *, scale=0.0, window=0, out=None, lse=None, workspace=None, stream=None):
        """Causal attention of the new tokens' queries q [T][H_q][d] (request s: rows cu[s]..cu[s+1], the last of
        its kv_lens[s] positions).  lse: fp32 [T][H_q] for the rows' log-sum-exp.  Returns out."""
        shape = q.shape
        sq = self._rows(q, shape, "q")
        T, H_q, _ = shape
        B = kv_lens.numel()
        if B > self.max_requests:
            raise ValueError("more requests than the block table has rows")
        if out is None:
            out = torch.empty(shape, dtype=q.dtype, device=q.device)
        elif out.shape != shape:
            raise ValueError("out: q's shape")
        so = self._rows(out, shape, "out")
        if lse is None:
            lse_ptr = None
        else:
            if lse.dtype is not torch.float32 or not lse.is_contiguous() or lse.shape != shape[:2]:
                raise ValueError("lse: contiguous float32 [T][H_q]")
            lse_ptr = lse.data_ptr()
        at = _raw_stream(self._device) if stream is None else stream.cuda_stream
        ws = _workspace(self._device, at) if workspace is None else (workspace.data_ptr(), workspace.numel())
        rc = kvev.load().kvev_paged_attention(
            self._desc, q.data_ptr(), sq[0], sq[1], _int32(cu, B + 1, "cu"), _int32(kv_lens, B, "kv_lens"), self._table,
            self.max_pages, B, T, H_q, scale, window, out.data_ptr(), so[0], so[1], lse_ptr, ws[0], ws[1], self._status, at)
        if rc:
            raise kvev.KvevError(rc, "kvev_paged_attention")
        return out

    def gather(self, lens, out_K, out_V, stream=None):
        """The first lens[s] tokens of every request into out_K, out_V [B][H_kv][S_cap][d] (contiguous)."""
        B, shape = lens.numel(), out_K.shape
        if (len(shape) != 4 or shape[0] != B or shape[1] != self.H_kv or shape[3] != self.d or out_V.shape != shape
                or out_K.dtype is not self.dtype or out_V.dtype is not self.dtype
                or not out_K.is_contiguous() or not out_V.is_contiguous()):
            raise ValueError(f"out_K, out_V: contiguous [{B}][{self.H_kv}][S_cap][{self.d}] of the cache's type")
        if B > self.max_requests:
            raise ValueError("more requests than the block table has rows")
        rc = kvev.load().kvev_paged_gather(
            self._desc, self._table, self.max_pages, _int32(lens, B, "lens"), B, shape[2], out_K.data_ptr(), out_V.data_ptr(),
            self._status, _raw_stream(self._device) if stream is None else stream.cuda_stream)
        if rc:
            raise kvev.KvevError(rc, "kvev_paged_gather")

    def status(self) -> int:
        """Synchronises, reads and clears the device status word (0: every call so far was in order)."""
        v = int(self.device_status.item())
        if v:
            self.device_status.zero_()
        return v
