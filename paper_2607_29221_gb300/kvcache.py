"""Paged key/value cache of a decode step: append, attention, eviction.

Attention stays on the trusted side (Sec. 3.2 "Local attention computation"),
and so does its cache.  ``PagedCache`` is a handle on a pool of pages that the
caller allocated (or ``PagedCache.empty`` does); every method is one library
call on the current stream:

  rope  = Rope(128, base=500000.0, device="cuda")
  cache = PagedCache.empty(pages, kv_heads, page_size, head_dim, table, torch.bfloat16)
  q     = cache.append(qkv, heads, seq, slot, index, rope=rope, pos=pos)
  out   = cache.attend(q, lens, max_len)
  lens  = cache.evict(lens, max_len, keep, recent_from=recent_from)
  k, v  = cache.rows(seq, slot)

Keys and values are held in float32, bfloat16, float16 or 4 bits (``INT4``: uint8
pools, rows of codes with a step and a base for every 32 channels).  ``HeadNorm``
norms the query and key heads on the way in.

Arguments are tensors on the cache's device.  Scratch is kept for the last few
streams of each host thread until the thread ends (5 us a call to allocate it
anew); calls that are captured into a graph get scratch of their own, since the
graph may run beside anything.
``PageTable`` is the host's account of which page belongs to whom.
"""
from __future__ import annotations

import ctypes
import threading

import torch

from . import mosaic as M

_STREAMS = 4   # streams of a host thread whose scratch is kept
INT4 = torch.uint8   # the element type of 4-bit pools: bytes of packed rows
_TYPES = {torch.float32: M.KV_F32, torch.bfloat16: M.KV_BF16, torch.float16: M.KV_F16, INT4: M.KV_Q4}


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _int32(t, name: str, n: int, index: int) -> None:
    if t.dtype is not torch.int32 or t.get_device() != index or t.dim() != 1 or t.numel() != n or (
            n > 1 and t.stride(0) != 1):
        raise ValueError(f"{name}: a contiguous int32 tensor of {n} elements on the cache's device is needed")


def _row_stride(t, width: int, name: str) -> int:
    """The distance of t's rows, at least ``width``: rows that share memory
    (expanded or overlapping views) have no leading dimension."""
    stride = t.stride(0)
    if stride >= width:
        return stride
    if t.shape[0] > 1:
        raise ValueError(f"{name}: rows must not share memory (an expanded view needs .contiguous())")
    return width


def _rows(t, name: str, n: int, heads: int, dim: int, index: int) -> int:
    """The row stride of a float32 n x heads x dim tensor whose rows are contiguous."""
    st = t.stride() if t.dim() == 3 else (0, 0, 0)
    if (t.dtype is not torch.float32 or t.get_device() != index or t.shape != (n, heads, dim) or st[2] != 1
            or (heads > 1 and st[1] != dim)):
        raise ValueError(f"{name}: float32, {n} x {heads} x {dim}, rows contiguous, on the cache's device")
    return _row_stride(t, heads * dim, name)


class Rope:
    """Rotary frequencies of ``rot_dim`` channels.  ``sections`` gives the
    number of channel pairs that each of up to four position axes turns (text:
    one axis; images and video: time, height, width), in order."""

    def __init__(self, rot_dim: int, base: float = 10000.0, sections=None, interleaved: bool = False,
                 device="cuda"):
        sections = [rot_dim // 2] if sections is None else [int(n) for n in sections]
        _need(rot_dim % 8 == 0 and rot_dim > 0, "rot_dim: a positive multiple of 8")
        _need(1 <= len(sections) <= 4 and min(sections) >= 0 and sum(sections) == rot_dim // 2,
              "sections: one to four counts that add up to rot_dim / 2")
        self.rot_dim, self.axes, self.interleaved = rot_dim, len(sections), bool(interleaved)
        self.turns = torch.from_numpy(M.mosaic_rope_turns(rot_dim, base).view("int64")).to(device)
        self.axis = torch.repeat_interleave(torch.arange(self.axes, dtype=torch.int32),
                                            torch.tensor(sections)).to(device)
        self._turns, self._axis = self.turns.data_ptr(), self.axis.data_ptr()

    def at(self, pos: torch.Tensor) -> M.mosaic_rope:
        """The rotation of tokens at ``pos`` (axes x tokens, or tokens for one axis)."""
        pos = pos[None] if pos.dim() == 1 else pos
        if (pos.dtype is not torch.int32 or pos.dim() != 2 or pos.shape[0] != self.axes
                or (pos.shape[1] > 1 and pos.stride(1) != 1) or pos.get_device() != self.turns.get_device()):
            raise ValueError(f"pos: int32, {self.axes} x tokens, rows contiguous, on the rope's device")
        return M.mosaic_rope(self.rot_dim, self.interleaved, self.axes, self._turns, self._axis, pos.data_ptr(),
                             _row_stride(pos, pos.shape[1], "pos"))


def row_bytes(head_dim: int) -> int:
    """Bytes of a row of a 4-bit cache: the last axis of its uint8 pools."""
    n = M.mosaic_kv_row_bytes(M.KV_Q4, head_dim)
    _need(n > 0, "head_dim: a multiple of 32 up to 256 for 4-bit caches")
    return n


class HeadNorm:
    """Norms of query and key heads: x / sqrt(mean(x^2) + eps) over a head, times
    ``q_gain`` or ``k_gain`` (float32, a value a channel, the same for all heads;
    None: 1).  It keeps the gains alive."""

    def __init__(self, head_dim: int, eps: float = 1e-6, q_gain=None, k_gain=None):
        _need(eps >= 0.0, "eps: not negative")
        for g, name in ((q_gain, "q_gain"), (k_gain, "k_gain")):
            _need(g is None or (g.dtype is torch.float32 and g.shape == (head_dim,)
                                and (head_dim == 1 or g.stride(0) == 1)),
                  f"{name}: a contiguous float32 tensor of head_dim values")
        self.head_dim, self.q_gain, self.k_gain = head_dim, q_gain, k_gain
        self._devices = {g.get_device() for g in (q_gain, k_gain) if g is not None}
        self._c = M.mosaic_head_norm(eps, *(None if g is None else g.data_ptr() for g in (q_gain, k_gain)))
        self._ref = ctypes.byref(self._c)

    def on(self, head_dim: int, index: int):
        """The library's argument for a cache of head_dim channels on device ``index``."""
        _need(head_dim == self.head_dim, "norm: of another head_dim than the cache")
        _need(self._devices <= {index}, "norm: gains on another device than the cache")
        return self._ref


class PagedCache:
    """Handle on a paged cache.  k, v: pages x kv_heads x page_size x head_dim
    views (float32, bfloat16 or float16; equal strides, channels contiguous; uint8
    with row_bytes(head_dim) instead of head_dim: 4 bits),
    table: seqs x columns int32 page ids; position (int32) and weight
    (float32): contiguous pages x kv_heads x page_size, or None."""

    def __init__(self, k, v, table, position=None, weight=None):
        _need(k.dim() == 4 and k.shape == v.shape and k.stride() == v.stride() and k.dtype == v.dtype
              and k.dtype in _TYPES and k.stride(3) == 1 and k.is_cuda and v.device == k.device,
              "k and v: CUDA tensors of one type and shape (4 axes), equal strides, channels contiguous")
        pages, kv_heads, page, dim = k.shape
        if k.dtype is INT4:
            dim = next((d for d in range(32, 257, 32) if row_bytes(d) == dim), 0)
            _need(dim > 0, "k and v: rows of row_bytes(head_dim) bytes for 4 bits")
        _need(table.dtype == torch.int32 and table.dim() == 2 and table.device == k.device
              and (table.shape[1] <= 1 or table.stride(1) == 1), "table: int32, seqs x columns, rows contiguous")
        for t, dt, name in ((position, torch.int32, "position"), (weight, torch.float32, "weight")):
            _need(t is None or (t.dtype == dt and t.shape == k.shape[:3] and t.is_contiguous()
                                and t.device == k.device),
                  f"{name}: contiguous {dt}, pages x kv_heads x page_size, on the cache's device")
        self.k, self.v, self.table, self.position, self.weight = k, v, table, position, weight
        self.device, self.kv_heads, self.head_dim, self.seqs = k.device, kv_heads, dim, table.shape[0]
        self._index = k.get_device()
        ptr = [None if t is None else t.data_ptr() for t in (k, v, table, position, weight)]
        self._c = M.mosaic_kv_cache(_TYPES[k.dtype], kv_heads, dim, page, pages, table.shape[0], table.shape[1],
                                    _row_stride(table, table.shape[1], "table"), k.stride(0), k.stride(1), k.stride(2),
                                    *ptr)
        self._ref = ctypes.byref(self._c)
        lib = M.lib()
        self._calls = lib.mosaic_kv_append, lib.mosaic_kv_attention, lib.mosaic_kv_evict
        self._ws, self._scratch = {}, threading.local()

    @classmethod
    def empty(cls, pages: int, kv_heads: int, page_size: int, head_dim: int, table, dtype=torch.bfloat16,
              weights: bool = True):
        """A new pool (head-major pages), with positions, and weights unless turned off."""
        shape, dev = (pages, kv_heads, page_size), table.device
        row = row_bytes(head_dim) if dtype is INT4 else head_dim
        k, v = (torch.zeros(*shape, row, dtype=dtype, device=dev) for _ in range(2))
        return cls(k, v, table, torch.zeros(shape, dtype=torch.int32, device=dev),
                   torch.zeros(shape, dtype=torch.float32, device=dev) if weights else None)

    def _bytes(self, key, size, *args) -> int:
        n = self._ws.get(key)
        if n is None:
            if len(self._ws) > 256:   # max_len grows with every step of a loop
                self._ws.clear()
            n = self._ws[key] = size(self._ref, *args)
        return n

    def _stream(self) -> int:
        """The current stream, which has to be one of the cache's device."""
        if torch.cuda.current_device() != self._index:
            raise ValueError("the cache's device is not the current one")
        return M._stream(None)

    def _workspace(self, need: int, stream: int):
        if not need:
            return None
        if torch.cuda.is_current_stream_capturing():
            return torch.empty(need, dtype=torch.uint8, device=self.device)
        held = self._scratch.__dict__   # the host thread's, by stream; it ends with the thread
        ws = held.get(stream)
        if ws is None or ws.numel() < need:
            held.pop(stream, None)
            if len(held) >= _STREAMS:   # the allocator reuses it in its own stream's order
                held.pop(next(iter(held)))
            ws = held[stream] = torch.empty(need, dtype=torch.uint8, device=self.device)
        return ws

    def read(self, seq: int, n: int):
        """Keys and values of the first n slots of a sequence, kv_heads x n x head_dim in the cache's type (a copy;
        float16 for 4 bits)."""
        page = self.k.shape[2]
        if self.k.dtype is INT4:
            seqs, columns = self.table.shape
            slot = torch.arange(min(n, columns * page), dtype=torch.int32, device=self.device)
            return self.rows(torch.full_like(slot, range(seqs)[seq]), slot, token_major=False)   # refused as an index is
        ids = self.table[seq, : -(-n // page)].long()
        return tuple(x[ids].transpose(0, 1).reshape(self.kv_heads, -1, self.head_dim)[:, :n] for x in (self.k, self.v))

    def rows(self, seq, slot, token_major: bool = True):
        """Keys and values in slot[t] of sequence seq[t], l x kv_heads x head_dim (or kv_heads x l x head_dim) in the
        cache's type, the values in float16 for 4 bits; a token without a slot or page reads zeros."""
        l, h, d = slot.numel(), self.kv_heads, self.head_dim
        _int32(seq, "seq", l, self._index)
        _int32(slot, "slot", l, self._index)
        dtype = torch.float16 if self.k.dtype is INT4 else self.k.dtype
        k = torch.empty((l, h, d) if token_major else (h, l, d), dtype=dtype, device=self.device)
        v = torch.empty_like(k)
        status = M.lib().mosaic_kv_rows(self._ref, seq.data_ptr(), slot.data_ptr(), l, k.data_ptr(), v.data_ptr(),
                                        h * d if token_major else d, d if token_major else l * d, self._stream())
        if status:
            raise M.MosaicError("mosaic_kv_rows", status)
        return k, v

    def append(self, qkv, heads: int, seq, slot, index=None, rope: Rope | None = None, pos=None, out=None,
               norm: HeadNorm | None = None):
        """Norms (if given) and rotates row t of qkv (l x (heads + 2 kv_heads)
        head_dim fp32) and stores its keys and values in slot[t] of sequence
        seq[t] (a negative slot: not stored); returns the queries, l x heads x
        head_dim fp32."""
        d, width = self.head_dim, (heads + 2 * self.kv_heads) * self.head_dim
        if (qkv.dtype is not torch.float32 or qkv.dim() != 2 or qkv.get_device() != self._index
                or qkv.shape[1] != width or qkv.stride(1) != 1):
            raise ValueError("qkv: float32, l x (heads + 2 kv_heads) head_dim, rows contiguous, on the cache's device")
        l, ldx = qkv.shape[0], _row_stride(qkv, width, "qkv")
        _int32(seq, "seq", l, self._index)
        _int32(slot, "slot", l, self._index)
        if index is not None:
            _int32(index, "index", l, self._index)
        r = None
        if rope is not None:
            if rope.turns.get_device() != self._index:
                raise ValueError("rope: on another device than the cache")
            _need(pos is not None and pos.shape[-1] == l, "pos: a position for every token goes with rope")
            r = rope.at(pos)
        nm = None if norm is None else norm.on(d, self._index)
        q = torch.empty((l, heads, d), dtype=torch.float32, device=self.device) if out is None else out
        args = (self._ref, qkv.data_ptr(), ldx, l, heads, seq.data_ptr(), slot.data_ptr(),
                None if index is None else index.data_ptr(), None if r is None else ctypes.byref(r))
        to = (q.data_ptr(), heads * d if out is None else _rows(q, "out", l, heads, d, self._index), self._stream())
        if nm is None:
            status = self._calls[0](*args, *to)
        else:
            status = M.lib().mosaic_kv_append_norm(*args, nm, *to)
        if status:
            raise M.MosaicError("mosaic_kv_append" if nm is None else "mosaic_kv_append_norm", status)
        return q

    def attend(self, q, lens, max_len: int, first=None, scale: float | None = None, decay: float = 1.0, out=None):
        """Attention of one query a sequence (q: seqs x heads x head_dim fp32)
        over its first lens[i] <= max_len slots, without the slots whose
        position is below first[i]; adds the attention weights to
        ``weight`` (after scaling it by decay) if the cache keeps them."""
        n, d, at = self.seqs, self.head_dim, self._index
        heads = q.shape[1] if q.dim() == 3 else 0
        ldq = _rows(q, "q", n, heads, d, at)
        _int32(lens, "lens", n, at)
        if first is not None:
            _int32(first, "first", n, at)
        o = torch.empty((n, heads, d), dtype=torch.float32, device=self.device) if out is None else out
        stream = self._stream()
        need = self._bytes((heads, max_len), M.mosaic_kv_attention_workspace, heads, max_len)
        ws = self._workspace(need, stream)
        status = self._calls[1](self._ref, q.data_ptr(), ldq, heads, lens.data_ptr(), max_len,
                                None if first is None else first.data_ptr(), d ** -0.5 if scale is None else scale,
                                decay, o.data_ptr(), heads * d if out is None else _rows(o, "out", n, heads, d, at),
                                None if ws is None else ws.data_ptr(), need, stream)
        if status:
            raise M.MosaicError("mosaic_kv_attention", status)
        return o

    def evict(self, lens, max_len: int, keep: int, recent_from=None, new_lens=None):
        """Cuts every sequence to ``keep`` slots by least gathered weight (ties:
        the lower slot leaves), sparing positions >= recent_from[i]; returns
        the new lengths."""
        _int32(lens, "lens", self.seqs, self._index)
        if recent_from is not None:
            _int32(recent_from, "recent_from", self.seqs, self._index)
        new = torch.empty_like(lens) if new_lens is None else new_lens
        if new_lens is not None:
            _int32(new, "new_lens", self.seqs, self._index)
        stream = self._stream()
        need = self._bytes(("evict", max_len, keep), M.mosaic_kv_evict_workspace, max_len, keep)
        ws = self._workspace(need, stream)
        status = self._calls[2](self._ref, lens.data_ptr(), max_len, keep,
                                None if recent_from is None else recent_from.data_ptr(), new.data_ptr(),
                                None if ws is None else ws.data_ptr(), need, stream)
        if status:
            raise M.MosaicError("mosaic_kv_evict", status)
        return new


class PageTable:
    """Which page belongs to which sequence: the host's account and its copy
    on the device (``table``).  Page 0 is nobody's (the table's filler)."""

    def __init__(self, seqs: int, columns: int, pages: int, page_size: int, device="cuda"):
        _need(pages >= 1 and page_size >= 1, "pages and page_size: at least 1")
        self.page_size = page_size
        self.free = list(range(pages - 1, 0, -1))
        self.owned = [[] for _ in range(seqs)]
        self.columns = columns
        self.table = torch.zeros(seqs, columns, dtype=torch.int32, device=device)

    def resize(self, seq: int, slots: int) -> None:
        """Gives sequence ``seq`` the pages that ``slots`` slots need, and takes back what it has beyond."""
        need, own = -(-slots // self.page_size), self.owned[seq]
        _need(need <= self.columns, "the table has too few columns")
        _need(need - len(own) <= len(self.free), "no free page")
        while len(own) > need:
            self.free.append(own.pop())
        if len(own) < need:
            at = len(own)
            own += [self.free.pop() for _ in range(need - at)]
            self.table[seq, at:need] = torch.tensor(own[at:], dtype=torch.int32)
