"""Keys and values of several continuations in pages that they share: a handle for the ouro_paged_* calls of include/ouro.h.

    cache = PagedCache(n_layers, n_pages, page_size, n_kv_heads, head_dim, "bf16", max_seqs=8, max_pages=64)
    slots, positions = cache.extend(seqs, new_tokens, width)          # room for a prompt, or for the next token
    q = cache.append(layer, q, k, v, slots.view(-1), positions.view(-1), cos, sin)
    out = cache.attend(layer, q.view(n, 1, heads, head_dim), seqs)    # the newest token of every sequence
    out = cache.attend_chunk(layer, q, starts, seqs)                  # a prompt's or several tokens of each, q [rows, heads, head_dim]
    cache.fork(parents, beams)                                        # beams[i] goes on from what parents[i] was

Arguments are CUDA tensors on the cache's device (lists: int32).  Calls are enqueued on torch's current stream; all calls on one cache
share its workspace and belong on one stream, or on streams that wait for one another.  Nothing synchronises except ``check``.  What the
host can see wrong raises; lists that turn out wrong on the device make their call do nothing and show in ``check``.
"""
from __future__ import annotations

import ctypes as C
import math

import torch

from . import binding
from .binding import OURO_BF16, OURO_F32, PagedCacheC, _check, current_stream, lib

_DTYPES = {torch.float32: OURO_F32, torch.bfloat16: OURO_BF16}
_NAMES = {"f32": torch.float32, "bf16": torch.bfloat16, torch.float32: torch.float32, torch.bfloat16: torch.bfloat16}


def rotary_tables(n_positions: int, head_dim: int, theta: float = 10000.0, device="cuda:0"):
    """cos, sin [n_positions, head_dim/2] f32 for ``PagedCache.append``, computed in 64 bits."""
    inv = theta ** (-2.0 * torch.arange(head_dim // 2, dtype=torch.float64, device=device) / head_dim)
    a = torch.arange(n_positions, dtype=torch.float64, device=device)[:, None] * inv
    return torch.cos(a).float(), torch.sin(a).float()


def set_wait_limit(polls: int):
    """Test aid: polls of the attention's bounded waits from now on, in this process (negative: the default)."""
    _check(lib().ouro_paged_debug_set_wait_limit(polls))


class PagedCache:
    """Pages of keys and values ``k``, ``v`` [layers, pages, page_size, kv heads, head_dim], and who names them: ``table`` [max_seqs, max_pages],
    ``lens`` [max_seqs], ``refs`` [pages], which lie side by side in ``state`` (so that a copy of ``state`` is all of it but the pages)."""

    def __init__(self, n_layers: int = 0, n_pages: int = 0, page_size: int = 0, n_kv_heads: int = 0, head_dim: int = 0, dtype: str | torch.dtype = "bf16", *,
                 max_seqs: int, max_pages: int, k: torch.Tensor | None = None, v: torch.Tensor | None = None, device="cuda:0"):
        """The sizes, from which pages are allocated (zeros), or tensors ``k`` and ``v`` of the caller, whose strides are kept (the last is 1).  Besides the pages a
        cache has a workspace for its calls: 43 MB with heads of 128, 22 with 64."""
        if (k is None) != (v is None):
            raise ValueError("k and v come together")
        if k is None:
            if dtype not in _NAMES:
                raise ValueError(f"dtype {dtype!r}: 'f32' or 'bf16' is needed")
            k = torch.zeros((n_layers, n_pages, page_size, n_kv_heads, head_dim), dtype=_NAMES[dtype], device=device)
            v = torch.zeros_like(k)
        if k.shape != v.shape or k.dim() != 5 or k.dtype != v.dtype or k.dtype not in _DTYPES or k.stride() != v.stride() or k.stride(4) != 1:
            raise ValueError("k and v are [layers, pages, page_size, kv heads, head_dim] of one type (f32, bf16) and layout, the last dimension dense")
        if not k.is_cuda or k.device != v.device:
            raise ValueError("k and v are on one CUDA device: this library has no CPU path")
        self.k, self.v, self.device = k, v, k.device
        self._dtype, self._index = k.dtype, k.device.index
        self.page_size, self.n_kv_heads, self.head_dim = k.shape[2:]
        self.max_seqs, self.max_pages = max_seqs, max_pages
        with torch.cuda.device(self.device):
            self.state = torch.empty(max_seqs * max_pages + max_seqs + k.shape[1], dtype=torch.int32, device=self.device)
            self.status = torch.empty(1, dtype=torch.int32, device=self.device)
            self.table = self.state[: max_seqs * max_pages].view(max_seqs, max_pages)
            self.lens = self.state[max_seqs * max_pages:][:max_seqs]
            self.refs = self.state[max_seqs * max_pages + max_seqs:]
            # (a dimension of one element is never stepped over: its stride may be anything)
            strides = [s if n > 1 else 0 for s, n in zip(k.stride()[:4], k.shape[:4])]
            self._c = PagedCacheC(*k.shape, _DTYPES[k.dtype], max_seqs, max_pages, *strides, k.data_ptr(), v.data_ptr(), self.table.data_ptr(),
                                  self.lens.data_ptr(), self.refs.data_ptr(), self.status.data_ptr(), 0, 0)
            self._L, self._p = lib(), C.byref(self._c)
            nbytes = self._L.ouro_paged_workspace_bytes(self._p)
            if nbytes == 0:
                raise binding.OuroError(binding.OURO_EINVAL)
            self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
            self._c.workspace, self._c.workspace_bytes = (self.workspace.data_ptr() + 255) & ~255, nbytes
            self.reset()

    def _stream(self):
        return current_stream(self._index)

    def _like(self, q, contiguous):
        # (empty_like is the quickest way to a new tensor, but keeps strides)
        return torch.empty_like(q) if contiguous else torch.empty(q.shape, dtype=q.dtype, device=self.device)

    def _list(self, t, name, n=None):
        if t.dtype is not torch.int32 or t.get_device() != self._index or not t.is_contiguous() or (n is not None and t.numel() != n):
            raise ValueError(f"{name}: a contiguous int32 tensor on {self.device}" + ("" if n is None else f" of {n} elements") + " is needed")
        return t.data_ptr()

    # ---- pages ---------------------------------------------------------------------------------
    def reset(self):
        """No sequences; all pages are free."""
        _check(self._L.ouro_paged_reset(self._p, self._stream()))

    def check(self):
        """Synchronises; raises the first refusal of a call since the last ``check`` (that call changed nothing)."""
        _check(self._L.ouro_paged_status(self._p, self._stream()))

    def fork(self, src, dst):
        """All at once, sequence dst[i] becomes what src[i] was; pages are shared, and given up by whom they were dst's."""
        n = src.numel()
        _check(self._L.ouro_paged_fork(self._p, self._list(src, "src"), self._list(dst, "dst", n), n, self._stream()))

    def truncate(self, seqs, keep):
        """Sequence seqs[i] keeps its first keep[i] tokens; 0 frees it."""
        n = seqs.numel()
        _check(self._L.ouro_paged_truncate(self._p, self._list(seqs, "seqs"), self._list(keep, "keep", n), n, self._stream()))

    def extend(self, seqs, new_tokens, width: int):
        """Room for new_tokens[i] <= width more tokens of sequence seqs[i].  Returns slots and positions [n, width], -1 where there is none."""
        n = seqs.numel()
        slots = torch.empty_strided((n, width), (width, 1), dtype=torch.int32, device=self.device)
        positions = torch.empty_like(slots)
        _check(self._L.ouro_paged_extend(self._p, self._list(seqs, "seqs"), self._list(new_tokens, "new_tokens", n), n, width, slots.data_ptr(),
                                         positions.data_ptr(), self._stream()))
        return slots, positions

    def compact(self):
        """Moves the pages in use to the lowest ids.  Returns their number [1]."""
        live = torch.empty(1, dtype=torch.int32, device=self.device)
        _check(self._L.ouro_paged_compact(self._p, live.data_ptr(), self._stream()))
        return live

    # ---- a layer of a forward --------------------------------------------------------------------
    def _rows(self, t, name, heads=None):
        """Rows [.., heads, head_dim] whose heads lie side by side: distance between rows in elements."""
        shape = t.shape                                     # (every question to a tensor is 0.05 to 0.2 us of a call of ten)
        if t.dtype is not self._dtype or t.get_device() != self._index or shape[-1] != self.head_dim or (heads is not None and shape[-2] != heads):
            raise ValueError(f"{name}: [.., {'heads' if heads is None else heads}, {self.head_dim}] of {self._dtype} on {self.device} is needed")
        if t.is_contiguous():
            return shape[-2] * self.head_dim
        strides = t.stride()
        if strides[-1] != 1 or (shape[-2] > 1 and strides[-2] != self.head_dim):
            raise ValueError(f"{name}: the heads of a row have to lie side by side")
        step = None
        for i in range(len(shape) - 3, -1, -1):             # rows at one distance throughout
            if shape[i] == 1:
                continue
            if step is None:
                step = each = strides[i]
            elif strides[i] != each:
                raise ValueError(f"{name}: the rows have to lie at one distance")
            each *= shape[i]
        return shape[-2] * self.head_dim if step is None else step

    def _out(self, out, q):
        if out is None:
            return self._like(q, q.is_contiguous())
        if out.shape != q.shape or not out.is_contiguous() or out.dtype is not q.dtype or out.device != self.device:
            raise ValueError("out has to be like q, and contiguous")
        return out

    def _new_rows(self, q, k, v):
        """Distances between the rows of new queries, and of new keys and values."""
        of_q, of_k, of_v = q.shape, k.shape, v.shape
        if not len(of_q) == len(of_k) == len(of_v) == 3:
            raise ValueError("q, k and v: [rows, heads, head_dim] is needed")
        q_stride, k_stride = self._rows(q, "q"), self._rows(k, "k", self.n_kv_heads)
        if self._rows(v, "v", self.n_kv_heads) != k_stride or not of_q[0] == of_k[0] == of_v[0]:
            raise ValueError("q, k and v need the same number of rows, k and v the same distance between them")
        return q_stride, k_stride

    def append(self, layer: int, q, k, v, slots, positions, cos, sin, out=None):
        """Rotates the queries q [rows, heads, head_dim] (returned; ``out`` may be q) and the keys k [rows, kv heads, head_dim], and writes keys
        and values to their slots; rows with a negative slot are padding."""
        q_stride, k_stride = self._new_rows(q, k, v)
        rows, heads, _ = q.shape
        out = self._out(out, q)
        if cos.dim() != 2 or cos.dtype is not torch.float32 or cos.shape != sin.shape or cos.shape[-1] * 2 != self.head_dim or not (cos.is_contiguous() and sin.is_contiguous()) \
                or sin.dtype is not torch.float32 or cos.device != self.device or sin.device != self.device:
            raise ValueError("cos and sin are contiguous f32 tensors [positions, head_dim/2] on the cache's device")
        _check(self._L.ouro_paged_append(self._p, layer, q.data_ptr(), q_stride, k.data_ptr(), v.data_ptr(), k_stride, rows, heads,
                                         self._list(slots, "slots", rows), self._list(positions, "positions", rows), cos.data_ptr(), sin.data_ptr(),
                                         cos.shape[0], out.data_ptr(), self._stream()))
        return out

    def append_rotary(self, layer: int, q, k, v, slots, positions, rotary, out=None):
        """``append`` with the positions of a ``rotary.Rotary``: interleaved pairs, part of the head, stretched contexts; no tables."""
        q_stride, k_stride = self._new_rows(q, k, v)
        rows, heads, _ = q.shape
        out = self._out(out, q)
        if rotary.head_dim != self.head_dim or rotary.turns.get_device() != self._index:
            raise ValueError(f"rotary: positions for heads of {self.head_dim} on {self.device} are needed")
        _check(self._L.ouro_paged_append_rotary(self._p, layer, q.data_ptr(), q_stride, k.data_ptr(), v.data_ptr(), k_stride, rows, heads,
                                                self._list(slots, "slots", rows), self._list(positions, "positions", rows), rotary._p, out.data_ptr(),
                                                self._stream()))
        return out

    def attend(self, layer: int, q, seqs=None, scale: float | None = None, out=None, want_lse: bool = False):
        """Attention of the newest tokens of sequences ``seqs`` (None: 0, 1, ..): q [n, heads, head_dim] for one token each, or [n, t, heads,
        head_dim] for the t newest, each of which sees the keys up to its own.  Returns the output like q, with ``want_lse`` also the logarithm of
        the sum of exponentials [.., heads] f32."""
        if not 3 <= q.dim() <= 4:
            raise ValueError("q: [n, heads, head_dim] or [n, t, heads, head_dim] is needed")
        n, t, heads = q.shape[0], 1 if q.dim() == 3 else q.shape[1], q.shape[-2]
        stride = self._rows(q, "q")
        out = self._out(out, q)
        lse = torch.empty(q.shape[:-1], dtype=torch.float32, device=self.device) if want_lse else None
        _check(self._L.ouro_paged_attention(self._p, layer, None if seqs is None else self._list(seqs, "seqs", n), n, t, q.data_ptr(), stride, heads,
                                            1.0 / math.sqrt(self.head_dim) if scale is None else scale, out.data_ptr(),
                                            lse.data_ptr() if want_lse else None, self._stream()))
        return (out, lse) if want_lse else out

    def attend_chunk(self, layer: int, q, starts, seqs=None, scale: float | None = None, out=None, want_lse: bool = False):
        """Attention of a chunk of the newest tokens of each of the sequences ``seqs`` (None: 0, 1, ..), from one to thousands: those of sequence i
        are the rows starts[i] .. starts[i + 1] - 1 of q [rows, heads, head_dim]; each sees the keys up to its own.  Returns the output like q, with ``want_lse`` also
        the logarithm of the sum of exponentials [rows, heads] f32; rows of no sequence are left as they are (in a new output: undefined)."""
        if q.dim() != 3:
            raise ValueError("q: [rows, heads, head_dim] is needed")
        stride = self._rows(q, "q")
        n = starts.numel() - 1
        if n < 0:
            raise ValueError("starts: one more element than there are sequences is needed")
        out = self._out(out, q)
        lse = torch.empty(q.shape[:-1], dtype=torch.float32, device=self.device) if want_lse else None
        _check(self._L.ouro_paged_chunk_attention(self._p, layer, None if seqs is None else self._list(seqs, "seqs", n), self._list(starts, "starts"), n, q.shape[0],
                                                  q.data_ptr(), stride, q.shape[1], 1.0 / math.sqrt(self.head_dim) if scale is None else scale, out.data_ptr(),
                                                  lse.data_ptr() if want_lse else None, self._stream()))
        return (out, lse) if want_lse else out
