"""The operators of a decode step over the paged cache, on torch tensors: new tokens
into their pages (with rotary positions), attention of one new token per request,
eviction of the blocks that attention has weighed least.

Same names, rules and result codes as include/duplexkv.h.  Nothing is copied, cast
or laid out anew on the way: a tensor of another type, shape or device than the call
takes, or whose last dimension is not contiguous, is refused with KV_EINVAL.  A call
goes to the current stream of the cache's device, unless it is given another
(an integer handle); as with any torch operator, tensors that are used on another stream
than their own must not be freed before that stream is done with them.
"""
from __future__ import annotations

import ctypes as C
import math
from typing import Optional, Sequence

import torch

from . import binding as B

_X = {B.KV_BF16: torch.bfloat16, B.KV_FP16: torch.float16}
_INT, _FLOAT = torch.int32, torch.float32


class Rope:
    """How heads rotate: `inv_freq` (float32, on the cache's device) has one entry per pair;
    sections[i] pairs go by the positions of axis i (default: one axis has them all)."""

    def __init__(self, inv_freq: torch.Tensor, sections: Optional[Sequence[int]] = None, interleaved: bool = False):
        if inv_freq.dtype != _FLOAT or inv_freq.dim() != 1 or not inv_freq.is_contiguous() or not inv_freq.is_cuda:
            raise ValueError("inv_freq is a contiguous float32 vector on the GPU")
        self.inv_freq = inv_freq
        self.sections = tuple(int(n) for n in (sections or (inv_freq.numel(),)))
        if not 1 <= len(self.sections) <= 3 or min(self.sections) < 0 or sum(self.sections) != inv_freq.numel():
            raise ValueError("sections are one to three numbers of pairs that add up to inv_freq's")
        self.interleaved = bool(interleaved)
        self.c_sections = (C.c_int32 * 3)(*(self.sections + (0, 0, 0))[:3])


class Decoder:
    """Owns one kv_decoder handle.  `cfg` and `cache_ptr` are the Engine's; the cache must
    outlive the decoder.  Calls have to be ordered one after the other (one stream, or
    streams that the caller orders): steps that overlap in time take a decoder each."""

    def __init__(self, cfg: B.kv_config, cache_ptr: int, n_heads: int, max_seqs: int, max_blocks: int,
                 x_type: int = B.KV_BF16, kv_type: Optional[int] = None, k_scale: float = 1.0, v_scale: float = 1.0):
        self.cfg = cfg
        self._h = C.c_void_p()
        dc = B.kv_decoder_config(n_heads, x_type, x_type if kv_type is None else kv_type, max_seqs, max_blocks, k_scale, v_scale)
        rc = B.lib.kv_decoder_create(C.byref(self._h), C.byref(cfg), C.byref(dc), C.c_void_p(cache_ptr or None))
        if rc != B.KV_OK:
            self._h = C.c_void_p()
            raise B.KVError(rc, "kv_decoder_create")
        self._x = _X[x_type]
        self.n_heads, self.max_blocks = n_heads, max_blocks
        self._heads, self._dim = int(cfg.n_kv_heads), int(cfg.head_dim)
        self._scale = 1.0 / math.sqrt(self._dim)

    def _rows(self, to: B.kv_rows, t: torch.Tensor, n: int, heads: int) -> bool:
        """[row, head, dim] tensors: where they lie, or False if they do not fit."""
        if t.dtype != self._x or not t.is_cuda:
            return False
        shape, (row, head, one) = t.shape, t.stride() if t.dim() == 3 else (0, 0, 0)
        if one != 1 or shape[0] != n or shape[1] != heads or shape[2] != self._dim:
            return False
        to.data, to.row, to.head = t.data_ptr(), row, head
        return True

    def _tables(self, a, table: torch.Tensor, lens: torch.Tensor) -> bool:
        """The table and the lengths that every call has."""
        n = lens.shape[0] if lens.dim() == 1 else -1
        if table.dtype != _INT or lens.dtype != _INT or not table.is_cuda or not lens.is_cuda or table.dim() != 2:
            return False
        shape, (row, one) = table.shape, table.stride()
        if n < 0 or shape[0] != n or shape[1] != self.max_blocks or (one != 1 and shape[1] > 1) or (n > 1 and lens.stride(0) != 1):
            return False
        if n > 1 and not self.max_blocks <= row < 1 << 31:
            return False
        a.n_seqs, a.table_stride, a.table, a.lens = n, row if n > 1 else self.max_blocks, table.data_ptr(), lens.data_ptr()
        return True

    @staticmethod
    def _vector(t: torch.Tensor, dtype, n: int) -> bool:
        return t.dtype == dtype and t.is_cuda and t.dim() == 1 and t.shape[0] == n and (n < 2 or t.stride(0) == 1)

    @staticmethod
    def _matrix(t: torch.Tensor, dtype, n: int, m: int) -> bool:
        return t.dtype == dtype and t.is_cuda and t.dim() == 2 and t.shape[0] == n and t.shape[1] == m and t.is_contiguous()

    @staticmethod
    def _stream(stream: Optional[int], t: torch.Tensor) -> Optional[int]:
        return (torch.cuda.current_stream(t.device).cuda_stream if stream is None else stream) or None

    def kv_put(self, layer: int, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, *,
               q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
               starts: Optional[torch.Tensor] = None, rope: Optional[Rope] = None,
               positions: Optional[torch.Tensor] = None, stream: Optional[int] = None) -> int:
        """k, v [row, kv_head, dim] (and q, q_out [row, head, dim]): the last starts[s + 1] - starts[s] tokens
        of each request s, or the last one of each.  positions: int32 [axis, row]."""
        a = B.kv_put_args()
        if k.dim() != 3 or not self._tables(a, table, lens) or not self._rows(a.k, k, k.shape[0], self._heads) or \
                not self._rows(a.v, v, k.shape[0], self._heads) or (q is None) != (q_out is None):
            return B.KV_EINVAL
        n = a.n_rows = k.shape[0]
        a.layer = layer
        if q is not None and not (self._rows(a.q, q, n, self.n_heads) and self._rows(a.q_out, q_out, n, self.n_heads)):
            return B.KV_EINVAL
        if starts is not None:
            if not self._vector(starts, _INT, a.n_seqs + 1):
                return B.KV_EINVAL
            a.starts = starts.data_ptr()
        if rope is not None:
            a.inv_freq, a.rot_dim, a.interleaved = rope.inv_freq.data_ptr(), 2 * rope.inv_freq.numel(), rope.interleaved
            a.n_axes, a.sections = len(rope.sections), rope.c_sections
            if positions is not None:
                if positions.dtype != _INT or not positions.is_cuda or positions.dim() != 2 or positions.shape[0] != a.n_axes or \
                        positions.shape[1] != n or (n > 1 and positions.stride(1) != 1):
                    return B.KV_EINVAL
                a.positions, a.position_stride = positions.data_ptr(), positions.stride(0) if a.n_axes > 1 else n
        elif positions is not None:
            return B.KV_EINVAL
        return B.lib.kv_put(self._h, C.byref(a), self._stream(stream, k))

    def kv_attend(self, layer: int, q: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, out: torch.Tensor, *,
                  scale: Optional[float] = None, lse: Optional[torch.Tensor] = None, mass: Optional[torch.Tensor] = None,
                  mass_out: Optional[torch.Tensor] = None, stream: Optional[int] = None) -> int:
        """q, out [request, head, dim]; lse float32 [request, head]; mass, mass_out float32
        [request, max_blocks].  With mass alone, the weights are added to it in place."""
        a = B.kv_attend_args()
        if not self._tables(a, table, lens):
            return B.KV_EINVAL
        n = a.n_seqs
        if not self._rows(a.q, q, n, self.n_heads) or not self._rows(a.out, out, n, self.n_heads):
            return B.KV_EINVAL
        if lse is not None:
            if not self._matrix(lse, _FLOAT, n, self.n_heads):
                return B.KV_EINVAL
            a.lse = lse.data_ptr()
        if mass is not None or mass_out is not None:
            mass_out = mass if mass_out is None else mass_out
            if not self._matrix(mass_out, _FLOAT, n, self.max_blocks) or \
                    (mass is not None and not self._matrix(mass, _FLOAT, n, self.max_blocks)):
                return B.KV_EINVAL
            a.mass, a.mass_out, a.mass_stride = None if mass is None else mass.data_ptr(), mass_out.data_ptr(), self.max_blocks
        a.layer, a.scale = layer, self._scale if scale is None else scale
        return B.lib.kv_attend(self._h, C.byref(a), self._stream(stream, q))

    def kv_evict(self, table: torch.Tensor, lens: torch.Tensor, mass: torch.Tensor, *, budget: int, n_first: int, n_last: int,
                 evicted_ids: torch.Tensor, evicted_at: torch.Tensor, n_evicted: torch.Tensor,
                 table_out: Optional[torch.Tensor] = None, lens_out: Optional[torch.Tensor] = None,
                 mass_out: Optional[torch.Tensor] = None, stream: Optional[int] = None) -> int:
        """table int32 and mass float32 [request, max_blocks], lens int32 [request]; evicted_ids and
        evicted_at int32 [request, most to leave]; outputs that are not given: in place."""
        a = B.kv_evict_args()
        table_out, lens_out = table if table_out is None else table_out, lens if lens_out is None else lens_out
        mass_out = mass if mass_out is None else mass_out
        n = lens.shape[0] if lens.dim() == 1 else -1
        if not all(self._vector(t, _INT, n) for t in (lens, lens_out, n_evicted)) or evicted_ids.dim() != 2:
            return B.KV_EINVAL
        m = evicted_ids.shape[1]
        if not all(self._matrix(t, _INT, n, self.max_blocks) for t in (table, table_out)) or \
                not all(self._matrix(t, _FLOAT, n, self.max_blocks) for t in (mass, mass_out)) or \
                not all(self._matrix(t, _INT, n, m) for t in (evicted_ids, evicted_at)):
            return B.KV_EINVAL
        a.n_seqs, a.budget, a.n_first, a.n_last, a.max_evict = n, budget, n_first, n_last, m
        a.table_stride = a.mass_stride = self.max_blocks
        a.table, a.table_out, a.lens, a.lens_out = table.data_ptr(), table_out.data_ptr(), lens.data_ptr(), lens_out.data_ptr()
        a.mass, a.mass_out, a.n_evicted = mass.data_ptr(), mass_out.data_ptr(), n_evicted.data_ptr()
        a.evicted_ids, a.evicted_at = evicted_ids.data_ptr(), evicted_at.data_ptr()
        return B.lib.kv_evict(self._h, C.byref(a), self._stream(stream, table))

    def kv_decoder_destroy(self) -> int:
        if self._h:
            rc = B.lib.kv_decoder_destroy(self._h)
            self._h = C.c_void_p()
            return rc
        return B.KV_OK

    def __del__(self):
        try:
            self.kv_decoder_destroy()
        except Exception:
            pass
