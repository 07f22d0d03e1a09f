"""The operators of a decode step over the paged cache, on torch tensors: new tokens
into their pages (with rotary positions), attention of one new token per request,
eviction of the blocks that attention has weighed least.

Same names, rules and result codes as include/duplexkv.h.  Nothing is copied, cast
or laid out anew on the way: a tensor of another type, shape or device than the call
takes, or whose last dimension is not contiguous, is refused with KV_EINVAL.  Rows of q,
k, v and the outputs beside them, of positions and of kv_put's and kv_attend's tables may
lie apart; every other tensor is contiguous as a whole.  A tensor that asks for a gradient,
outside torch.no_grad(), that carries a tangent of forward-mode differentiation, or that
stands for others inside torch.func's transforms is refused too: there are no gradients.
What a call writes counts as changed in place, as by torch's own operators (the cache does
not: it is known by its address alone).  A call goes to the current stream of the cache's
device, unless it is given another (an integer handle); as with any torch operator, tensors
that are used on another stream than their own must not be freed before that stream is done
with them.
"""
from __future__ import annotations

import ctypes as C
import math
from typing import Optional, Sequence

import torch

from . import binding as B
from . import _decode_tensors as _T     # built in-tree like the library; there is no other path


class Rope:
    """How heads rotate: `inv_freq` (float32, on the cache's device) has one entry per pair;
    sections[i] pairs go by the positions of axis i (default: one axis has them all)."""

    def __init__(self, inv_freq: torch.Tensor, sections: Optional[Sequence[int]] = None, interleaved: bool = False):
        if inv_freq.dtype != torch.float32 or inv_freq.dim() != 1 or not inv_freq.is_contiguous() or not inv_freq.is_cuda:
            raise ValueError("inv_freq is a contiguous float32 vector on the GPU")
        self.inv_freq = inv_freq
        self.sections = tuple(int(n) for n in (sections or (inv_freq.numel(),)))
        if not 1 <= len(self.sections) <= 3 or min(self.sections) < 0 or sum(self.sections) != inv_freq.numel():
            raise ValueError("sections are one to three numbers of pairs that add up to inv_freq's")
        self.interleaved = bool(interleaved)


class Decoder:
    """Owns one kv_decoder handle.  `cfg` and `cache_ptr` are the Engine's; the cache must
    outlive the decoder.  Calls have to be ordered one after the other (one stream, or
    streams that the caller orders) and come from one host thread at a time: steps that overlap
    in time take a decoder each.  weigh=False: without the memory that kv_attend's mass takes."""

    def __init__(self, cfg: B.kv_config, cache_ptr: int, n_heads: int, max_seqs: int, max_blocks: int,
                 x_type: int = B.KV_BF16, kv_type: Optional[int] = None, k_scale: float = 1.0, v_scale: float = 1.0,
                 weigh: bool = True):
        self.cfg = cfg
        self._h = C.c_void_p()
        dc = B.kv_decoder_config(n_heads, x_type, x_type if kv_type is None else kv_type, max_seqs, max_blocks,
                                 k_scale, v_scale, int(weigh))
        rc = B.lib.kv_decoder_create(C.byref(self._h), C.byref(cfg), C.byref(dc), C.c_void_p(cache_ptr or None))
        if rc != B.KV_OK:
            self._h = C.c_void_p()
            raise B.KVError(rc, "kv_decoder_create")
        self._spec = _T.spec(self._h.value, cache_ptr, n_heads, int(cfg.n_kv_heads), int(cfg.head_dim), max_blocks, x_type,
                             1.0 / math.sqrt(cfg.head_dim))

    def kv_put(self, layer: int, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, *,
               q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
               starts: Optional[torch.Tensor] = None, rope: Optional[Rope] = None,
               positions: Optional[torch.Tensor] = None, stream: Optional[int] = None) -> int:
        """k, v [row, kv_head, dim] (and q, q_out [row, head, dim]): the last starts[s + 1] - starts[s] tokens
        of each request s, or the last one of each.  positions: int32 [axis, row] (expanded along the axes: the same for each);
        without them a row stands at its place in the request, which it does no more once kv_evict has shortened that."""
        if rope is None:
            return _T.put(self._spec, layer, k, v, table, lens, q, q_out, starts, None, False, (), positions, stream)
        return _T.put(self._spec, layer, k, v, table, lens, q, q_out, starts, rope.inv_freq, rope.interleaved, rope.sections,
                      positions, stream)

    def kv_attend(self, layer: int, q: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, out: torch.Tensor, *,
                  scale: Optional[float] = None, lse: Optional[torch.Tensor] = None, mass: Optional[torch.Tensor] = None,
                  mass_out: Optional[torch.Tensor] = None, stream: Optional[int] = None) -> int:
        """q, out [request, head, dim]; lse float32 [request, head]; mass, mass_out float32
        [request, max_blocks].  With mass alone, the weights are added to it in place."""
        return _T.attend(self._spec, layer, q, table, lens, out, scale, lse, mass, mass_out, stream)

    def kv_evict(self, table: torch.Tensor, lens: torch.Tensor, mass: torch.Tensor, *, budget: int, n_first: int, n_last: int,
                 evicted_ids: torch.Tensor, evicted_at: torch.Tensor, n_evicted: torch.Tensor,
                 table_out: Optional[torch.Tensor] = None, lens_out: Optional[torch.Tensor] = None,
                 mass_out: Optional[torch.Tensor] = None, stream: Optional[int] = None) -> int:
        """table int32 and mass float32 [request, max_blocks], lens int32 [request]; evicted_ids and
        evicted_at int32 [request, most to leave]; outputs that are not given: in place.  Later tokens of a request that
        gave up blocks need kv_put's positions: the keys that stay keep theirs."""
        return _T.evict(self._spec, table, lens, mass, budget, n_first, n_last, evicted_ids, evicted_at, n_evicted, table_out,
                        lens_out, mass_out, stream)

    def kv_decoder_destroy(self) -> int:
        if self._h:
            rc = B.lib.kv_decoder_destroy(self._h)
            self._h, self._spec = C.c_void_p(), None
            return rc
        return B.KV_OK

    def __del__(self):
        try:
            self.kv_decoder_destroy()
        except Exception:
            pass
