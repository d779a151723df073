"""A K/V cache in 4 bits: a quarter of the memory and of the bytes that attention reads.  Sixteen channels of a token and head share a scale (an 8-bit float); a channel is a 4-bit float times that
(format and contracts: include/specdec.h).  It stands in a tree.PagedCache's place: reserve, append, compact, release, fork and reorder are the same calls, and tree.attention reads it.

    cache = fp4.Fp4Cache(n_layers, n_heads, head_dim, n_pages=..., n_seqs=..., max_pages=...)
    cache.reserve(seqs, T)
    cache.append(seqs, k, v, layer=i)                        # fp32, bf16 or fp16
    o = tree.attention(q, cache, i, seqs, mask)              # of q's type
    k, v = cache.read(seqs, T, layer=i)                      # the values that the attention sees
"""
from __future__ import annotations

import ctypes as C
import struct
from typing import Optional

import torch

from . import binding, tree
from .tree import DTYPES, PagedCache, _ints, _launch, _NoGradient

BLOCK = 16                                                   # channels of a scale
_FP4 = 3                                                     # SPECDEC_DTYPE_FP4
_tokens_args = struct.Struct("@PPPPqqqqiiiii0q")             # PackedTokens in one go
assert _tokens_args.size == C.sizeof(binding.PackedTokens)


class Fp4Cache(PagedCache):
    """codes [n_layers, 2, n_pages, n_heads, page_tokens, head_dim / 2] uint8, scales [.., head_dim / 16] float8_e4m3fn, unit [n_layers, 2, n_heads] fp32 (None: 1) and the bookkeeping of a
    PagedCache.  A value is unit * scale * code.  The larger the unit, the larger the values that can be held: scales reach from 2^-9 to 448, values to 2688 units.  head_dim: 64 or 128."""

    def __init__(self, n_layers: int, n_heads: int, head_dim: int, *, n_pages: int, n_seqs: int, max_pages: int, page_tokens: int = 16, unit=None, device="cuda"):
        i32, shape = dict(dtype=torch.int32, device=device), (n_layers, 2, n_pages, n_heads, page_tokens)
        self._set(torch.zeros(*shape, head_dim // 2, dtype=torch.uint8, device=device), torch.zeros(*shape, head_dim // BLOCK, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn),
                  torch.full((n_seqs, max_pages), -1, **i32), torch.zeros(n_seqs, **i32), torch.zeros(n_seqs, **i32), torch.zeros(n_pages, **i32), unit)

    @classmethod
    def over(cls, codes, scales, table, length, held, refs, unit=None):
        """A cache over tensors that exist.  codes and scales: of any strides, with contiguous tokens of a page and head."""
        self = cls.__new__(cls)
        self._set(codes, scales, table, length, held, refs, unit)
        return self

    def _set(self, codes, scales, table, length, held, refs, unit):
        if codes.dim() != 6 or codes.shape[1] != 2 or codes.dtype is not torch.uint8 or not codes.is_cuda or codes.stride(5) != 1 or (codes.stride(4) != codes.shape[5] and codes.shape[4] != 1):
            raise ValueError("codes: a uint8 device tensor [n_layers, 2, n_pages, n_heads, page_tokens, head_dim / 2] with contiguous tokens is wanted")
        L, _, P, H, page, half = codes.shape
        D, at = 2 * half, codes.get_device()
        if (D not in (64, 128) or scales.shape != (L, 2, P, H, page, D // BLOCK) or scales.dtype is not torch.float8_e4m3fn or scales.get_device() != at or scales.stride(5) != 1
                or (scales.stride(4) != D // BLOCK and page != 1)):
            raise ValueError("scales: a float8_e4m3fn tensor [n_layers, 2, n_pages, n_heads, page_tokens, head_dim / 16] with contiguous tokens is wanted beside the codes, head_dim 64 or 128")
        if unit is not None and (unit.shape != (L, 2, H) or unit.dtype is not torch.float32 or unit.get_device() != at or not unit.is_contiguous()):
            raise ValueError("unit: a contiguous fp32 tensor [n_layers, 2, n_heads] is wanted beside the codes")
        n_seqs = length.numel()
        _ints("table", table, (n_seqs, table.shape[1]), at), _ints("length", length, (n_seqs,), at), _ints("held", held, (n_seqs,), at), _ints("refs", refs, (P,), at)
        self.codes, self.scales, self.unit, self.table, self.length, self.held, self.refs = codes, scales, unit, table, length, held, refs
        self.status = torch.zeros(1, dtype=torch.int32, device=codes.device)
        self._scratch = self._new_scratch(n_seqs, table.shape[1], P, codes.device)
        s, z = codes.stride(), scales.stride()
        self._c = binding.Fp4Cache(binding.Cache(codes.data_ptr(), _FP4, L, H, D, P, page, n_seqs, table.shape[1], s[0], s[1], s[2], half, s[3],
                                                 table.data_ptr(), length.data_ptr(), held.data_ptr(), refs.data_ptr(), self.status.data_ptr(), self._scratch.data_ptr()),
                                   scales.data_ptr(), z[0], z[1], z[2], z[3], None if unit is None else unit.data_ptr())
        self._ref, self.dtype = C.byref(self._c), None         # (of no type of its own)
        self._finish("specdec_packed_cache_", at, n_layers=L, n_heads=H, head_dim=D, page=page, max_pages=table.shape[1])
        self._call["read"] = self._lib.specdec_packed_cache_read

    def append(self, seqs, k, v, layer: Optional[int] = None, count=None):
        """Writes k, v [n, T, n_heads, head_dim] (layer=None: [n_layers, n, T, n_heads, head_dim], every layer), fp32, bf16 or fp16, in 4 bits behind the committed tokens; of
        sequence i the first count[i] of the T.  Lengths stay: compact moves them."""
        n, dtype = seqs.numel(), k.dtype
        code = DTYPES.get(dtype)
        if code is None:
            raise ValueError("k, v: fp32, bf16 or fp16 is wanted")
        layer, layers, shape, s = self._block(n, k, v, layer, dtype)
        if (k.requires_grad or v.requires_grad) and torch.is_grad_enabled() and self._source is None:
            self._source = torch.zeros((), requires_grad=True)
        at = self._device
        self._tokens("append", _ints("seqs", seqs, (n,), at), k.data_ptr(), v.data_ptr(), 0 if count is None else _ints("count", count, (n,), at), s[0], s[1], s[2], s[3], n, layer, layers, code, shape[2])

    def _tokens(self, call, *args):
        try:
            a = _tokens_args.pack(*args)
        except struct.error as e:
            raise ValueError(f"layer or number of tokens: {e}") from None
        _launch(self._call[call], self._device, (self._ref, a, tree._raw_stream(self._device)))

    def read(self, seqs, n_tokens: int, layer: Optional[int] = None, start=None, dtype=torch.bfloat16):
        """(k, v) [(n_layers,) n, n_tokens, n_heads, head_dim]: the values of tokens start[i], start[i] + 1, ... of each sequence (start=None: those behind the committed ones); zeros where it
        has no page."""
        n, at = seqs.numel(), self._device
        code = DTYPES.get(dtype)
        if code is None or n_tokens < 0:
            raise ValueError("dtype: fp32, bf16 or fp16, and a number of tokens, are wanted")
        layers = self.n_layers if layer is None else 1
        k, v = torch.empty((2, layers, n, n_tokens, self.n_heads, self.head_dim) if layer is None else (2, n, n_tokens, self.n_heads, self.head_dim), dtype=dtype, device=self.codes.device).unbind(0)
        token = self.n_heads * self.head_dim
        self._tokens("read", _ints("seqs", seqs, (n,), at), k.data_ptr(), v.data_ptr(), 0 if start is None else _ints("start", start, (n,), at), n * n_tokens * token, n_tokens * token, token,
                     self.head_dim, n, 0 if layer is None else layer, layers, code, n_tokens)
        if self._source is not None and torch.is_grad_enabled():
            return tuple(_NoGradient.apply(x, "Fp4Cache.read", self._source) for x in (k, v))
        return k, v
