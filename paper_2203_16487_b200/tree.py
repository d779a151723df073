"""Operators of tree speculation on the caller's own tensors: a paged K/V cache, attention of drafted trees over it, sampling,
and the walk that accepts a branch.  Thin wrappers of the specdec_cache_* / specdec_tree_* / specdec_sample calls (contracts: include/specdec.h);
every call runs on the tensors' device, on its current stream, and returns without waiting for it.  They serve inference: a result of tensors that require a gradient
passes on, and raises when the gradient is asked for.

    mask, depth = tree.ancestors(parents)                    # once a step
    cache.reserve(seqs, T)
    for layer in ...:
        cache.append(seqs, k, v, layer=layer)                # the block's keys and values, behind the committed tokens
        o = tree.attention(q, cache, layer, seqs, mask)
    sampled, logprob = tree.sample(logits, uniform, temperature, top_k, top_p, min_p)
    path, n_path, emitted = tree.accept(parents, tokens, sampled)
    cache.compact(seqs, path, n_path)                        # the accepted nodes are committed tokens now

Lengths and pages are read on the device, so a step may be captured in a CUDA graph and replayed as the sequences grow (without max_length, which a graph would keep).
"""
from __future__ import annotations

import ctypes as C
import struct
from typing import Optional

import torch

from .binding import Cache, SpecDecError, TreeAttentionArgs, lib

DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_I32 = torch.int32
# TreeAttentionArgs in one go: 0.7 us less than filling the structure
_attention_args = struct.Struct("@PPqqqqqqiiiiPPqPifPq")
assert _attention_args.size == C.sizeof(TreeAttentionArgs)
# torch.cuda.current_stream(i).cuda_stream and torch.cuda.current_device(), 3 us cheaper: small calls are bounded by the host
_raw_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice


def _fail(rc):
    raise SpecDecError(rc, lib().specdec_last_error(None).decode())


def _launch(f, at, args):
    """f(*args) with the tensors' device `at` current: the library launches on the current device, and the default streams of all devices are one handle."""
    if _current_device() == at:
        rc = f(*args)
    else:
        with torch.cuda.device(at):
            rc = f(*args)
    if rc:
        _fail(rc)


class _NoGradient(torch.autograd.Function):
    """Passes a result on as one of `sources` (None: none), some of which require a gradient; there is none to give."""

    @staticmethod
    def forward(ctx, result, name, *sources):
        ctx.name = name
        return result

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError(f"{ctx.name} has no gradient: call it under torch.no_grad(), or on detached tensors")


def _ints(name, t, shape, device):
    """Address of a contiguous int32 tensor of that shape on that device (a number; -1 is none)."""
    if t.dtype is _I32 and t.shape == shape and t.get_device() == device >= 0 and t.is_contiguous():
        return t.data_ptr()
    raise ValueError(f"{name}: a contiguous int32 device tensor of shape {tuple(shape)} is wanted, on the device of the others, got {t.dtype} {tuple(t.shape)} on {t.device}")


class PagedCache:
    """A K/V cache in pages: kv [n_layers, 2, n_pages, page_tokens, n_heads, head_dim] and its bookkeeping (see specdec_cache).  Sequences are
    numbers 0 .. n_seqs - 1; calls take them as int32 device tensors, all different within a call."""

    def __init__(self, n_layers: int, n_heads: int, head_dim: int, *, n_pages: int, n_seqs: int, max_pages: int, page_tokens: int = 16,
                 dtype=torch.bfloat16, device="cuda"):
        i32 = dict(dtype=torch.int32, device=device)
        self._set(torch.zeros(n_layers, 2, n_pages, page_tokens, n_heads, head_dim, dtype=dtype, device=device),
                  torch.full((n_seqs, max_pages), -1, **i32), torch.zeros(n_seqs, **i32), torch.zeros(n_seqs, **i32), torch.zeros(n_pages, **i32))

    @classmethod
    def over(cls, kv, table, length, held, refs):
        """A cache over tensors that exist: kv [n_layers, 2, n_pages, page_tokens, n_heads, head_dim] of any strides with a contiguous last dimension
        (permute a [.., n_heads, page_tokens, ..] layout), table [n_seqs, max_pages], length and held [n_seqs], refs [n_pages]."""
        self = cls.__new__(cls)
        self._set(kv, table, length, held, refs)
        return self

    def _set(self, kv, table, length, held, refs):
        if kv.dim() != 6 or kv.shape[1] != 2 or kv.stride(5) != 1 or kv.dtype not in DTYPES or not kv.is_cuda:
            raise ValueError("kv: a device tensor [n_layers, 2, n_pages, page_tokens, n_heads, head_dim] with a contiguous last dimension is wanted")
        L, _, P, page, H, D = kv.shape
        n_seqs = length.numel()
        at = kv.get_device()
        _ints("table", table, (n_seqs, table.shape[1]), at), _ints("length", length, (n_seqs,), at), _ints("held", held, (n_seqs,), at), _ints("refs", refs, (P,), at)
        self.kv, self.table, self.length, self.held, self.refs = kv, table, length, held, refs
        self.status = torch.zeros(1, dtype=torch.int32, device=kv.device)
        self._scratch = self._new_scratch(n_seqs, table.shape[1], P, kv.device)
        s = kv.stride()
        self._c = Cache(kv.data_ptr(), DTYPES[kv.dtype], L, H, D, P, page, n_seqs, table.shape[1], s[0], s[1], s[2], s[3], s[4],
                        table.data_ptr(), length.data_ptr(), held.data_ptr(), refs.data_ptr(), self.status.data_ptr(), self._scratch.data_ptr())
        self._ref, self._code = C.byref(self._c), DTYPES[kv.dtype]
        self.dtype = kv.dtype
        self._finish("specdec_cache_", kv.get_device(), n_layers=L, n_heads=H, head_dim=D, page=page, max_pages=table.shape[1])

    @staticmethod
    def _new_scratch(n_seqs, max_pages, n_pages, device):
        n = lib().specdec_cache_scratch(n_seqs, max_pages, n_pages)
        if n < 0:
            _fail(n)
        return torch.zeros(n, dtype=torch.int32, device=device)

    def _finish(self, calls, device, *, n_layers, n_heads, head_dim, page, max_pages):
        """What every cache has: the library's calls of its kind, sizes, workspaces."""
        self._lib, self._device, self._page = lib(), device, page
        self._call = {name: getattr(self._lib, calls + name) for name in ("reserve", "append", "compact", "release", "fork", "reorder")}
        self._workspaces = {}                              # bytes by sizes of a call
        self._source = None                                # requires a gradient, where keys or values did
        self.n_layers, self.n_heads, self.head_dim, self.max_length = n_layers, n_heads, head_dim, max_pages * page

    def reserve(self, seqs, n_tokens: int):
        """Pages for n_tokens tokens behind the committed ones."""
        n = seqs.numel()
        _launch(self._call["reserve"], self._device, (self._ref, _ints("seqs", seqs, (n,), self._device), n, n_tokens, _raw_stream(self._device)))

    def _block(self, n, k, v, layer, dtype):
        """(layer, layers, shape, strides) of tokens k, v [(n_layers,) n, T, n_heads, head_dim]; raises where they are none."""
        shape, s = k.shape, k.stride()
        if layer is None:
            layer, layers = 0, self.n_layers
            good = len(shape) == 5 and shape[0] == layers
        else:
            layers, shape, s = 1, (1,) + tuple(shape), (0,) + tuple(s)
            good = len(shape) == 5
        if not (good and v.shape == k.shape and (v.stride() == k.stride() or all(a == b or m == 1 for a, b, m in zip(v.stride(), k.stride(), k.shape))) and k.dtype is dtype and v.dtype is dtype and k.get_device() == v.get_device() == self._device
                and s[4] == 1 and shape[1] == n and shape[3] == self.n_heads and shape[4] == self.head_dim):
            raise ValueError("k, v: device tensors [(n_layers,) n, T, n_heads, head_dim] of the cache's type and alike in their strides are wanted")      # (a dimension of 1 has none)
        return layer, layers, shape, s

    def append(self, seqs, k, v, layer: Optional[int] = None, count=None):
        """Writes k, v [n, T, n_heads, head_dim] (layer=None: [n_layers, n, T, n_heads, head_dim], every layer) behind the committed tokens; of
        sequence i the first count[i] of the T.  Lengths stay: compact moves them."""
        n = seqs.numel()
        layer, layers, shape, s = self._block(n, k, v, layer, self.dtype)
        if (k.requires_grad or v.requires_grad) and torch.is_grad_enabled() and self._source is None:
            self._source = torch.zeros((), requires_grad=True)
        _launch(self._call["append"], self._device, (self._ref, _ints("seqs", seqs, (n,), self._device), n, layer, layers, k.data_ptr(), v.data_ptr(), shape[2],
                s[0], s[1], s[2], s[3], None if count is None else _ints("count", count, (n,), self._device), _raw_stream(self._device)))

    def compact(self, seqs, path, n_path):
        """Commits the nodes path[i, :n_path[i]] of each sequence's block and gives back the pages behind them."""
        n, T = seqs.numel(), path.shape[-1]
        _launch(self._call["compact"], self._device, (self._ref, _ints("seqs", seqs, (n,), self._device), n, _ints("path", path, (n, T), self._device), T,
                _ints("n_path", n_path, (n,), self._device), _raw_stream(self._device)))

    def release(self, seqs):
        """Gives back all pages of the sequences; their lengths are 0."""
        n = seqs.numel()
        _launch(self._call["release"], self._device, (self._ref, _ints("seqs", seqs, (n,), self._device), n, _raw_stream(self._device)))

    def fork(self, src, dst):
        """Sequence dst[i] becomes a copy of what src[i] was before the call: full pages shared, the last, partly filled one copied."""
        n = src.numel()
        _launch(self._call["fork"], self._device, (self._ref, _ints("src", src, (n,), self._device), _ints("dst", dst, (n,), self._device), n, _raw_stream(self._device)))

    def reorder(self, seqs, parents):
        """Beams: of seqs [..., K], groups of K sequences (all different, over all groups), each becomes what sequence parents [..., K] (its place in the group, 0 .. K - 1; -1: none) was before the call.  Full pages
        are shared; the last, partly filled one goes on with one child (the parent itself if it is one, else the first) and is copied for the others."""
        if seqs.dim() < 1:
            raise ValueError("seqs: groups of sequences [..., K] are wanted")
        shape, n = seqs.shape, seqs.numel()
        _launch(self._call["reorder"], self._device, (self._ref, _ints("seqs", seqs, shape, self._device), _ints("parents", parents, shape, self._device), n, max(shape[-1], 1),
                                                      _raw_stream(self._device)))

    def check(self):
        """Raises if a call found too few pages or bad numbers since the last check (waits for the stream)."""
        s = int(self.status.item())
        if s:
            self.status.zero_()
            what = [m for bit, m in ((1, "not enough free pages"), (2, "a sequence has no room for more pages"), (4, "a sequence number or path out of range"),
                                     (8, "tokens outside the pages reserved"), (16, "a wait inside a kernel gave up")) if s & bit]
            raise SpecDecError(-3, "cache: " + ", ".join(what))


def ancestors(parents, n_nodes=None):
    """(mask [B, T, ceil(T / 32)] int32 of ancestor bits, depth [B, T] int32) of trees given by their parents [B, T]."""
    B, T = parents.shape
    at = parents.get_device()
    p = _ints("parents", parents, (B, T), at)
    mask, depth = parents.new_empty(B, T, (T + 31) // 32), torch.empty_like(parents)
    _launch(lib().specdec_tree_ancestors, at, (p, None if n_nodes is None else _ints("n_nodes", n_nodes, (B,), at), B, T, mask.data_ptr(), depth.data_ptr(), _raw_stream(at)))
    return mask, depth


def accept(parents, tokens, sampled, n_nodes=None):
    """(path [B, T], n_path [B], emitted [B, T]): the nodes from the root along the sampled tokens, and the sampled token of each (-1 behind)."""
    shape = parents.shape
    B, T = shape
    at = parents.get_device()
    p = _ints("parents", parents, shape, at)
    path, emitted, n_path = torch.empty_like(parents), torch.empty_like(parents), parents.new_empty(B)
    _launch(lib().specdec_tree_accept, at, (p, _ints("tokens", tokens, shape, at), _ints("sampled", sampled, shape, at), None if n_nodes is None else _ints("n_nodes", n_nodes, (B,), at),
            B, T, path.data_ptr(), n_path.data_ptr(), emitted.data_ptr(), _raw_stream(at)))
    return path, n_path, emitted


def attention(q, cache: PagedCache, layer: int, seqs, mask, *, n_nodes=None, max_length: int = 0, scale: Optional[float] = None, out=None):
    """Attention of tree nodes q [B, T, n_q_heads, head_dim] over the committed tokens of sequences seqs [B] and, by mask [B or 1, T, ceil(T / 32)], over
    the block's nodes (appended before).  max_length: an upper bound of the committed lengths, if known.  scale: 1 / sqrt(head_dim).  q is of the cache's type; over a cache in 4 bits
    (fp4.Fp4Cache) of any of the three."""
    B, T, H, D = q.shape
    sq, at, fp4 = q.stride(), cache._device, cache.dtype is None
    code = DTYPES.get(q.dtype) if fp4 else cache._code
    if (code is None if fp4 else q.dtype is not cache.dtype) or D != cache.head_dim or sq[3] != 1 or q.get_device() != at:
        raise ValueError(f"q: a device tensor [B, T, heads, {cache.head_dim}] of {cache.dtype or 'fp32, bf16 or fp16'} with a contiguous last dimension is wanted")
    if out is None:
        out = torch.empty_like(q) if q.is_contiguous() else q.new_empty(B, T, H, D)
    elif out.shape != q.shape or out.dtype is not q.dtype or out.stride(3) != 1 or out.get_device() != at:
        raise ValueError("out: of q's shape and type, with a contiguous last dimension")
    W, so = (T + 31) // 32, out.stride()
    one = mask.shape[0] == 1
    m = _ints("mask", mask, (1 if one else B, T, W), at)
    bound = cache.max_length
    if 0 < max_length < bound:
        bound = max_length
    L = cache._lib
    n = cache._workspaces.get((B, T, H, bound, code))
    if n is None:
        n = (L.specdec_packed_attention_workspace if fp4 else L.specdec_tree_attention_workspace)(B, T, H, cache.n_heads, D, code, cache._page, bound)
        if n < 0:
            _fail(n)
        if len(cache._workspaces) > 4096:
            cache._workspaces.clear()
        cache._workspaces[B, T, H, bound, code] = n
    ws = torch.empty(n, dtype=torch.uint8, device=q.device) if n else None
    try:
        a = _attention_args.pack(q.data_ptr(), out.data_ptr(), sq[0], sq[1], sq[2], so[0], so[1], so[2], B, T, H, layer, _ints("seqs", seqs, (B,), at), m,
                                 0 if one else T * W, 0 if n_nodes is None else _ints("n_nodes", n_nodes, (B,), at), bound, D ** -0.5 if scale is None else scale,
                                 ws.data_ptr() if n else 0, n)
    except struct.error as e:
        raise ValueError(f"layer or scale: {e}") from None
    if fp4:
        _launch(L.specdec_packed_attention, at, (cache._ref, a, code, _raw_stream(at)))
    else:
        _launch(L.specdec_tree_attention, at, (cache._ref, a, _raw_stream(at)))
    if (q.requires_grad or cache._source is not None) and torch.is_grad_enabled():
        return _NoGradient.apply(out, "tree.attention", q, cache._source)
    return out


def sample(logits, uniform, temperature=None, top_k=None, top_p=None, min_p=None):
    """One token for each row of logits [..., V] (the last dimension contiguous, rows evenly spaced) from uniform [...] fp32 in [0, 1): (token int32 [...], log
    probability fp32 [...]).  The parameters (fp32, top_k int32; None: off) are tensors of one entry for each row, or for each equal run of rows ([n] for logits [n, T, V])."""
    shape = logits.shape
    V, lead = shape[-1], shape[:-1]
    code, at = DTYPES.get(logits.dtype), logits.get_device()
    if code is None or not logits.is_cuda or (logits.stride(-1) != 1 and V != 1):
        raise ValueError("logits: a device tensor of fp32, bf16 or fp16 with a contiguous last dimension is wanted")
    if uniform.shape != lead or uniform.dtype is not torch.float32 or uniform.get_device() != at or not uniform.is_contiguous():
        raise ValueError("uniform: a contiguous fp32 device tensor, one number a row, is wanted")
    rows, stride = uniform.numel(), V
    if not logits.is_contiguous():
        logits = logits if len(shape) == 2 else logits.reshape(-1, V)
        stride = logits.stride(0) if rows > 1 else V
    n, ptrs = 0, [None] * 4
    for i, t in enumerate((temperature, top_k, top_p, min_p)):
        if t is not None:
            m = t.numel()
            if t.dtype is not (_I32 if i == 1 else torch.float32) or t.get_device() != at or not t.is_contiguous() or m < 1 or rows % m or (n and n != m):
                raise ValueError(("temperature", "top_k", "top_p", "min_p")[i] + ": a contiguous fp32 (top_k: int32) device tensor is wanted, one entry for each "
                                 "equal run of rows, as many as the other parameters")
            n = m
            ptrs[i] = t.data_ptr()
    logprob = torch.empty_like(uniform)
    token = torch.empty_like(uniform, dtype=_I32)
    _launch(lib().specdec_sample, at, (logits.data_ptr(), code, stride, rows, V, uniform.data_ptr(), *ptrs, rows // n if n and rows else 1, token.data_ptr(), logprob.data_ptr(), _raw_stream(at)))
    if (logits.requires_grad or (temperature is not None and temperature.requires_grad)) and torch.is_grad_enabled():
        logprob = _NoGradient.apply(logprob, "tree.sample", logits, temperature)
    return token, logprob
