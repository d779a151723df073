"""Beam search on the caller's own tensors: the best continuations of a sentence's beams over the whole vocabulary.  With a cache's reorder (tree.PagedCache, fp4.Fp4Cache) behind it a step is

    cache.reserve(seqs.view(-1), 1)
    ...                                                      # append and tree.attention in every layer: one node a beam
    cache.compact(seqs.view(-1), path, n_path)
    scores, parent, token = beam.select(logits, scores, K, finished=finished, end_token=eos, norm=norm)
    cache.reorder(seqs, parent)                              # seqs [B, K]

Every call runs on the tensors' device, on its current stream, and returns without waiting for it (contracts: include/specdec.h)."""
from __future__ import annotations

import ctypes as C
import struct

import torch

from . import tree
from .binding import BeamSelectArgs
from .tree import DTYPES, _I32, _NoGradient, _fail, _launch

_workspaces = {}                                             # bytes by sizes of a call
_args = struct.Struct("@PPPPPPPPqqiiiiii")                   # BeamSelectArgs in one go
assert _args.size == C.sizeof(BeamSelectArgs)


def _rows(name, t, shape, dtype, at):
    if t.shape != shape or t.dtype is not dtype or t.get_device() != at or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous {dtype} tensor [B, K] is wanted beside the logits")
    return t.data_ptr()


def select(logits, scores, n: int, *, finished=None, end_token: int = 0, norm=None):
    """The n best continuations of each sentence: (scores fp32 [B, n], parent int32 [B, n], token int32 [B, n]), best first, of logits [B, K, V] (fp32, bf16 or fp16; the last dimension contiguous,
    rows evenly spaced) behind beams of scores [B, K] (fp32; -inf: no beam).  A beam that has finished (bool [B, K]) goes on as it is, with end_token.  norm (fp32 [B, K]): continuations are ranked by
    score * norm, as a length penalty has it; the scores that come out are without it.  Where there are fewer continuations: -inf, -1, -1."""
    if logits.dim() != 3:
        raise ValueError("logits: [B, K, V] is wanted")
    shape = logits.shape
    B, K, V = shape
    code, at = DTYPES.get(logits.dtype), logits.get_device()
    if code is None or not logits.is_cuda or (logits.stride(2) != 1 and V != 1):
        raise ValueError("logits: a device tensor of fp32, bf16 or fp16 with a contiguous last dimension is wanted")
    stride = V
    if not logits.is_contiguous():
        s = logits.stride()
        if B == 1 or K == 1:
            stride = s[1] if B == 1 else s[0]
        elif s[0] == K * s[1]:
            stride = s[1]
        else:
            raise ValueError("logits: evenly spaced rows are wanted")
    pair = shape[:2]
    p_scores = _rows("scores", scores, pair, torch.float32, at)
    p_finished = 0 if finished is None else _rows("finished", finished, pair, torch.bool, at)
    p_norm = 0 if norm is None else _rows("norm", norm, pair, torch.float32, at)
    lib = tree.lib()
    size = _workspaces.get((B, K, V, n, code))
    if size is None:
        size = lib.specdec_beam_select_workspace(B, K, V, n, code)
        if size < 0:
            _fail(size)
        if len(_workspaces) > 4096:
            _workspaces.clear()
        _workspaces[B, K, V, n, code] = size
    m = B * n
    all_ = scores.new_empty(3 * m)                           # scores, parents, tokens
    p, ints = all_.data_ptr(), all_.view(_I32)
    out, parent, token = all_.as_strided((B, n), (n, 1)), ints.as_strided((B, n), (n, 1), m), ints.as_strided((B, n), (n, 1), 2 * m)
    ws = scores.new_empty(size // 4)
    try:
        a = _args.pack(logits.data_ptr(), p_scores, p_finished, p_norm, p, p + 4 * m, p + 8 * m, ws.data_ptr(), size, stride, code, B, K, V, n, end_token)
    except struct.error as e:
        raise ValueError(f"end_token: {e}") from None
    _launch(lib.specdec_beam_select, at, (a, tree._raw_stream(at)))
    if (logits.requires_grad or scores.requires_grad or (norm is not None and norm.requires_grad)) and torch.is_grad_enabled():
        out = _NoGradient.apply(out, "beam.select", logits, scores, norm)
    return out, parent, token
