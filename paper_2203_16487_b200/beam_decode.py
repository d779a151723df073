"""Beam search, end to end: the small decoder of `tree_decode` over a cache of 16 or 32 bits or of 4, with the operators of `tree`, `fp4` and `beam`.

    python -m paper_2203_16487_b200.beam_decode [--batch 4] [--beams 4] [--tokens 48] [--dtype fp32|bf16]

The prompt fills one beam's cache, and a reordering makes all beams continue it.  Every step writes and scores one token a beam, selects the best continuations of each sentence, and reorders the cache by
their parents; a beam that has emitted the end token goes on as it is, and beams are ranked by score over a power of their length.  The command decodes with both caches and says how far they agree.  The
weights are random (the text means nothing)."""
from __future__ import annotations

import argparse
import math

import torch

from . import beam, fp4
from .tree_decode import Decoder


def cache_of(model, n_seqs, tokens, four_bits=False, page_tokens=16):
    if not four_bits:
        return model.cache(n_seqs, tokens, page_tokens)
    pages = -(-tokens // page_tokens)
    return fp4.Fp4Cache(model.n_layers, model.kv_heads, model.head_dim, n_pages=n_seqs * pages, n_seqs=n_seqs, max_pages=pages, page_tokens=page_tokens, device=model.device)


def decode(model, prompt, n_tokens, beams=4, *, four_bits=False, end_token=0, alpha=0.6):
    """The beams of each prompt [B, S] (int32) after n_tokens steps, best first: (tokens [B, K, n_tokens], end_token behind a beam's end, and scores [B, K]: sums of log probabilities)."""
    dev, (B, S), K = model.device, prompt.shape, beams
    i32 = dict(dtype=torch.int32, device=dev)
    seqs = torch.arange(B * K, **i32).view(B, K)
    flat, first, one = seqs.view(-1), seqs[:, 0].contiguous(), torch.ones(1, 1, 1, **i32)
    cache = cache_of(model, B * K, S + n_tokens, four_bits)
    if S > 1:                                                  # the prompt but its last token, a chain, into the first beam; the others take over its pages
        words = torch.tensor([[(1 << min(max(t + 1 - 32 * w, 0), 32)) - 1 for w in range((S + 30) // 32)] for t in range(S - 1)])
        mask = torch.where(words >= 1 << 31, words - (1 << 32), words).to(**i32)[None].contiguous()
        depth = torch.arange(S - 1, **i32).expand(B, -1).contiguous()
        cache.reserve(first, S - 1)
        model.logits(prompt[:, :-1], depth, cache, first, mask)
        cache.compact(first, depth, torch.full((B,), S - 1, **i32))
        cache.reorder(seqs, torch.zeros(B, K, **i32))
    scores = torch.full((B, K), -math.inf, device=dev)
    scores[:, 0] = 0
    tokens, out = prompt[:, -1:].expand(B, K).contiguous(), torch.empty(B, K, 0, **i32)
    finished = torch.zeros(B, K, dtype=torch.bool, device=dev)
    path, n_path = torch.zeros(B * K, 1, **i32), torch.ones(B * K, **i32)
    for _ in range(n_tokens):
        cache.reserve(flat, 1)
        logits = model.logits(tokens.view(-1, 1), cache.length[:, None], cache, flat, one)
        cache.compact(flat, path, n_path)
        length = (~finished * 1.0).add_((out != end_token).sum(-1))       # of each beam's continuations
        scores, parent, token = beam.select(logits.view(B, K, -1), scores, K, finished=finished, end_token=end_token, norm=((5 + length) / 6) ** -alpha)
        cache.reorder(seqs, parent)
        at = parent.clamp(min=0).long()
        out = torch.cat((out.gather(1, at[..., None].expand(-1, -1, out.shape[2])), token[..., None]), 2)
        finished = finished.gather(1, at) | (token == end_token)
        tokens = token.clamp(min=0)
    cache.check()
    return out, scores


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--beams", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=12)
    ap.add_argument("--tokens", type=int, default=48)
    ap.add_argument("--dtype", choices=("fp32", "bf16"), default="fp32")
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args(argv)
    model = Decoder(d=512, dtype=torch.float32 if a.dtype == "fp32" else torch.bfloat16, seed=a.seed, positions=a.prompt + a.tokens)
    g = torch.Generator(device="cuda").manual_seed(a.seed + 1)
    prompt = torch.randint(1, model.vocab, (a.batch, a.prompt), generator=g, device="cuda").int()
    full, scores = decode(model, prompt, a.tokens, a.beams)
    small, held = decode(model, prompt, a.tokens, a.beams, four_bits=True)
    same = float((full[:, 0] == small[:, 0]).float().mean())
    print(f"{a.batch} sentences of {a.tokens} tokens with {a.beams} beams: best scores {[round(x, 2) for x in scores[:, 0].tolist()]}, with the cache in 4 bits "
          f"{[round(x, 2) for x in held[:, 0].tolist()]}; tokens alike: {100 * same:.1f} %")
    print(full[0, 0].tolist())
    return full, scores, small, held


if __name__ == "__main__":
    main()
