"""Tree speculation with sampling, end to end: a small decoder whose cache, trees, sampling and acceptance are the operators of `tree`.

    python -m paper_2203_16487_b200.tree_decode [--batch 8] [--tokens 64] [--dtype fp32|bf16]

Every step drafts a tree of seven continuations of the last token from a table of likely successors, scores all of its nodes at once, samples a token at every node from a
random number that belongs to the node's position, and keeps the branch that the samples follow.  As the numbers belong to positions, the text is the one that
sampling token by token gives, which the command checks: the tree changes how many steps it takes, not what comes out.  The weights are random (the text means nothing), drawn so
that a token mostly decides its successor."""
from __future__ import annotations

import argparse

import torch

from . import tree

PARENTS = [-1, 0, 0, 0, 1, 1, 4, 2]                            # a node's parent, and which of the parent's likely successors it is
RANK = [0, 0, 1, 2, 0, 1, 0, 0]


class Decoder:
    """Pre-norm decoder with grouped heads and learned positions; keys and values go to a tree.PagedCache."""

    def __init__(self, *, vocab=1000, d=256, heads=8, kv_heads=2, layers=3, positions=512, dtype=torch.float32, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        rand = lambda *s, std: (torch.randn(*s, generator=g, device=device) * std).to(dtype)  # noqa: E731
        self.vocab, self.d, self.heads, self.kv_heads, self.n_layers, self.head_dim, self.dtype, self.device = vocab, d, heads, kv_heads, layers, d // heads, dtype, device
        self.embed, self.pos, self.head = rand(vocab, d, std=1.0), rand(positions, d, std=0.05), rand(d, vocab, std=0.35)
        kv = kv_heads * self.head_dim
        self.layers = [dict(qkv=rand(d, d + 2 * kv, std=d ** -0.5), o=rand(d, d, std=0.3 * d ** -0.5), up=rand(d, 2 * d, std=d ** -0.5), down=rand(2 * d, d, std=0.3 * d ** -0.5))
                       for _ in range(layers)]

    def cache(self, n_seqs, tokens, page_tokens=16):
        pages = -(-tokens // page_tokens)
        return tree.PagedCache(self.n_layers, self.kv_heads, self.head_dim, n_pages=n_seqs * pages, n_seqs=n_seqs, max_pages=pages, page_tokens=page_tokens,
                               dtype=self.dtype, device=self.device)

    def logits(self, tokens, positions, cache, seqs, mask):
        """Logits [B, T, vocab] of the nodes; their keys and values are in the cache behind the committed tokens (reserve them first)."""
        B, T = tokens.shape
        norm = lambda x: torch.nn.functional.layer_norm(x.float(), (self.d,)).to(self.dtype)  # noqa: E731
        x = self.embed[tokens.long()] + self.pos[positions.long()]
        kv = self.kv_heads * self.head_dim
        for i, w in enumerate(self.layers):
            q, k, v = (norm(x) @ w["qkv"]).split((self.d, kv, kv), dim=-1)
            cache.append(seqs, k.unflatten(-1, (self.kv_heads, -1)), v.unflatten(-1, (self.kv_heads, -1)), layer=i)
            x = x + tree.attention(q.unflatten(-1, (self.heads, -1)), cache, i, seqs, mask).flatten(2) @ w["o"]
            x = x + torch.relu(norm(x) @ w["up"]) @ w["down"]
        return norm(x) @ self.head


def successors(model, n=3):
    """The n likeliest tokens behind each token, as the model sees it alone: what the drafts are taken from."""
    V, one = model.vocab, torch.ones(model.vocab, 1, 1, dtype=torch.int32, device=model.device)
    cache, seqs = model.cache(V, 1), torch.arange(V, dtype=torch.int32, device=model.device)
    cache.reserve(seqs, 1)
    tokens = seqs[:, None]
    return model.logits(tokens, torch.zeros_like(tokens), cache, seqs, one)[:, 0].topk(n).indices.int()


def decode(model, prompt, n_tokens, uniform, *, drafts=True, table=None, temperature=0.8, top_k=50, top_p=0.95, min_p=0.0):
    """n_tokens sampled tokens behind each prompt [B, S] (int32) and the number of steps.  uniform [B, S + n_tokens + a tree's depth]: the random number of each
    position.  drafts=False: one token a step.  table: successors(model)."""
    dev, (B, S) = model.device, prompt.shape
    i32 = dict(dtype=torch.int32, device=dev)
    parents = torch.tensor(PARENTS if drafts else [-1], **i32).expand(B, -1).contiguous()
    rank = RANK if drafts else [0]
    T, seqs = parents.shape[1], torch.arange(B, **i32)
    cache = model.cache(B, S + n_tokens + 2 * T)
    params = [torch.full((B,), v, dtype=torch.int32 if i == 1 else torch.float32, device=dev) for i, v in enumerate((temperature, top_k, top_p, min_p))]
    if S > 1:                                                  # the prompt but its last token, which is the first root: a chain, all of it kept
        chain = torch.arange(-1, S - 2, **i32).expand(B, -1).contiguous()
        mask, depth = tree.ancestors(chain)
        cache.reserve(seqs, S - 1)
        model.logits(prompt[:, :-1], depth, cache, seqs, mask)
        cache.compact(seqs, depth, torch.full((B,), S - 1, **i32))
    mask, depth = tree.ancestors(parents)                      # the same tree in every step
    tokens = torch.zeros(B, T, **i32)
    tokens[:, 0] = prompt[:, -1]
    out, count, steps = torch.zeros(B, n_tokens + T, **i32), torch.zeros(B, dtype=torch.long, device=dev), 0
    while int(count.min()) < n_tokens:
        for i in range(1, T):
            tokens[:, i] = table[tokens[:, PARENTS[i]].long(), rank[i]]
        cache.reserve(seqs, T)
        at = cache.length[:, None] + depth
        logits = model.logits(tokens, at, cache, seqs, mask)
        sampled, _ = tree.sample(logits, uniform.gather(1, at.long()), *params)
        path, n_path, emitted = tree.accept(parents, tokens, sampled)
        n_path = torch.minimum(n_path, (n_tokens - count).clamp(min=0).int())      # (a finished sequence keeps nothing more)
        cache.compact(seqs, path, n_path)
        new = torch.arange(T, device=dev) < n_path[:, None]
        out.scatter_(1, torch.where(new, count[:, None] + torch.arange(T, device=dev), n_tokens + T - 1), torch.where(new, emitted, 0))
        count += n_path
        last = emitted.gather(1, (n_path.long() - 1).clamp(min=0)[:, None])[:, 0]
        tokens[:, 0] = torch.where(n_path > 0, last, tokens[:, 0])
        steps += 1
    cache.check()
    return out[:, :n_tokens], steps


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=12)
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--dtype", choices=("fp32", "bf16"), default="fp32")
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args(argv)
    model = Decoder(dtype=torch.float32 if a.dtype == "fp32" else torch.bfloat16, seed=a.seed, positions=a.prompt + a.tokens + 32)
    g = torch.Generator(device="cuda").manual_seed(a.seed + 1)
    prompt = torch.randint(0, model.vocab, (a.batch, a.prompt), generator=g, device="cuda").int()
    uniform = torch.rand(a.batch, a.prompt + a.tokens + 32, generator=g, device="cuda")
    table = successors(model)
    plain, steps = decode(model, prompt, a.tokens, uniform, drafts=False)
    fast, fewer = decode(model, prompt, a.tokens, uniform, table=table)
    same = float((plain == fast).float().mean())
    print(f"{a.batch} sequences of {a.tokens} tokens: {steps} steps token by token, {fewer} with trees of {len(PARENTS)} nodes; the same tokens: {100 * same:.1f} %")
    print(fast[0].tolist())
    return steps, fewer, same


if __name__ == "__main__":
    main()
