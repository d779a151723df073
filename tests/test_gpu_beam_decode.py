"""Beam search through a model: cache, attention, selection and reordering together, against the same search without a cache."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def plain(model, prompt, n_tokens, K, end_token, alpha):
    """The same search with the whole text of every beam scored anew in each step, in 64 bits; also, for each sentence, the least distance between ranks that decided anything."""
    w = {k: v.double() for k, v in (("embed", model.embed), ("pos", model.pos), ("head", model.head))}
    layers = [{k: v.double() for k, v in l.items()} for l in model.layers]

    def logits(text):
        T = text.shape[1]
        norm = lambda x: torch.nn.functional.layer_norm(x, (model.d,))  # noqa: E731
        x = w["embed"][text] + w["pos"][:T]
        causal = torch.full((T, T), -math.inf, device=x.device, dtype=x.dtype).triu(1)
        kv = model.kv_heads * model.head_dim
        for l in layers:
            q, k, v = (norm(x) @ l["qkv"]).split((model.d, kv, kv), dim=-1)
            q = q.unflatten(-1, (model.heads, -1)).transpose(1, 2)
            k, v = (y.unflatten(-1, (model.kv_heads, -1)).repeat_interleave(model.heads // model.kv_heads, 2).transpose(1, 2) for y in (k, v))
            p = torch.softmax(q @ k.transpose(-1, -2) * model.head_dim ** -0.5 + causal, -1)
            x = x + (p @ v).transpose(1, 2).flatten(2) @ l["o"]
            x = x + torch.relu(norm(x) @ l["up"]) @ l["down"]
        return norm(x[:, -1]) @ w["head"]

    out, leasts = [], []
    for b in range(prompt.shape[0]):
        beams, least = [(0.0, [], False)], math.inf
        for _ in range(n_tokens):
            text = torch.stack([torch.tensor(prompt[b].tolist() + t, device=prompt.device) for _, t, _ in beams])
            logp = torch.log_softmax(logits(text), -1).cpu()
            found = []
            for i, (s, t, done) in enumerate(beams):
                n = sum(x != end_token for x in t) + (not done)
                f = ((5 + n) / 6) ** -alpha
                if done:
                    found.append((s * f, i, s, t + [end_token], True))
                else:
                    v, at = logp[i].topk(K + 1)
                    found += [((s + x) * f, i, s + x, t + [j], j == end_token) for x, j in zip(v.tolist(), at.tolist())]
            found.sort(key=lambda c: (-c[0], c[1]))
            least = min([least] + [x[0] - y[0] for x, y in zip(found[:K], found[1:K + 1])])
            beams = [(s, t, done) for _, _, s, t, done in found[:K]]
        out.append(beams)
        leasts.append(least)
    return out, leasts


@pytest.mark.parametrize("K,S,end_token", [(1, 5, 0), (4, 12, 0), (5, 40, 7)])
def test_beams_are_those_of_a_search_without_a_cache(K, S, end_token):
    """fp32: log probabilities are off by some 1e-5 (three layers of sums of 512 products, of 20 tokens), so ranks further apart than 1e-4 decide alike; of six sentences some have none nearer."""
    from paper_2203_16487_b200 import beam_decode
    from paper_2203_16487_b200.tree_decode import Decoder
    model = Decoder(d=512, vocab=300, seed=K, positions=S + 24)
    g = torch.Generator(device="cuda").manual_seed(K)
    prompt = torch.randint(1, 300, (6, S), generator=g, device="cuda").int()
    tokens, scores = beam_decode.decode(model, prompt, 20, K, end_token=end_token)
    want, leasts = plain(model, prompt, 20, K, end_token, 0.6)
    assert max(leasts) > 1e-4
    for b, (beams, least) in enumerate(zip(want, leasts)):
        if least > 1e-4:
            for k, (s, t, _) in enumerate(beams):
                assert abs(float(scores[b, k]) - s) < 1e-3 and tokens[b, k].tolist() == t, (b, k)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_the_command_runs_with_both_caches(dtype):
    from paper_2203_16487_b200 import beam_decode
    full, scores, small, held = beam_decode.main(["--batch", "3", "--tokens", "20", "--dtype", dtype])
    assert full.shape == small.shape == (3, 4, 20) and scores.isfinite().all() and held.isfinite().all() and (full >= 0).all() and (small >= 0).all()
