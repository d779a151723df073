"""Performance cases of beam search and of the cache in 4 bits: the attention over that cache, writing and reading it, selecting beams, reordering the cache.

A case is one call of the package's operators on the caller's tensors (append: writing tokens and reading them back):

  attention  queries of a tree of drafted tokens (one token: plain decoding) over a cache of 4-bit values, cached tokens and their ancestors
  append     keys and values of new tokens to 4 bits, and back to 16 or 32
  select     the best continuations of a sentence's beams over the whole vocabulary
  reorder    beams take over the cached tokens of the beams that they continue

`own` chooses between the framework's calls and the same operators written as elementary torch operations.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZES = {"bf16": 2, "f16": 2, "f32": 4}
BLOCK = 16                          # channels that share a scale
HELD = 9 / 16                       # bytes of a value: 4 bits and its part of a scale's 8


def listed():
    att = dict(kind="attention", page=16)
    return [
        # one sentence of the online translation setting: last token and k = 25 drafts, 8 heads of 64; latency counts
        dict(att, name="attention_sentence", batch=1, nodes=26, heads=8, kv_heads=8, dim=64, lo=64, hi=64, dtype="bf16"),
        # 128 ragged sequences of the offline setting, k = 50
        dict(att, name="attention_batch", batch=128, nodes=51, heads=8, kv_heads=8, dim=64, lo=0, hi=256, dtype="bf16"),
        # the beams of a few documents, one token each, over long caches with grouped heads
        dict(att, name="attention_decode_long", batch=4, nodes=1, heads=32, kv_heads=8, dim=128, page=64, lo=65537, hi=131071, dtype="f16"),
        # trees over long documents with grouped heads: the most arithmetic
        dict(att, name="attention_tree_long", batch=8, nodes=64, heads=32, kv_heads=8, dim=128, page=64, lo=8191, hi=16385, dtype="bf16"),
        # fp32 models over summarisation-length sources
        dict(att, name="attention_f32", batch=8, nodes=9, heads=8, kv_heads=8, dim=64, lo=300, hi=512, dtype="f32"),
        # the block of one step of 32 sentences: 6 layers, 8 heads of 64
        dict(kind="append", name="append_step", batch=32, nodes=26, layers=6, kv_heads=8, dim=64, page=16, lo=40, hi=300, dtype="bf16"),
        # eight long prompts, all layers
        dict(kind="append", name="append_prompt", batch=8, nodes=509, layers=32, kv_heads=8, dim=128, page=64, lo=0, hi=0, dtype="bf16"),
        # one sentence, four beams
        dict(kind="select", name="select_sentence", batch=1, beams=4, vocab=32768, n=8, dtype="f32", ended=False),
        # 128 sentences, eight beams and twice as many candidates
        dict(kind="select", name="select_batch", batch=128, beams=8, vocab=32768, n=16, dtype="bf16", ended=False),
        # an odd vocabulary, beams that have ended, a length penalty
        dict(kind="select", name="select_odd", batch=32, beams=5, vocab=50265, n=5, dtype="f32", ended=True),
        # four beams of each of 32 sentences: 6 layers, 8 heads of 64
        dict(kind="reorder", name="reorder_step", held="16", batch=32, beams=4, layers=6, kv_heads=8, dim=64, page=16, lo=40, hi=300, dtype="bf16"),
        # eight beams of four documents: 32 layers in pages of 128 tokens, held in 4 bits
        dict(kind="reorder", name="reorder_long", held="4", batch=4, beams=8, layers=32, kv_heads=8, dim=128, page=128, lo=700, hi=1023, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attention"] * 5 + ["append"] * 2 + ["select"] * 3 + ["reorder"] * 2)
    if kind == "attention":
        c = dict(kind=kind, page=rng.choice([16, 32, 64, 128]), nodes=rng.choice([1, _log_int(rng, 2, 128), _log_int(rng, 2, 128)]),
                 dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), dim=rng.choice([64, 128]), kv_heads=rng.choice([1, 2, 4, 8, 12]))
        group = rng.choice([1, 1, 2, 4, 8]) if c["kv_heads"] < 12 else 1
        c["heads"] = c["kv_heads"] * group
        hi = _log_int(rng, 16, 100000)
        products = 2e10 if c["dtype"] != "f32" else 2e9
        hi = max(16, min(hi, int(products / (c["heads"] * c["nodes"] * c["dim"])), int(2.5e8 / (c["heads"] * c["nodes"]))))
        c["batch"] = max(1, min(_log_int(rng, 1, 128), int(products / (c["heads"] * c["nodes"] * hi * c["dim"])),
                                int(2.5e8 / (c["heads"] * c["nodes"] * hi)), int(2e8 / (hi * c["kv_heads"] * c["dim"]))))
        c.update(lo=rng.randint(0, hi), hi=hi)
        return c
    if kind == "select":
        c = dict(kind=kind, vocab=rng.choice([1000, 32768, 50265, _log_int(rng, 1000, 131072)]), dtype=rng.choice(["bf16", "f16", "f32", "f32"]), beams=rng.randint(1, 12),
                 ended=rng.choice([False, True]))
        c["n"] = rng.choice([c["beams"], 2 * c["beams"], 2 * c["beams"] + 1])
        c["batch"] = max(1, min(_log_int(rng, 1, 128), int(3.3e7 // (c["vocab"] * c["beams"]))))
        return c
    c = dict(kind=kind, layers=rng.choice([2, 6, 12, 32]), kv_heads=rng.choice([1, 8, 12]), dim=rng.choice([64, 128]), page=rng.choice([16, 32, 64, 128]),
             dtype=rng.choice(["bf16", "f16", "f32"]))
    token = c["layers"] * c["kv_heads"] * c["dim"]
    hi = _log_int(rng, 16, 2000)
    if kind == "append":
        c["nodes"] = min(_log_int(rng, 1, 1000), int(1.2e8 // token))
        c["batch"] = max(1, min(_log_int(rng, 1, 64), int(1.2e8 / (token * (hi + c["nodes"] + c["page"])))))
    else:
        c.update(held=rng.choice(["16", "4"]), beams=rng.randint(1, 12))
        hi = max(16, min(hi, int(4e8 / (token * c["beams"])) - c["page"]))
        c["batch"] = max(1, min(_log_int(rng, 1, 64), int(4e8 / (token * c["beams"] * (hi + c["page"])))))
    c.update(lo=rng.randint(1, hi), hi=hi)
    return c


# ------------------------------------------------------------------------------------------------ 4 bits
def _blocks(x):
    """Scales [..., D / 16] and codes as numbers [..., D / 16, 16] of x [..., D] in fp32: the scale takes the block's largest value to 6, rounded to 8 bits (4 of
    exponent, 3 of fraction); a code is the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives, halfway to the one of even number."""
    x = x.unflatten(-1, (-1, BLOCK))
    top = x.abs().amax(-1)
    scale = (top / torch.full_like(top, 6)).clamp(max=448).to(torch.float8_e4m3fn)       # (by a number: a product with 1 / 6, which rounds twice)
    r = x / scale.float()[..., None]
    a = r.abs()
    number = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)      # (0 / 0: 0)
    return scale, number + 8 * (x < 0).to(torch.uint8)


def _pack4(x):
    """(codes [..., D / 2] uint8, scales [..., D / 16]) of x [..., D]: channel 2 i in the low four bits of byte i."""
    scale, number = _blocks(x)
    number = number.flatten(-2)
    return number[..., ::2] | number[..., 1::2] << 4, scale


def _values4(codes, scales):
    """fp32 values [..., D] of codes [..., D / 2] and scales [..., D / 16]."""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=codes.device)
    number = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    value = torch.where(number >= 8, -1.0, 1.0) * table[(number & 7).int()]
    return (value.unflatten(-1, (-1, BLOCK)) * scales.float()[..., None]).flatten(-2)


# ------------------------------------------------------------------------------------------------ inputs
def _lengths(c, n):
    """Cached tokens of each sequence: by the case alone, as its work is."""
    r = random.Random(c["lo"] * 1000003 + c["hi"] * 101 + n)
    return [c["hi"]] + [r.randint(c["lo"], c["hi"]) for _ in range(n - 1)]


def _nodes(c, n):
    """Nodes of each tree: full ones, and for every third sequence fewer."""
    return [c["nodes"] if b % 3 < 2 else max(1, c["nodes"] - b % 7) for b in range(n)]


def _parents_of(c):
    """The beam that each beam of each sentence continues: a few good ones have several successors, and some have none."""
    r = random.Random(c["batch"] * 1009 + c["beams"] * 31 + c["hi"])
    return [[min(int(r.expovariate(2.5 / c["beams"])), c["beams"] - 1) for _ in range(c["beams"])] for _ in range(c["batch"])]


def _closure(parents):
    """[B, T, T]: node j is node i or one of its ancestors."""
    i = torch.arange(parents.shape[1], device=parents.device)
    up = (parents.long()[:, :, None] == i) | (i[:, None] == i)
    return torch.linalg.matrix_power(up.double() / 2, max(1, parents.shape[1] - 1)) > 0    # the halves keep counts of paths in range


def _words(see):
    """Bits of a [B, T, T] mask: word w, bit j is node 32 w + j."""
    b, t, _ = see.shape
    w = (t + 31) // 32
    bits = torch.nn.functional.pad(see, (0, 32 * w - t)).view(b, t, w, 32).long()
    words = (bits << torch.arange(32, device=see.device)).sum(-1)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).int()


def _book(c, g, lengths, held, spare, width):
    """The bookkeeping of a cache whose sequences hold `held` pages each, scattered over the pool; `spare` more pages are free."""
    pages, n = sum(held) + spare, len(held)
    order = torch.randperm(pages, generator=g, device="cuda").int()[:sum(held)]
    table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    h = torch.tensor(held, device="cuda")
    table[torch.arange(width, device="cuda") < h[:, None]] = order
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    refs[order.long()] = 1
    return dict(table=table, length=torch.tensor(lengths, dtype=torch.int32, device="cuda"), held=h.int(), refs=refs)


def _codes(c, g, pages, layers, fill=True):
    """A pool in 4 bits: codes [layers, 2, pages, kv_heads, page, dim / 2], scales [.., dim / 16], of normal values."""
    shape = (layers, 2, pages, c["kv_heads"], c["page"])
    codes = torch.zeros(*shape, c["dim"] // 2, dtype=torch.uint8, device="cuda")
    scales = torch.zeros(*shape, c["dim"] // BLOCK, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    if fill:
        step = max(1, int(6e7 // (c["kv_heads"] * c["page"] * c["dim"])))
        for layer in range(layers):
            for side in range(2):
                for p in range(0, pages, step):
                    x = torch.randn(min(step, pages - p), *shape[3:], c["dim"], generator=g, device="cuda")
                    codes[layer, side, p:p + step], s = _pack4(x)
                    scales.view(torch.uint8)[layer, side, p:p + step] = s.view(torch.uint8)
    return dict(codes=codes, scales=scales)


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s, dt = {"case": c}, DTYPES[c["dtype"]]
    pages_of = lambda n: -(-n // c["page"])  # noqa: E731
    if c["kind"] == "attention":
        b, t = c["batch"], c["nodes"]
        lengths = _lengths(c, b)
        held = [pages_of(n + t) for n in lengths]
        s["pool"] = _book(c, g, lengths, held, 1, max(held))
        s["pool"].update(_codes(c, g, sum(held) + 1, 1))
        s["q"] = (torch.randn(b, t, c["heads"], c["dim"], generator=g, device="cuda") * 2).to(dt)
        i = torch.arange(t, device="cuda")                                  # random trees: a node hangs off one of the eight before it
        back = (torch.rand(b, t, generator=g, device="cuda") * torch.clamp(i, max=8)).long()
        s["mask"] = _words(_closure(torch.where(i > 0, i - 1 - back, -1).int()))
        s["n_nodes"] = torch.tensor(_nodes(c, b), dtype=torch.int32, device="cuda")
        s["seqs"] = torch.arange(b, dtype=torch.int32, device="cuda")
        s["max_length"] = c["hi"]
    elif c["kind"] == "append":
        b, t = c["batch"], c["nodes"]
        lengths = _lengths(c, b)
        held = [pages_of(n + t) for n in lengths]
        s["pool"] = _book(c, g, lengths, held, 0, max(held))
        s["pool"].update(_codes(c, g, sum(held), c["layers"], fill=False))
        s["seqs"] = torch.arange(b, dtype=torch.int32, device="cuda")
        shape = (c["layers"], b, t, c["kv_heads"], c["dim"])
        s["k"] = torch.randn(shape, generator=g, device="cuda", dtype=dt)
        s["k"][..., 5] *= 8                                                 # the channels of keys that are larger than the others
        s["v"] = torch.randn(shape, generator=g, device="cuda", dtype=dt)
    elif c["kind"] == "select":
        b, k, v = c["batch"], c["beams"], c["vocab"]
        logits = torch.randn(b * k, v, generator=g, device="cuda") * 2
        at = torch.randint(4, v, (b * k, 32), generator=g, device="cuda")
        logits.scatter_add_(1, at, 5 + 4 * torch.rand(b * k, 32, generator=g, device="cuda"))     # the tokens that fit
        logits[:, 0] = -math.inf                                            # padding is never written
        s["logits"] = logits.to(dt).view(b, k, v)
        s["scores"] = -40 * torch.rand(b, 1, generator=g, device="cuda") - 3 * torch.rand(b, k, generator=g, device="cuda")
        s["finished"] = s["norm"] = None
        if c["ended"]:
            s["finished"] = torch.rand(b, k, generator=g, device="cuda") < 0.3
            s["norm"] = ((5 + torch.randint(5, 60, (b, k), generator=g, device="cuda")) / 6.0) ** -0.6        # the length penalty of each beam's continuations
    else:
        b, k = c["batch"], c["beams"]
        lengths = [n for n in _lengths(c, b) for _ in range(k)]
        held = [pages_of(n) for n in lengths]
        s["pool"] = _book(c, g, lengths, held, 3, max(held) + 1)
        if c["held"] == "4":
            s["pool"].update(_codes(c, g, sum(held) + 3, c["layers"]))
        else:
            s["pool"]["kv"] = torch.randn(c["layers"], 2, sum(held) + 3, c["page"], c["kv_heads"], c["dim"], generator=g, device="cuda", dtype=dt)
        s["seqs"] = torch.arange(b * k, dtype=torch.int32, device="cuda").view(b, k)
        s["parents"] = torch.tensor(_parents_of(c), dtype=torch.int32, device="cuda")
    if own and "pool" in s:
        from paper_2203_16487_b200 import fp4, tree
        s["cache"] = (tree.PagedCache if "kv" in s["pool"] else fp4.Fp4Cache).over(**s["pool"])
    return s


def _state(pool):
    """The cache as it is after a call; scales as the bytes that they are."""
    return {name: x.view(torch.uint8) if name == "scales" else x for name, x in pool.items()}


# ------------------------------------------------------------------------------------------------ the framework's calls
def _own(s):
    from paper_2203_16487_b200 import beam, tree
    c = s["case"]
    if c["kind"] == "attention":
        return tree.attention(s["q"], s["cache"], 0, s["seqs"], s["mask"], n_nodes=s["n_nodes"], max_length=s["max_length"])
    if c["kind"] == "append":
        s["cache"].append(s["seqs"], s["k"], s["v"])
        return s["cache"].read(s["seqs"], c["nodes"], dtype=s["k"].dtype)
    if c["kind"] == "select":
        return beam.select(s["logits"], s["scores"], c["n"], finished=s["finished"], end_token=2, norm=s["norm"])
    s["cache"].reorder(s["seqs"], s["parents"])
    return _state(s["pool"])


# ------------------------------------------------------------------------------------------------ plain forms
def _slots(table, pos, page):
    """Page and place in it of each position [n, T]."""
    return torch.gather(table, 1, (pos // page).long()).long(), (pos % page).long()


def _attention(s):
    c, pool = s["case"], s["pool"]
    t, h, n, d = c["nodes"], c["heads"], c["kv_heads"], c["dim"]
    length, nodes = pool["length"][s["seqs"].long()], s["n_nodes"]
    pos = torch.arange(s["max_length"] + t, device="cuda").expand(c["batch"], -1)
    there = pos < (length + nodes)[:, None]
    page, place = _slots(pool["table"][s["seqs"].long()], torch.where(there, pos, 0), c["page"])
    page = torch.where(there, page, 0)
    scales = pool["scales"].view(torch.uint8)
    k, v = (torch.where(there[:, :, None, None], _values4(pool["codes"][0, side][page, :, place], scales[0, side][page, :, place].view(torch.float8_e4m3fn)), 0)
            for side in range(2))
    node = (pos - length[:, None])[:, None, :].expand(-1, t, -1)
    at = node.clamp(0, t - 1).long()
    bit = (torch.gather(s["mask"].long(), 2, at // 32) >> (at % 32)) & 1
    see = there[:, None, :] & ((node < 0) | (bit > 0)) & (torch.arange(t, device="cuda") < nodes[:, None])[:, :, None]
    q = s["q"].float().view(c["batch"], t, n, h // n, d)
    score = torch.einsum("btngd,bsnd->bngts", q, k).mul_(1 / math.sqrt(d))
    score.masked_fill_(~see[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    score.sub_(torch.where(top > -math.inf, top, 0)).exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.einsum("bngts,bsnd->bngtd", score, v) / torch.where(total > 0, total, 1)
    return out.permute(0, 3, 1, 2, 4).reshape(c["batch"], t, h, d).to(s["q"].dtype)


def _append(s):
    pool, c, seqs = s["pool"], s["case"], s["seqs"].long()
    page, place = _slots(pool["table"][seqs], pool["length"][seqs][:, None] + torch.arange(c["nodes"], device="cuda"), c["page"])
    scales, out = pool["scales"].view(torch.uint8), []
    for side, x in enumerate((s["k"], s["v"])):
        back = torch.empty_like(x)
        for layer in range(c["layers"]):
            codes, scale = _pack4(x[layer].float())
            pool["codes"][layer, side][page, :, place], scales[layer, side][page, :, place] = codes, scale.view(torch.uint8)
            back[layer] = _values4(pool["codes"][layer, side][page, :, place], scales[layer, side][page, :, place].view(torch.float8_e4m3fn)).to(x.dtype)
        out.append(back)
    return tuple(out)


def _select(s):
    c, n = s["case"], s["case"]["n"]
    b, k, v = s["logits"].shape
    logit = s["logits"].double()                                   # 64 bits: candidates of different beams may lie next to one another
    top = logit.amax(-1, keepdim=True)
    x = logit - top
    logp = x - torch.log(torch.exp(x).sum(-1, keepdim=True))
    m = min(n, v)
    order = s["logits"].sort(dim=-1, descending=True, stable=True).indices[..., :m]
    score = s["scores"].double()[..., None] + logp.gather(-1, order)
    if s["finished"] is not None:                                  # a beam that has ended goes on as it is
        done, first = s["finished"][..., None], torch.arange(m, device="cuda") == 0
        score = torch.where(done, torch.where(first, s["scores"].double()[..., None], -math.inf), score)
        order = torch.where(done, 2, order)
    rank = score if s["norm"] is None else score * s["norm"].double()[..., None]
    rank, at = rank.view(b, -1).sort(dim=-1, descending=True, stable=True)
    rank, at = rank[:, :n], at[:, :n]
    there = rank > -math.inf
    out = [torch.where(there, x, none) for x, none in ((score.view(b, -1).gather(1, at).float(), -math.inf), ((at // m).int(), -1), (order.reshape(b, -1).gather(1, at).int(), -1))]
    if at.shape[1] < n:
        out = [torch.nn.functional.pad(x, (0, n - at.shape[1]), value=none) for x, none in zip(out, (-math.inf, -1, -1))]
    return tuple(out)


def _reorder(s):
    pool, c = s["pool"], s["case"]
    page, k = c["page"], c["beams"]
    seqs, parents = s["seqs"].long(), s["parents"].long()
    table, refs = pool["table"], pool["refs"]
    i = torch.arange(k, device="cuda")
    # the child that goes on with a beam's last page: the beam itself if it is one, else its first
    child = parents[:, None, :] == i[:, None]                                      # [B, beam, child]
    heir = torch.where(child.diagonal(dim1=1, dim2=2), i, child.int().argmax(2))
    heir = heir.gather(1, parents) == i                                            # of each child: whether it is its parent's heir
    src, dst, heir = seqs.gather(1, parents).view(-1), seqs.view(-1), heir.view(-1)
    rows, old, length = table[src], table[dst], pool["length"][src]
    at = torch.arange(table.shape[1], device="cuda")
    full, part = length // page, length % page
    keep = (at < full[:, None]) | ((at == full[:, None]) & (part > 0)[:, None] & heir[:, None])
    refs.scatter_add_(0, old.clamp(min=0).view(-1).long(), -(old >= 0).int().view(-1))
    refs.scatter_add_(0, rows.clamp(min=0).view(-1).long(), keep.int().view(-1))
    need = (~heir & (part > 0)).int()
    rank = need.cumsum(0) - need
    free = (refs == 0).int().sort(descending=True, stable=True).indices
    new = free[rank.long()].int()
    refs[free] += (torch.arange(free.numel(), device="cuda") < need.sum()).int()
    here = (at == full[:, None]) & (need > 0)[:, None]
    table[dst] = torch.where(keep, rows, torch.where(here, new[:, None], -1))
    pool["held"][dst], pool["length"][dst] = full + (part > 0).int(), length
    fro = rows.gather(1, full.clamp(max=table.shape[1] - 1).long()[:, None])[:, 0].clamp(min=0).long()
    move = (torch.arange(page, device="cuda") < part[:, None]) & (need > 0)[:, None]
    place = torch.arange(page, device="cuda").expand_as(move)[move]
    fro, to = fro[:, None].expand_as(move)[move], new.long()[:, None].expand_as(move)[move]
    if c["held"] == "16":
        pool["kv"][:, :, to, place] = pool["kv"][:, :, fro, place]
    else:
        for x in (pool["codes"], pool["scales"].view(torch.uint8)):
            x[:, :, to, :, place] = x[:, :, fro, :, place]
    return _state(pool)


def run(s):
    if own:
        return _own(s)
    return {"attention": _attention, "append": _append, "select": _select, "reorder": _reorder}[s["case"]["kind"]](s)


# ------------------------------------------------------------------------------------------------ floors
def work(c):
    e = SIZES[c["dtype"]]
    if c["kind"] == "attention":
        b, t = c["batch"], c["nodes"]
        lengths, nodes = _lengths(c, b), _nodes(c, b)
        cached = sum(n + m for n, m in zip(lengths, nodes)) * c["kv_heads"] * c["dim"] * 2 * HELD
        rows = 2 * b * t * c["heads"] * c["dim"] * e + b * t * ((t + 31) // 32) * 4
        return {"bytes": cached + rows, "flops": 4 * c["dim"] * c["heads"] * sum(m * (n + 1) for n, m in zip(lengths, nodes))}
    if c["kind"] == "append":
        values = 2 * c["layers"] * c["batch"] * c["nodes"] * c["kv_heads"] * c["dim"]
        return {"bytes": values * (2 * e + HELD), "flops": 6 * values}             # the 4 bits, once written, are still at hand to be read
    if c["kind"] == "select":
        rows = c["batch"] * c["beams"]
        return {"bytes": rows * (c["vocab"] * e + 4) + c["batch"] * c["n"] * 12, "flops": 4 * rows * c["vocab"]}
    token = c["layers"] * 2 * c["kv_heads"] * c["dim"] * (HELD if c["held"] == "4" else e)
    copied, tables = 0, 0
    for n, parents in zip(_lengths(c, c["batch"]), _parents_of(c)):
        copied += (n % c["page"]) * (c["beams"] + len(set(parents)))               # each source read once, each copy written
        copied -= (n % c["page"]) * sum(2 if parents.count(p) == 1 else 1 for p in set(parents))      # heirs write nothing; a source without copies is not read
        tables += 8 * c["beams"] * -(-n // c["page"])
    return {"bytes": token * copied + tables, "flops": 0}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(c, seed):
    s = prepare(c, seed)
    return {"attention": _exact_attention, "append": _exact_append, "select": _exact_select, "reorder": _exact_reorder}[c["kind"]](c, s)


def _floats(exponents, fractions, bias):
    """What a small float of so many exponents and fractions can be, ascending: its bits are the place."""
    return torch.tensor([m / fractions * 2.0 ** (1 - bias) if e == 0 else (1 + m / fractions) * 2.0 ** (e - bias) for e in range(exponents) for m in range(fractions)],
                        dtype=torch.float64, device="cuda")


def _exact_values(codes, scales):
    """Values of codes and scales, from their bits."""
    fours, s = _floats(4, 2, 1), _floats(16, 8, 7)[scales.view(torch.uint8).int()]

    def number(c):
        return torch.where(c >= 8, -1, 1) * fours[(c & 7).int()]
    out = torch.empty(*codes.shape[:-1], codes.shape[-1] * 2, dtype=torch.float64, device=codes.device)
    out[..., ::2], out[..., 1::2] = number(codes & 15), number(codes >> 4)
    return out * s.repeat_interleave(BLOCK, -1)


def _exact_attention(c, s):
    pool, g = s["pool"], c["heads"] // c["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lengths, nodes = pool["length"].tolist(), s["n_nodes"].tolist()
    words = s["mask"].cpu().long() & 0xFFFFFFFF
    scales = pool["scales"].view(torch.uint8)
    for b in range(c["batch"]):
        n, m = lengths[b], nodes[b]
        pages = pool["table"][b, :-(-(n + m) // c["page"])].long()
        see = torch.ones(m, n + m, dtype=torch.bool)
        for j in range(m):
            see[:, n + j] = ((words[b, :m, j // 32] >> (j % 32)) & 1).bool()
        see = see.cuda()
        for h in range(c["kv_heads"]):
            k, v = (_exact_values(pool["codes"][0, side, pages, h], scales[0, side, pages, h]).flatten(0, 1)[:n + m] for side in range(2))
            for j in range(h * g, h * g + g):
                a = s["q"][b, :m, j].double() @ k.T / math.sqrt(c["dim"])
                a = torch.softmax(a.masked_fill(~see, -math.inf), 1)
                out[b, :m, j] = a @ v
    return out


def _exact_append(c, s):
    """Values by distance: the nearest scale, then the nearest code, of two alike the even one."""
    if s["k"].numel() > 3e7:
        return None
    eights, fours = _floats(16, 8, 7)[:127], _floats(4, 2, 1)

    def nearest(x, values):
        hi = torch.searchsorted(values, x).clamp(max=values.numel() - 1)
        lo = (hi - 1).clamp(min=0)
        below, above = x - values[lo], values[hi] - x
        return torch.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)

    def back(x):
        x = x.double().unflatten(-1, (-1, BLOCK))
        scale = eights[nearest(x.abs().amax(-1), 6 * eights)][..., None]
        code = fours[nearest(torch.where(scale > 0, x.abs() / scale, 0), fours)]
        return (code * scale * x.sign()).flatten(-2)
    return back(s["k"]), back(s["v"])


def _exact_select(c, s):
    """Sentence by sentence; the scores alone, as tokens of equal rank are anyone's."""
    b, k, v = s["logits"].shape
    out = torch.full((b, c["n"]), -math.inf, dtype=torch.float64, device="cuda")
    for i in range(b):
        score = torch.log_softmax(s["logits"][i].double(), -1) + s["scores"][i].double()[:, None]
        if s["finished"] is not None:
            for j in s["finished"][i].nonzero()[:, 0].tolist():
                score[j] = -math.inf
                score[j, 2] = s["scores"][i, j].double()
        rank = score if s["norm"] is None else score * s["norm"][i].double()[:, None]
        value, at = rank.flatten().topk(min(c["n"], k * v))
        out[i, :len(at)] = torch.where(value > -math.inf, score.flatten()[at], -math.inf)
    return out, None, None


def _exact_reorder(c, s):
    """Beam by beam, with lists of pages."""
    pool, page, k = s["pool"], c["page"], c["beams"]
    if c["held"] == "4":
        return None
    kv = pool["kv"].double()
    before = [[p for p in row if p >= 0] for row in pool["table"].tolist()]
    length, seqs, parents = pool["length"].tolist(), s["seqs"].tolist(), s["parents"].tolist()
    count = [0] * pool["refs"].numel()
    copies = []
    for mine, up in zip(seqs, parents):
        for j, p in enumerate(up):
            n = length[mine[p]]
            children = [x for x in range(k) if up[x] == p]
            takes = j == (p if p in children else children[0])
            for q in before[mine[p]][:n // page + (takes and n % page > 0)]:
                count[q] += 1
            if n % page and not takes:
                copies.append((before[mine[p]][n // page], n % page))
    free = [p for p, x in enumerate(count) if x == 0]
    for (fro, n), to in zip(copies, free):
        kv[:, :, to, :n] = kv[:, :, fro, :n]
    return {name: kv if name == "kv" else None for name in _state(pool)}
