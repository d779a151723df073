"""Performance cases of the tree-speculation operators: attention over a paged cache, sampling, the cache's pages, the tree itself.

A case is one call (pages, tree: the short fixed sequence of calls that a decoding step makes) of paper_2203_16487_b200.tree:

  attention  queries of a tree of drafted tokens (one token: plain decoding) over the cached tokens and their ancestors
  sample     one token a row with temperature, top-k, top-p and min-p from a given random number, and its log probability
  pages      fork: branches that share a prompt's full pages and copy its last one
             step: fork, reserve, append the block's keys and values, keep the accepted path
  tree       ancestor bits and depths of drafted trees, then the walk along the sampled tokens

`own` chooses between the framework's calls and the same operators written as elementary torch operations.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def listed():
    att = dict(kind="attention", page=16)
    return [
        # one sentence of the online translation setting: last token and k = 25 drafts, 8 heads of 64; latency counts
        dict(att, name="attention_sentence", batch=1, nodes=26, heads=8, kv_heads=8, dim=64, lo=64, hi=64, dtype="bf16"),
        # the benchmark's largest verify step: 128 ragged sequences, k = 50
        dict(att, name="attention_batch", batch=128, nodes=51, heads=8, kv_heads=8, dim=64, lo=0, hi=256, dtype="bf16"),
        # one token a sequence over long caches with grouped heads
        dict(att, name="attention_decode_long", batch=2, nodes=1, heads=32, kv_heads=8, dim=128, page=64, lo=65537, hi=131071, dtype="f16"),
        # trees over long documents with grouped heads: the most arithmetic
        dict(att, name="attention_tree_long", batch=8, nodes=64, heads=32, kv_heads=8, dim=128, page=64, lo=8191, hi=16385, dtype="bf16"),
        # the fp32 types of the small reference pair, over summarisation-length sources
        dict(att, name="attention_f32", batch=8, nodes=9, heads=8, kv_heads=8, dim=64, lo=300, hi=512, dtype="f32"),
        # the nodes of one sentence's tree; every node is sampled
        dict(kind="sample", name="sample_sentence", requests=1, nodes=26, vocab=32768, dtype="f32", filters="nucleus"),
        # the nodes of 128 sentences, each with parameters of its own
        dict(kind="sample", name="sample_batch", requests=128, nodes=26, vocab=32768, dtype="bf16", filters="mixed"),
        # an odd vocabulary: rows that begin anywhere
        dict(kind="sample", name="sample_odd", requests=32, nodes=3, vocab=50265, dtype="f32", filters="mixed"),
        # the cache's part of one step of 32 sentences: 6 layers, 8 heads of 64
        dict(kind="pages", name="pages_step", what="step", prompts=32, ways=1, layers=6, kv_heads=8, dim=64, page=16, lo=40, hi=300, nodes=26, dtype="bf16"),
        # eight prompts into four branches each: 32 layers, pages of 128 tokens
        dict(kind="pages", name="pages_fork", what="fork", prompts=8, ways=4, layers=32, kv_heads=8, dim=128, page=128, lo=700, hi=1023, nodes=0, dtype="bf16"),
        # one sentence's tree, and many large ones
        dict(kind="tree", name="tree_sentence", batch=1, nodes=26),
        dict(kind="tree", name="tree_batch", batch=128, nodes=256),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attention"] * 4 + ["sample"] * 3 + ["pages"] * 2 + ["tree"])
    if kind == "attention":
        c = dict(kind=kind, page=rng.choice([16, 32, 64, 128]), nodes=rng.choice([1, _log_int(rng, 2, 128), _log_int(rng, 2, 128)]),
                 dtype=rng.choice(["bf16", "bf16", "f16", "f32"]))
        c["kv_heads"] = rng.choice([1, 2, 4, 8, 12])
        group = rng.choice([1, 1, 2, 4, 8]) if c["kv_heads"] < 12 else 1
        c.update(heads=c["kv_heads"] * group, dim=rng.choice([64, 64, 128, 16, 80]))
        hi = _log_int(rng, 16, 100000)
        products = 2e10 if c["dtype"] != "f32" else 2e9
        hi = max(16, min(hi, int(products / (c["heads"] * c["nodes"] * c["dim"])), int(2.5e8 / (c["heads"] * c["nodes"]))))
        c["batch"] = max(1, min(_log_int(rng, 1, 128), int(products / (c["heads"] * c["nodes"] * hi * c["dim"])),
                                int(2.5e8 / (c["heads"] * c["nodes"] * hi)), int(2e8 / (hi * c["kv_heads"] * c["dim"]))))
        c.update(lo=rng.randint(0, hi), hi=hi)
        return c
    if kind == "sample":
        c = dict(kind=kind, vocab=rng.choice([1000, 32768, 50265, _log_int(rng, 1000, 131072)]), dtype=rng.choice(["bf16", "f16", "f32", "f32"]),
                 filters=rng.choice(["none", "nucleus", "top_k", "mixed", "mixed"]), nodes=_log_int(rng, 1, 51))
        c["requests"] = max(1, min(_log_int(rng, 1, 128), int(1e8 // (c["vocab"] * c["nodes"]))))
        return c
    if kind == "pages":
        c = dict(kind=kind, what=rng.choice(["fork", "step", "step"]), ways=rng.choice([1, 2, 4]), layers=rng.choice([2, 6, 12, 32]),
                 kv_heads=rng.choice([1, 8, 12]), dim=rng.choice([64, 128]), page=rng.choice([16, 32, 64, 128]), dtype=rng.choice(["bf16", "f16", "f32"]))
        c["nodes"] = _log_int(rng, 2, 64) if c["what"] == "step" else 0
        hi = _log_int(rng, 16, 2000)
        token = c["layers"] * c["kv_heads"] * c["dim"]
        c["prompts"] = max(1, min(_log_int(rng, 1, 64), int(2e8 / (token * (hi + c["ways"] * (c["nodes"] + c["page"]))))))
        c.update(lo=rng.randint(1, hi), hi=hi)
        return c
    return dict(kind=kind, batch=_log_int(rng, 1, 128), nodes=_log_int(rng, 1, 256))


# ------------------------------------------------------------------------------------------------ inputs
def _lengths(c, n):
    """Cached tokens of each sequence: by the case alone, as its work is."""
    r = random.Random(c["lo"] * 1000003 + c["hi"] * 101 + n)
    return [c["hi"]] + [r.randint(c["lo"], c["hi"]) for _ in range(n - 1)]


def _nodes(c, n):
    """Nodes of each tree: full ones, and for every third sequence fewer."""
    return [c["nodes"] if b % 3 < 2 else max(1, c["nodes"] - b % 7) for b in range(n)]


def _parents(c, g, batch):
    """Random trees: a node hangs off one of the eight before it."""
    i = torch.arange(c["nodes"], device="cuda")
    back = (torch.rand(batch, c["nodes"], generator=g, device="cuda") * torch.clamp(i, max=8)).long()
    return torch.where(i > 0, i - 1 - back, -1).int()


def _closure(parents):
    """[B, T, T]: node j is node i or one of its ancestors."""
    i = torch.arange(parents.shape[1], device=parents.device)
    up = (parents.long()[:, :, None] == i) | (i[:, None] == i)
    return torch.linalg.matrix_power(up.double() / 2, max(1, parents.shape[1] - 1)) > 0    # the halves keep counts of paths in range


def _pack(see):
    """Bits of a [B, T, T] mask: word w, bit j is node 32 w + j."""
    b, t, _ = see.shape
    w = (t + 31) // 32
    bits = torch.nn.functional.pad(see, (0, 32 * w - t)).view(b, t, w, 32).long()
    words = (bits << torch.arange(32, device=see.device)).sum(-1)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).int()


def _pool(c, g, lengths, held, n_seqs, spare):
    """A cache whose first sequences hold `held` pages each, scattered over the pool; `spare` more pages are free."""
    dt, pages = DTYPES[c["dtype"]], sum(held) + spare
    layers = c.get("layers", 1)
    kv = torch.randn(layers, 2, pages, c["page"], c["kv_heads"], c["dim"], generator=g, device="cuda", dtype=torch.float32 if dt == torch.float32 else dt)
    width = max(held + [1]) + (c["nodes"] + c["page"] - 1) // c["page"] + 1
    order = torch.randperm(pages, generator=g, device="cuda").int()[:sum(held)]
    table = torch.full((n_seqs, width), -1, dtype=torch.int32, device="cuda")
    h = torch.tensor(held, device="cuda")
    table[:len(held)][torch.arange(width, device="cuda") < h[:, None]] = order
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    refs[order.long()] = 1
    rest = [0] * (n_seqs - len(held))
    return dict(kv=kv, table=table, length=torch.tensor(list(lengths) + rest, dtype=torch.int32, device="cuda"),
                held=torch.tensor(list(held) + rest, dtype=torch.int32, device="cuda"), refs=refs)


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": c}
    if c["kind"] == "attention":
        b, t = c["batch"], c["nodes"]
        lengths, nodes = _lengths(c, b), _nodes(c, b)
        held = [-(-(n + t) // c["page"]) for n in lengths]
        s["pool"] = _pool(c, g, lengths, held, b, 1)
        s["q"] = (torch.randn(b, t, c["heads"], c["dim"], generator=g, device="cuda") * 2).to(DTYPES[c["dtype"]])
        s["mask"] = _pack(_closure(_parents(c, g, b)))
        s["n_nodes"] = torch.tensor(nodes, dtype=torch.int32, device="cuda")
        s["seqs"] = torch.arange(b, dtype=torch.int32, device="cuda")
        s["max_length"] = c["hi"]
    elif c["kind"] == "sample":
        n, v = c["requests"], c["vocab"]
        rows = n * c["nodes"]
        logits = torch.randn(rows, v, generator=g, device="cuda") * 2
        at = torch.randint(4, v, (rows, 32), generator=g, device="cuda")
        logits.scatter_add_(1, at, 5 + 4 * torch.rand(rows, 32, generator=g, device="cuda"))     # the tokens that fit
        logits[:, :2] = -math.inf                                                                # ids that are never written
        s["logits"] = logits.to(DTYPES[c["dtype"]]).view(n, c["nodes"], v)
        s["uniform"] = torch.rand(n, c["nodes"], generator=g, device="cuda")
        u = torch.rand(4, n, generator=g, device="cuda")
        f, one = c["filters"], torch.ones(n, device="cuda")
        s["temperature"] = torch.where(u[0] < 0.1, 0.0, 0.5 + u[0]) if f == "mixed" else one * 0.8
        s["top_k"] = torch.where(u[1] < 0.4, 0, (1 + u[1] * 100)).int() if f == "mixed" else (one * (40 if f == "top_k" else 0)).int()
        s["top_p"] = torch.where(u[2] < 0.3, 1.0, 0.6 + 0.39 * u[2]) if f == "mixed" else one * (0.95 if f == "nucleus" else 1.0)
        s["min_p"] = torch.where(u[3] < 0.5, 0.0, 0.1 * u[3]) if f == "mixed" else one * 0.0
    elif c["kind"] == "pages":
        n, ways = c["prompts"], c["ways"]
        lengths = _lengths(c, n)
        spare = n * ways * (2 + -(-c["nodes"] // c["page"]))
        s["pool"] = _pool(c, g, lengths, [-(-x // c["page"]) for x in lengths], n + n * ways, spare)
        s["src"] = torch.arange(n, device="cuda").repeat_interleave(ways).int()
        s["dst"] = torch.arange(n, n + n * ways, device="cuda").int()
        if c["what"] == "step":
            b, t = n * ways, c["nodes"]
            shape = (c["layers"], b, t, c["kv_heads"], c["dim"])
            s["k"], s["v"] = (torch.randn(shape, generator=g, device="cuda").to(DTYPES[c["dtype"]]) for _ in "kv")
            keep = torch.rand(b, t, generator=g, device="cuda") < min(1.0, 6.0 / t)
            keep[:, 0] = True
            s["n_path"] = keep.sum(1).int()
            at = torch.where(keep, torch.arange(t, device="cuda"), t).sort(1).values
            s["path"] = torch.where(at < t, at, -1).int()
    else:
        b, t = c["batch"], c["nodes"]
        s["parents"] = _parents(c, g, b)
        s["tokens"] = torch.randint(0, 6, (b, t), generator=g, device="cuda").int()              # few ids, so that walks go deep
        s["sampled"] = torch.randint(0, 6, (b, t), generator=g, device="cuda").int()
        s["n_nodes"] = torch.tensor(_nodes(c, b), dtype=torch.int32, device="cuda")
    if own and "pool" in s:
        from paper_2203_16487_b200 import tree
        s["cache"] = tree.PagedCache.over(**s["pool"])
    return s


# ------------------------------------------------------------------------------------------------ the framework's calls
def _own(s):
    from paper_2203_16487_b200 import tree
    kind = s["case"]["kind"]
    if kind == "attention":
        return tree.attention(s["q"], s["cache"], 0, s["seqs"], s["mask"], n_nodes=s["n_nodes"], max_length=s["max_length"])
    if kind == "sample":
        return tree.sample(s["logits"], s["uniform"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])
    if kind == "tree":
        mask, depth = tree.ancestors(s["parents"], s["n_nodes"])
        return (mask, depth) + tree.accept(s["parents"], s["tokens"], s["sampled"], s["n_nodes"])
    cache = s["cache"]
    cache.fork(s["src"], s["dst"])
    if s["case"]["what"] == "step":
        cache.reserve(s["dst"], s["case"]["nodes"])
        cache.append(s["dst"], s["k"], s["v"])
        cache.compact(s["dst"], s["path"], s["n_path"])
    return s["pool"]


# ------------------------------------------------------------------------------------------------ plain forms
def _slots(table, pos, page):
    """Row of each position in the pool seen as [pages * page tokens]."""
    return torch.gather(table, 1, (pos // page).long()) * page + pos % page


def _attention(s):
    c, pool = s["case"], s["pool"]
    t, h, n, d = c["nodes"], c["heads"], c["kv_heads"], c["dim"]
    length, nodes = pool["length"][s["seqs"].long()], s["n_nodes"]
    pos = torch.arange(s["max_length"] + t, device="cuda").expand(c["batch"], -1)
    there = pos < (length + nodes)[:, None]
    rows = torch.where(there, _slots(pool["table"][s["seqs"].long()], torch.where(there, pos, 0), c["page"]), 0).long()
    k, v = (torch.where(there[:, :, None, None], x.reshape(-1, n, d)[rows], 0).float() for x in pool["kv"][0])
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


UNIT = 2.0 ** 40                    # weights are whole multiples of 1 / UNIT, so that their sums do not depend on an order


def _sample(s):
    c = s["case"]
    rows, v = c["requests"] * c["nodes"], c["vocab"]
    temperature, top_k, top_p, min_p = (s[x].repeat_interleave(c["nodes"])[:, None] for x in ("temperature", "top_k", "top_p", "min_p"))
    logit = s["logits"].reshape(rows, v).float()
    logit = torch.where(torch.isnan(logit), -math.inf, logit)
    order = logit.sort(dim=1, descending=True, stable=True).indices
    top = logit.gather(1, order[:, :1])
    greedy = temperature <= 0
    x = torch.where(logit == top, 0.0, (logit - top) * (1 / torch.where(greedy, 1.0, temperature)))
    w = torch.where(logit > -math.inf, torch.exp(x), 0.0)
    unit = (w * UNIT).long()
    ranked = unit.gather(1, order)
    rank = torch.arange(v, device="cuda")
    k = torch.where(greedy, 1, torch.where((top_k <= 0) | (top_k > v), v, top_k))
    ranked = torch.where(rank < k, ranked, 0)
    total = ranked.sum(1, keepdim=True)
    before = ranked.cumsum(1) - ranked
    keep = (rank < k) & ((top_p >= 1) | (before.double() < top_p.double() * total.double())) & (w.gather(1, order) >= min_p)
    keep |= rank == 0
    kept = torch.zeros_like(unit).scatter_(1, order, torch.where(keep, ranked, 0))
    upto = kept.cumsum(1)
    total = upto[:, -1:]
    goal = (s["uniform"].reshape(rows, 1).double() * total.double()).long()
    token = (upto <= torch.minimum(goal, total - 1)).sum(1)
    none = total[:, 0] <= 0
    logp = x.gather(1, token.clamp(max=v - 1)[:, None])[:, 0] - torch.log((total[:, 0].float() / UNIT))
    token, logp = torch.where(none, -1, token).int(), torch.where(none, -math.inf, logp)
    return token.view(c["requests"], -1), logp.view(c["requests"], -1)


def _tree(s):
    parents, tokens, sampled, nodes = s["parents"].long(), s["tokens"], s["sampled"], s["n_nodes"]
    b, t = parents.shape
    i = torch.arange(t, device="cuda")
    real = i < nodes[:, None]
    see = _closure(s["parents"]) & real[:, :, None] & real[:, None, :]
    depth = torch.where(real, see.sum(2) - 1, -1).int()
    p = parents.clamp(min=0)
    match = (parents >= 0) & real & (tokens == sampled.gather(1, p))
    twin = (parents[:, :, None] == parents[:, None, :]) & (tokens[:, :, None] == tokens[:, None, :]) & (i < i[:, None])
    match &= ~twin.any(2)                                          # of children with the same token the first
    good = match | (i == 0)
    on = (see & ~good[:, None, :]).sum(2).eq(0) & real
    on &= see[:, :, 0]
    n_path = on.sum(1)
    path = torch.where(on, i, t).sort(1).values
    emitted = torch.where(path < t, sampled.gather(1, path.clamp(max=t - 1)), -1).int()
    return _pack(see), depth, torch.where(path < t, path, -1).int(), n_path.int(), emitted


def _take(pool, seqs, need):
    """Gives the i-th of `seqs` need[i] more pages behind those it holds: the lowest free ones, in order."""
    rank = torch.arange(int(pool["refs"].numel()), device="cuda")
    free = (pool["refs"] == 0).int().sort(descending=True, stable=True).indices
    first = need.cumsum(0) - need
    at = torch.arange(pool["table"].shape[1], device="cuda") - pool["held"][seqs][:, None]
    new = (at >= 0) & (at < need[:, None])
    page = free[(at + first[:, None]).clamp(0, free.numel() - 1)].int()
    pool["table"][seqs] = torch.where(new, page, pool["table"][seqs])
    pool["refs"][free] += (rank < need.sum()).int()
    pool["held"][seqs] += need.int()


def _fork(s):
    pool, page = s["pool"], s["case"]["page"]
    src, dst = s["src"].long(), s["dst"].long()
    table, refs = pool["table"], pool["refs"]
    at = torch.arange(table.shape[1], device="cuda")
    length = pool["length"][src]
    full, part = length // page, (length % page > 0).int()
    old, rows = table[dst], table[src]
    share = at < full[:, None]
    refs.scatter_add_(0, old.clamp(min=0).view(-1).long(), -(old >= 0).int().view(-1))
    refs.scatter_add_(0, rows.clamp(min=0).view(-1).long(), share.int().view(-1))
    table[dst] = torch.where(share, rows, -1)
    pool["held"][dst], pool["length"][dst] = full, length
    _take(pool, dst, part)
    last = full.clamp(max=table.shape[1] - 1).long()[:, None]
    fro, to = rows.gather(1, last)[:, 0].clamp(min=0).long(), table[dst].gather(1, last)[:, 0].clamp(min=0).long()
    token = torch.arange(page, device="cuda")
    move = token < (length % page)[:, None]
    flat = pool["kv"].view(pool["kv"].shape[0], 2, -1, *pool["kv"].shape[4:])
    a, b = (fro[:, None] * page + token)[move], (to[:, None] * page + token)[move]
    flat[:, :, b] = flat[:, :, a]


def _step(s):
    pool, c = s["pool"], s["case"]
    page, t, dst = c["page"], c["nodes"], s["dst"].long()
    flat = pool["kv"].view(c["layers"], 2, -1, c["kv_heads"], c["dim"])
    length = pool["length"][dst]
    _take(pool, dst, (length + t + page - 1) // page - pool["held"][dst])
    slot = _slots(pool["table"][dst], length[:, None] + torch.arange(t, device="cuda"), page).long()
    flat[:, 0, slot], flat[:, 1, slot] = s["k"], s["v"]
    on = s["path"] >= 0
    fro = slot.gather(1, s["path"].clamp(min=0).long())
    flat[:, :, slot[on]] = flat[:, :, fro[on]]
    length = length + s["n_path"]
    hold = (length + page - 1) // page
    table = pool["table"][dst]
    gone = (torch.arange(table.shape[1], device="cuda") >= hold[:, None]) & (table >= 0)
    pool["refs"].scatter_add_(0, table.clamp(min=0).view(-1).long(), -gone.int().view(-1))
    pool["table"][dst] = torch.where(gone, -1, table)
    pool["length"][dst], pool["held"][dst] = length, hold


def run(s):
    if own:
        return _own(s)
    kind = s["case"]["kind"]
    if kind == "pages":
        _fork(s)
        if s["case"]["what"] == "step":
            _step(s)
        return s["pool"]
    return {"attention": _attention, "sample": _sample, "tree": _tree}[kind](s)


# ------------------------------------------------------------------------------------------------ floors
def work(c):
    e = {"bf16": 2, "f16": 2, "f32": 4}.get(c.get("dtype"), 4)
    if c["kind"] == "attention":
        b, t = c["batch"], c["nodes"]
        lengths, nodes = _lengths(c, b), _nodes(c, b)
        cached = sum(n + m for n, m in zip(lengths, nodes)) * c["kv_heads"] * c["dim"] * 2 * e
        rows = 2 * b * t * c["heads"] * c["dim"] * e + b * t * ((t + 31) // 32) * 4
        return {"bytes": cached + rows, "flops": 4 * c["dim"] * c["heads"] * sum(m * (n + 1) for n, m in zip(lengths, nodes))}
    if c["kind"] == "sample":
        rows = c["requests"] * c["nodes"]
        return {"bytes": rows * c["vocab"] * e + rows * 12 + c["requests"] * 16, "flops": 10 * rows * c["vocab"]}
    if c["kind"] == "pages":
        token = c["layers"] * 2 * c["kv_heads"] * c["dim"] * e
        lengths = _lengths(c, c["prompts"])
        copied = c["ways"] * sum(n % c["page"] for n in lengths)
        new = c["ways"] * c["prompts"] * c["nodes"]
        kept = c["ways"] * c["prompts"] * min(6, c["nodes"])
        tables = 8 * (1 + c["ways"]) * sum(-(-n // c["page"]) for n in lengths)
        return {"bytes": 2 * token * (copied + new + kept) + tables, "flops": 0}
    words = (c["nodes"] + 31) // 32
    return {"bytes": 4 * c["batch"] * c["nodes"] * (3 + words + 1 + 2) + 8 * c["batch"], "flops": 0}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "attention":
        return _exact_attention(c, s)
    if c["kind"] == "sample":
        return _exact_sample(c, s)
    if c["kind"] == "pages":
        return _exact_pages(c, s)
    return None


def _exact_attention(c, s):
    pool, g = s["pool"], c["heads"] // c["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lengths, nodes = pool["length"].tolist(), s["n_nodes"].tolist()
    words = s["mask"].cpu().long() & 0xFFFFFFFF
    for b in range(c["batch"]):
        n, m = lengths[b], nodes[b]
        pages = pool["table"][b, :-(-(n + m) // c["page"])].long()
        k, v = (x[pages].flatten(0, 1)[:n + m].double() for x in pool["kv"][0])
        see = torch.ones(m, n + m, dtype=torch.bool)
        for j in range(m):
            see[:, n + j] = ((words[b, :m, j // 32] >> (j % 32)) & 1).bool()
        see = see.cuda()
        for h in range(c["heads"]):
            a = s["q"][b, :m, h].double() @ k[:, h // g].T / math.sqrt(c["dim"])
            a = torch.softmax(a.masked_fill(~see, -math.inf), 1)
            out[b, :m, h] = a @ v[:, h // g]
    return out


def _exact_sample(c, s):
    """Row by row, over the entries above the row's cut alone."""
    n, t = c["requests"], c["nodes"]
    logit = s["logits"].double()
    if n * t > 2000:
        return None
    logp = torch.empty(n, t, dtype=torch.float64)
    pars = [s[x].double().tolist() for x in ("temperature", "top_k", "top_p", "min_p")]
    uniform = s["uniform"].double().tolist()
    for r in range(n):
        temperature, top_k, top_p, min_p = (x[r] for x in pars)
        for j in range(t):
            row = logit[r, j]
            if temperature <= 0:
                logp[r, j] = 0.0
                continue
            value, index = torch.sort(row, descending=True, stable=True)
            w = torch.floor(torch.exp((value - value[0]) / temperature) * UNIT) / UNIT
            if top_k > 0:
                w[int(top_k):] = 0
            before = torch.cumsum(w, 0) - w
            keep = (w >= min_p) & ((before < top_p * w.sum()) | (top_p >= 1))
            keep[0] = True
            w = torch.where(keep, w, 0)
            back = torch.zeros_like(w)
            back[index] = w
            upto = torch.cumsum(back, 0)
            token = int((upto <= uniform[r][j] * upto[-1]).sum())
            logp[r, j] = (row[token] - value[0]) / temperature - torch.log(upto[-1])
    return None, logp


def _exact_pages(c, s):
    """Sequence by sequence, with lists of pages."""
    pool, page = s["pool"], c["page"]
    kv = pool["kv"].double()
    table = [[p for p in row if p >= 0] for row in pool["table"].tolist()]
    length, refs = pool["length"].tolist(), pool["refs"].tolist()

    def lowest():
        p = refs.index(0)
        refs[p] = 1
        return p

    for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
        full = length[a] // page
        for p in table[a][:full]:
            refs[p] += 1
        table[b], length[b] = table[a][:full], length[a]
        if length[a] % page:
            p = lowest()
            kv[:, :, p, :length[a] % page] = kv[:, :, table[a][full], :length[a] % page]
            table[b] = table[b] + [p]
    if c["what"] == "step":
        for i, b in enumerate(s["dst"].tolist()):
            while len(table[b]) * page < length[b] + c["nodes"]:
                table[b].append(lowest())
        for i, b in enumerate(s["dst"].tolist()):
            at = [(table[b][(length[b] + j) // page], (length[b] + j) % page) for j in range(c["nodes"])]
            for j, (p, o) in enumerate(at):
                kv[:, 0, p, o], kv[:, 1, p, o] = s["k"][:, i, j].double(), s["v"][:, i, j].double()
            for j, node in enumerate(s["path"][i, :int(s["n_path"][i])].tolist()):
                kv[:, :, at[j][0], at[j][1]] = kv[:, :, at[node][0], at[node][1]]
    return dict(kv=kv, table=None, length=None, held=None, refs=None)
