"""Plain implementations of the tree-speculation operators: Python loops and float64 on the CPU, written from their contracts."""
import math

import numpy as np
import torch


def ancestors(parents, n_nodes):
    """([B][T] sets of visible nodes, depths)."""
    see, depth = [], []
    for row, n in zip(parents, n_nodes):
        s, d = [], []
        for i in range(len(row)):
            j, up = i, set()
            while i < n and j >= 0:
                up.add(j)
                j = row[j] if 0 <= row[j] < j else -1
            s.append(up)
            d.append(len(up) - 1)
        see.append(s)
        depth.append(d)
    return see, depth


def pack(see, T):
    W = (T + 31) // 32
    out = np.zeros((len(see), T, W), dtype=np.uint32)
    for b, rows in enumerate(see):
        for i, up in enumerate(rows):
            for j in up:
                out[b, i, j // 32] |= np.uint32(1 << (j % 32))
    return torch.from_numpy(out.view(np.int32))


def accept(parents, tokens, sampled, n):
    path, i = [], 0
    while n > 0:
        path.append(i)
        nxt = [j for j in range(i + 1, n) if parents[j] == i and tokens[j] == sampled[i]]
        if not nxt:
            break
        i = nxt[0]
    return path, [sampled[j] for j in path]


def attention(q, k, v, see, scale):
    """q [T, H, D], k, v [S, Hkv, D], see [T, S]: (out, sum of p |v|, in float64)."""
    T, H, D = q.shape
    kk, vv = (x.double().repeat_interleave(H // k.shape[1], 1).transpose(0, 1) for x in (k, v))      # [H, S, D]
    s = (q.double().transpose(0, 1) @ kk.transpose(1, 2)) * scale
    s = s.masked_fill(~see, -math.inf)
    top = s.max(-1, keepdim=True).values if s.shape[2] else s.new_zeros(H, T, 1)
    p = torch.exp(s - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    return (p @ vv).transpose(0, 1), (p @ vv.abs()).transpose(0, 1)


def sample_row(logits, u, temperature, top_k, top_p, min_p):
    """(token, log probability, margin): margin is how near, relative to the row's weight, any of the row's decisions is to falling otherwise."""
    l = np.where(np.isnan(logits), -math.inf, logits.astype(np.float64))
    top = l.max()
    if top == -math.inf:
        return -1, -math.inf, 1.0
    first = int(l.argmax())
    if not temperature > 0:
        return first, 0.0, 1.0
    with np.errstate(invalid="ignore", over="ignore"):
        x = np.where(l == top, 0.0, (l - top) / temperature)
    ratio = np.where(l > -math.inf, np.exp(x), 0.0)
    w = np.floor(ratio * 2.0 ** 40)
    order = np.lexsort((np.arange(len(l)), -l))
    margin = 1.0
    wo = w[order]
    if 0 < top_k < len(l):
        wo[top_k:] = 0
    total = wo.sum()
    keep = wo > 0
    if top_p < 1:
        before = np.cumsum(wo) - wo
        keep &= before < top_p * total
        margin = min([margin] + list(np.abs(before - top_p * total)[1:][wo[1:] > 0] / total))      # (the first is kept anyway)
    if min_p > 0:
        keep &= ratio[order] >= min_p
        margin = min([margin] + list(np.abs(ratio - min_p)[l < top]))                              # (the largest have 1 exactly)
    keep[0] = True
    kept = np.zeros_like(w)
    kept[order[keep]] = wo[keep]
    cum = np.cumsum(kept)
    goal = math.floor(min(max(u, 0.0), 1.0) * cum[-1])
    goal = min(goal, cum[-1] - 1)
    token = int((cum <= goal).sum())
    margin = min(margin, np.abs(cum[kept > 0] - goal).min() / cum[-1], 1.0)
    if np.isin(ratio, (0.0, 1.0)).all():
        margin = 1.0                                           # equal weights: every sum and product above is exact
    return token, x[token] - math.log(cum[-1] / 2.0 ** 40), margin


class Pages:
    """The cache's bookkeeping and contents, one token at a time."""

    def __init__(self, kv, n_seqs, max_pages):
        self.kv = kv.clone()                                   # [L, 2, P, page, H, D]
        self.page, self.max_pages = kv.shape[3], max_pages
        self.table = [[] for _ in range(n_seqs)]
        self.length = [0] * n_seqs
        self.refs = [0] * kv.shape[2]

    def need(self, s, n):
        return max(0, -(-(self.length[s] + n) // self.page) - len(self.table[s]))

    def take(self):
        p = self.refs.index(0)
        self.refs[p] = 1
        return p

    def reserve(self, seqs, n):
        if any(len(self.table[s]) + self.need(s, n) > self.max_pages for s in seqs):
            return 2
        if sum(self.need(s, n) for s in seqs) > self.refs.count(0):
            return 1
        for s in seqs:
            for _ in range(self.need(s, n)):
                self.table[s].append(self.take())
        return 0

    def at(self, s, t):
        return self.table[s][t // self.page], t % self.page

    def append(self, seqs, k, v, layers, count):
        for i, s in enumerate(seqs):
            for t in range(count[i]):
                p, o = self.at(s, self.length[s] + t)
                for n, l in enumerate(layers):
                    self.kv[l, 0, p, o], self.kv[l, 1, p, o] = k[n, i, t], v[n, i, t]

    def compact(self, seqs, paths):
        for s, path in zip(seqs, paths):
            rows = [self.kv[(slice(None), slice(None)) + self.at(s, self.length[s] + j)].clone() for j in path]
            for j, r in enumerate(rows):
                self.kv[(slice(None), slice(None)) + self.at(s, self.length[s] + j)] = r
            self.length[s] += len(path)
            keep = -(-self.length[s] // self.page)
            for p in self.table[s][keep:]:
                self.refs[p] -= 1
            del self.table[s][keep:]

    def release(self, seqs):
        for s in seqs:
            for p in self.table[s]:
                self.refs[p] -= 1
            self.table[s], self.length[s] = [], 0

    def fork(self, src, dst):
        pairs = [(a, b) for a, b in zip(src, dst) if a != b]
        old = {a: (list(self.table[a]), self.length[a]) for a, _ in pairs}
        held = [old[a][0][old[a][1] // self.page] for a, _ in pairs if old[a][1] % self.page]
        refs = list(self.refs)
        for a, b in pairs:
            for p in self.table[b]:
                refs[p] -= 1
        for a, b in pairs:
            for p in old[a][0][:old[a][1] // self.page]:
                refs[p] += 1
        free = [p for p, n in enumerate(refs) if n == 0 and p not in held]
        if len(free) < len(held):
            return 1
        self.refs = refs
        content = self.kv.clone()
        for a, b in pairs:
            table, n = old[a]
            full, part = n // self.page, n % self.page
            self.table[b], self.length[b] = table[:full], n
            if part:
                p = free.pop(0)
                self.refs[p] = 1
                self.kv[:, :, p, :part] = content[:, :, table[full], :part]
                self.table[b].append(p)
        return 0
