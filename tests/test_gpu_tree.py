"""Tree speculation on the caller's tensors: trees, cache pages, attention, sampling, against plain implementations in 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests import tree_reference as R

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def random_parents(rng, B, T, wild=False):
    p = [[-1] + [int(rng.integers(max(0, i - 6), i)) for i in range(1, T)] for _ in range(B)]
    if wild:                                                   # second roots and numbers that are no parents
        for row in p:
            for i in rng.integers(0, T, max(1, T // 7)):
                row[i] = int(rng.choice([-1, i, i + 3, 10 ** 6, -(10 ** 6)]))
    return p


# ------------------------------------------------------------------ trees
@pytest.mark.parametrize("B,T,wild", [(1, 1, False), (3, 26, False), (2, 31, True), (2, 32, True), (5, 33, False), (2, 100, True), (1, 257, True), (1, 1024, True)])
def test_ancestors_and_accept(B, T, wild):
    from paper_2203_16487_b200 import tree
    rng = np.random.default_rng(B * 1000 + T)
    parents = random_parents(rng, B, T, wild)
    if T == 1024:
        parents[0] = list(range(-1, T - 1))                    # one chain: as deep as can be
    n = [int(x) for x in rng.integers(0, T + 1, B)]
    n[0] = T
    tokens, sampled = rng.integers(0, 3, (B, T)), rng.integers(0, 3, (B, T))
    if T == 1024:
        tokens[0, 1:] = sampled[0, :-1]
    see, depth = R.ancestors(parents, n)
    mask, d = tree.ancestors(ints(parents), ints(n))
    assert torch.equal(mask.cpu(), R.pack(see, T)) and d.cpu().tolist() == depth
    path, n_path, emitted = (x.cpu().tolist() for x in tree.accept(ints(parents), ints(tokens), ints(sampled), ints(n)))
    for b in range(B):
        want, out = R.accept(parents[b], tokens[b].tolist(), sampled[b].tolist(), n[b])
        assert n_path[b] == len(want) and path[b] == want + [-1] * (T - len(want)) and emitted[b] == out + [-1] * (T - len(out))


# ------------------------------------------------------------------ pages
def same(cache, ref):
    assert cache.length.tolist() == ref.length and cache.refs.tolist() == ref.refs
    assert cache.held.tolist() == [len(t) for t in ref.table]
    assert cache.table.tolist() == [t + [-1] * (ref.max_pages - len(t)) for t in ref.table]
    assert torch.equal(cache.kv.cpu(), ref.kv)


@pytest.mark.parametrize("page,H,D,L,dtype,heads_first", [(16, 8, 64, 2, torch.bfloat16, False), (4, 3, 8, 3, torch.float16, True), (1, 1, 16, 1, torch.float32, False),
                                                          (64, 2, 128, 2, torch.bfloat16, True), (8, 5, 24, 1, torch.float32, False)])
def test_pages_random_walk(page, H, D, L, dtype, heads_first):
    """Every call, in random order, with calls that find too few pages among them: tables, counts and contents as one token at a time gives them."""
    from paper_2203_16487_b200 import tree
    rng = np.random.default_rng(page * 7 + H)
    n_seqs, max_pages, n_pages, T = 7, 9, 12, 2 * page + 3
    shape = (L, 2, n_pages, H, page, D) if heads_first else (L, 2, n_pages, page, H, D)
    kv = torch.randn(shape, device="cuda").to(dtype)
    kv = kv.transpose(3, 4) if heads_first else kv
    cache = tree.PagedCache.over(kv, torch.full((n_seqs, max_pages), -1, dtype=torch.int32, device="cuda"), ints([0] * n_seqs), ints([0] * n_seqs), ints([0] * n_pages))
    ref = R.Pages(kv.cpu(), n_seqs, max_pages)
    refused = 0
    for step in range(60):
        seqs = rng.permutation(n_seqs)[:rng.integers(1, 4)].tolist()
        what = rng.choice(["block", "block", "block", "fork", "beams", "release"])
        status = 0
        if what == "block":
            t = int(rng.integers(1, T + 1))
            status = ref.reserve(seqs, t)
            cache.reserve(ints(seqs), t)
            if status == 0:
                count = [int(x) for x in rng.integers(0, t + 1, len(seqs))]
                k = torch.randn(L, len(seqs), t, H, D + 8, device="cuda").to(dtype)[..., :D]          # strided rows
                v = torch.randn(L, len(seqs), t, H, D + 8, device="cuda").to(dtype)[..., :D]
                if rng.random() < 0.5:
                    cache.append(ints(seqs), k, v, count=ints(count))
                else:
                    for l in range(L):
                        cache.append(ints(seqs), k[l], v[l], layer=l, count=ints(count))
                ref.append(seqs, k.cpu(), v.cpu(), range(L), count)
                paths = [sorted(rng.permutation(t)[:rng.integers(0, t + 1)].tolist()) for _ in seqs]
                pad = [p + [-1] * (t - len(p)) for p in paths]
                cache.compact(ints(seqs), ints(pad), ints([len(p) for p in paths]))
                ref.compact(seqs, paths)
        elif what == "release":
            cache.release(ints(seqs))
            ref.release(seqs)
        else:
            dst = rng.permutation(n_seqs)[:len(seqs)].tolist()
            src = seqs if what == "fork" else [int(rng.choice(seqs)) for _ in seqs]
            status = ref.fork(src, dst)
            cache.fork(ints(src), ints(dst))
        assert int(cache.status.item()) == status, (step, what)
        refused += status != 0
        cache.status.zero_()
        same(cache, ref)
        # a token that can still be written belongs to one sequence alone
        assert all(ref.refs[p] == 1 for s in range(n_seqs) for p in ref.table[s][ref.length[s] // page:])
    assert refused, "the walk should meet a full pool"


@pytest.mark.parametrize("n", [1023, 1024, 1025, 2049, 2600])
def test_pages_long_paths(n):
    """A prompt's tokens committed in one go, some left out: more than any tree has.  A path that goes wrong late moves nothing."""
    from paper_2203_16487_b200 import tree
    rng, T, page, H, D, L = np.random.default_rng(n), 2600, 16, 3, 24, 2
    kv = torch.zeros(L, 2, 400, page, H, D, dtype=torch.float16, device="cuda")
    cache = tree.PagedCache.over(kv, torch.full((2, 200), -1, dtype=torch.int32, device="cuda"), ints([0, 0]), ints([0, 0]), ints([0] * 400))
    ref, seqs = R.Pages(kv.cpu(), 2, 200), [1, 0]
    k, v = (torch.randn(L, 2, T + 5, H, D, device="cuda").half() for _ in "kv")
    for c in (cache, ref):
        c.reserve(ints(seqs) if c is cache else seqs, T + 5)
    cache.append(ints(seqs), k[:, :, :5].contiguous(), v[:, :, :5].contiguous())
    ref.append(seqs, k[:, :, :5].cpu(), v[:, :, :5].cpu(), range(L), [5, 5])
    cache.compact(ints(seqs), ints([[0, 2]] * 2), ints([2, 2]))                # (blocks that begin inside a page)
    ref.compact(seqs, [[0, 2]] * 2)
    cache.reserve(ints(seqs), T)
    ref.reserve(seqs, T)
    cache.append(ints(seqs), k[:, :, 5:], v[:, :, 5:])
    ref.append(seqs, k[:, :, 5:].cpu(), v[:, :, 5:].cpu(), range(L), [T, T])
    paths = [sorted(rng.permutation(T)[:n].tolist()), list(range(n))]
    before = kv.clone()
    for at, to, status in ((n - 1, paths[0][n - 2], 4), (n - 1, T + 100, 8)):
        bad = list(paths[0])
        bad[at] = to
        cache.compact(ints(seqs[:1]), ints([bad]), ints([n]))
        assert int(cache.status.item()) == status and torch.equal(kv, before) and cache.length.tolist() == ref.length
        cache.status.zero_()
    cache.compact(ints(seqs), ints([p + [-1] * (T - n) for p in paths]), ints([n, n]))
    ref.compact(seqs, paths)
    cache.check()
    same(cache, ref)


def test_pages_refuse_what_is_wrong():
    from paper_2203_16487_b200 import binding, tree
    cache = tree.PagedCache(1, 2, 8, n_pages=4, n_seqs=3, max_pages=2, page_tokens=4)
    cache.reserve(ints([0, 5, 1]), 4)                          # no such sequence: the others are served
    assert int(cache.status.item()) == 4 and cache.held.tolist() == [1, 1, 0]
    with pytest.raises(binding.SpecDecError, match="out of range"):
        cache.check()
    cache.check()
    cache.reserve(ints([0]), 9)
    with pytest.raises(binding.SpecDecError, match="no room"):
        cache.check()
    assert cache.held.tolist() == [1, 1, 0]
    k = torch.randn(1, 1, 6, 2, 8, device="cuda").bfloat16()
    cache.append(ints([0]), k, k)                              # two tokens more than were reserved
    with pytest.raises(binding.SpecDecError, match="reserved"):
        cache.check()
    assert torch.equal(cache.kv[0, 0, 0], k[0, 0, :4])
    for path, n, why in (([[0, 0]], 2, "path"), ([[1, 0]], 2, "path"), ([[0, 1]], 3, "path"), ([[0, 1]], -1, "path"), ([[0, 5]], 2, "reserved"), ([[-2, 1]], 2, "path")):
        cache.compact(ints([0]), ints(path), ints([n]))
        with pytest.raises(binding.SpecDecError, match=why):
            cache.check()
    assert cache.length.tolist() == [0, 0, 0] and cache.held.tolist() == [1, 1, 0] and cache.refs.tolist() == [1, 1, 0, 0]
    for bad in (lambda: cache.reserve(ints([0]), -1), lambda: cache.reserve(ints([0, 1, 2, 0]), 1)):
        with pytest.raises(binding.SpecDecError):
            bad()
    for bad in (lambda: cache.append(ints([0]), k.half(), k.half()), lambda: cache.append(ints([0]), k[..., :4], k[..., :4]), lambda: cache.release(torch.tensor([0])),
                lambda: cache.compact(ints([0]), ints([0]), ints([1]))):
        with pytest.raises(ValueError):
            bad()


# ------------------------------------------------------------------ attention
def attention_case(dtype, lens, T, H, Hkv, D, page, *, nodes=None, one_mask=False, seed=0, strided=False, heads_first=False, mask=None, layer=0, spare=0):
    """A cache with those lengths (its slots elsewhere hold NaN), queries, masks, and the answer in 64 bits."""
    rng = np.random.default_rng(seed)
    g = torch.Generator().manual_seed(seed)
    B, L = len(lens), layer + 1
    nodes = [T] * B if nodes is None else nodes
    held = [-(-(n + T) // page) for n in lens]
    P = sum(held) + 2
    kv = torch.full((L, 2, P, Hkv, page, D) if heads_first else (L, 2, P, page, Hkv, D), math.nan).to(dtype)
    kv = kv.transpose(3, 4) if heads_first else kv
    table = torch.full((B + 1, max(held) + spare), -1, dtype=torch.int32)
    seqs = rng.permutation(B + 1)[:B]                          # rows of q and sequences are not in the same order
    order = rng.permutation(P)[:sum(held)]
    length = torch.zeros(B + 1, dtype=torch.int32)
    parents = random_parents(rng, B, T)
    see_nodes, _ = R.ancestors(parents, [T] * B)
    if one_mask:
        see_nodes = [see_nodes[0]] * B
    if mask is not None:
        see_nodes = [mask(b) for b in range(B)]
    q = torch.randn(B, T, H, D, generator=g).mul(2).to(dtype)
    want, mag = torch.zeros(B, T, H, D, dtype=torch.float64), torch.zeros(B, T, H, D, dtype=torch.float64)
    at = 0
    for b in range(B):
        n, s = lens[b], int(seqs[b])
        pages = order[at:at + held[b]]
        at += held[b]
        table[s, :held[b]] = torch.from_numpy(pages.astype(np.int32))
        length[s] = n
        S = n + nodes[b]
        x = torch.randn(2, S, Hkv, D, generator=g).to(dtype)
        see = torch.zeros(T, S, dtype=torch.bool)
        for t in range(nodes[b]):
            see[t, :n] = True
            for j in see_nodes[b][t]:
                if j < nodes[b]:
                    see[t, n + j] = True
        for j in range(S):
            if j < n or see[:, j].any():                       # what nobody sees stays NaN
                kv[layer, :, pages[j // page], j % page] = x[:, j]
        want[b], mag[b] = R.attention(q[b], x[0], x[1], see, D ** -0.5)
    kv, table, length = kv.cuda(), table.cuda(), length.cuda()
    from paper_2203_16487_b200 import tree
    hold = torch.zeros_like(length)
    cache = tree.PagedCache.over(kv, table, length, hold, ints([0] * P))
    qd = q.cuda()
    out = None
    if strided:                                                # rows inside a wider tensor, at odd places
        wide = torch.zeros(B, T, H * D * 3 + 1, dtype=dtype, device="cuda")
        wide[..., 1:1 + H * D] = qd.reshape(B, T, -1)
        qd = wide[..., 1:1 + H * D].unflatten(-1, (H, D))
        out = torch.zeros(B, H, T, D + 3, dtype=dtype, device="cuda")[..., 1:1 + D].transpose(1, 2)
    bits = R.pack([see_nodes[0]] if one_mask else see_nodes, T).cuda()
    got = tree.attention(qd, cache, layer, ints(seqs), bits, n_nodes=ints(nodes), out=out)
    return got, want, mag, (cache, qd, seqs, bits, nodes)


def check_attention(got, want, mag, dtype, keys):
    """One rounding of the probabilities (relative to their own size) and one of the output: 2^-8 each in bf16 (8 significant bits), 2^-11 in fp16, whose
    probabilities below 2^-14 keep 2^-25 absolute.  fp32: the score's and the exponential's rounding, some 2^-17 of a probability; the fp32 sums of
    the others are the 1e-5."""
    got = got.double().cpu()
    if dtype == torch.float32:
        tol = 1e-5 * mag + 1e-7
    else:
        u = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -11
        tol = u * (mag + want.abs()) + 1e-5 * mag + (keys * 2.0 ** -25 * 4 if dtype == torch.float16 else 0) + 1e-6
    off = (got - want).abs() - tol
    assert not got.isnan().any() and (off <= 0).all(), (float((got - want).abs().max()), float(off.max()))


LAYOUTS = [(8, 8, 64), (12, 12, 64), (4, 4, 16), (8, 2, 128), (6, 1, 80), (8, 1, 64), (32, 2, 128), (5, 5, 8)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("H,Hkv,D", LAYOUTS)
@pytest.mark.parametrize("T,page", [(1, 16), (5, 4), (26, 16), (33, 64), (70, 8)])
def test_attention_layouts(dtype, H, Hkv, D, T, page):
    lens = [0, 1, 63, 130]
    got, want, mag, _ = attention_case(dtype, lens, T, H, Hkv, D, page, seed=T + D)
    check_attention(got, want, mag, dtype, 200)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("T,H,Hkv,D,lens", [(1, 8, 2, 64, [3000]), (1, 4, 4, 128, [2047, 1, 2048]), (3, 8, 1, 128, [1500, 0]), (64, 8, 4, 64, [1029]), (17, 8, 8, 64, [64, 700])])
def test_attention_split_keys(dtype, T, H, Hkv, D, lens):
    """Few rows over long caches: keys split over CTAs, also where a sequence of the batch is short."""
    got, want, mag, _ = attention_case(dtype, lens, T, H, Hkv, D, 32, seed=5, spare=200)
    check_attention(got, want, mag, dtype, 3100)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("T,H,Hkv,D,n", [(2, 12, 12, 64, 41), (2, 12, 12, 128, 41), (20, 12, 12, 64, 41), (3, 48, 4, 64, 60), (20, 12, 12, 128, 30), (66, 7, 7, 64, 30), (130, 6, 3, 64, 30),
                                         (66, 7, 7, 128, 30)])
def test_attention_many_short_sequences(dtype, T, H, Hkv, D, n):
    """More sequences and heads than CTAs that run at once, of every number of key blocks: CTAs that take several."""
    if T > 30 and dtype == torch.float32:
        T = 30
    lens = [(i * 37) % 331 for i in range(n)]
    got, want, mag, _ = attention_case(dtype, lens, T, H, Hkv, D, 16, seed=T, one_mask=True)
    check_attention(got, want, mag, dtype, 500)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H,Hkv,D", [(1, 4, 2, 64), (9, 2, 2, 128), (12, 4, 2, 64), (40, 2, 1, 64), (100, 2, 2, 128), (90, 3, 1, 64)])
def test_attention_uneven_long_sequences(dtype, T, H, Hkv, D):
    """Sequences of one to thousands of keys: CTAs whose stretch of keys begins and ends inside sequences, or holds several."""
    if T > 12 and dtype == torch.float32:
        T = 3
    got, want, mag, _ = attention_case(dtype, [5000, 0, 3, 1900, 64, 65, 0, 700], T, H, Hkv, D, 16, seed=T, one_mask=True, nodes=[T, T, 1, T, 0, T, 0, T])
    check_attention(got, want, mag, dtype, 5100)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("H,Hkv,D", [(2, 1, 64), (2, 1, 128)])
def test_attention_two_groups_meet(dtype, H, Hkv, D):
    """Tiles of 128 rows, whose two groups take every second block of 128 keys and add up their outputs: none, one, two, three and many blocks, parts of a long sequence,
    the same bits every time."""
    from paper_2203_16487_b200 import tree
    T, lens = 50, [0, 70, 128 - 50, 206, 300, 1000, 6000]
    got, want, mag, (cache, q, seqs, bits, nodes) = attention_case(dtype, lens, T, H, Hkv, D, 16, seed=11, nodes=[T, T, T, T, 7, T, T])
    check_attention(got, want, mag, dtype, 6100)
    for _ in range(20):
        assert torch.equal(got, tree.attention(q, cache, 0, ints(seqs), bits, n_nodes=ints(nodes)))


@pytest.mark.parametrize("T,H,Hkv,D,lens", [(1024, 1, 1, 128, [70]), (970, 2, 1, 128, [0]), (1024, 1, 1, 64, [5, 1]), (300, 3, 1, 128, [129, 0]), (40, 12, 12, 64, [(i * 53) % 400 for i in range(41)])])
def test_attention_wide_trees(T, H, Hkv, D, lens):
    """The most nodes a tree may have (whose masks are 32 words a row), and whole sequences of 64 rows dealt to CTAs by length."""
    got, want, mag, _ = attention_case(torch.bfloat16, lens, T, H, Hkv, D, 32, seed=T, one_mask=len(lens) > 5)
    check_attention(got, want, mag, torch.bfloat16, T + max(lens))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kw", [dict(nodes=[9, 0, 3]), dict(one_mask=True), dict(strided=True), dict(heads_first=True), dict(layer=2), dict(nodes=[1, 9, 8], strided=True, heads_first=True)])
def test_attention_ragged_shared_strided(dtype, kw):
    got, want, mag, _ = attention_case(dtype, [40, 65, 0], 9, 8, 4, 64, 16, seed=3, **kw)
    check_attention(got, want, mag, dtype, 100)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_attention_masks(dtype):
    """Queries that see nothing, nodes that nobody sees (their slots hold NaN), nodes that see later ones."""
    T = 40
    def mask(b):
        return [set() if t % 3 == 0 else {T - 1, t} if t % 3 == 1 else {1, 34} for t in range(T)]
    got, want, mag, _ = attention_case(dtype, [0, 7], T, 4, 2, 64, 16, seed=9, mask=mask)
    check_attention(got, want, mag, dtype, 64)
    assert (got[0, ::3] == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,H,Hkv,D,page", [(1, 4, 4, 64, 16), (1, 16, 2, 128, 16), (20, 2, 2, 128, 16), (13, 4, 2, 64, 16), (50, 2, 2, 64, 16), (26, 4, 2, 64, 4), (9, 4, 2, 128, 2),
                                            (50, 4, 2, 128, 16), (100, 2, 2, 64, 32), (200, 4, 2, 128, 64), (70, 8, 2, 64, 16)])
def test_attention_weights_add_up_to_one(dtype, T, H, Hkv, D, page):
    """Values that lie around 8, peaked weights.  With weights w_j (1 + e_j) / sum_i w_i (1 + e_i), |e| <= u by the probabilities' rounding, the result is off by at most
    u / (1 - u) sum_j w_j |v_j - o|: by the spread of the values around the result, not by their size.  Then the output's rounding, u |o|, and fp32's."""
    from paper_2203_16487_b200 import tree
    g, lens = torch.Generator().manual_seed(T + D), [0, 40, 200, 1500]
    B, S = len(lens), max(lens)
    k, v = torch.randn(1, B, S + T, Hkv, D, generator=g).to(dtype), (8 + torch.randn(1, B, S + T, Hkv, D, generator=g) / 2).to(dtype)
    q = (torch.randn(B, T, H, D, generator=g) * 3).to(dtype)
    pages = -(-(S + T) // page)
    cache = tree.PagedCache(1, Hkv, D, n_pages=B * pages, n_seqs=B, max_pages=pages, page_tokens=page, dtype=dtype)
    seqs, n = ints(list(range(B))), ints(lens)
    cache.reserve(seqs, S)
    cache.append(seqs, k[:, :, :S].cuda(), v[:, :, :S].cuda(), count=n)
    cache.compact(seqs, torch.arange(S, dtype=torch.int32, device="cuda").expand(B, -1).contiguous(), n)
    cache.reserve(seqs, T)
    cache.append(seqs, k[:, :, S:].cuda(), v[:, :, S:].cuda())
    see, _ = R.ancestors(random_parents(np.random.default_rng(T), 1, T), [T])
    got = tree.attention(q.cuda(), cache, 0, seqs, R.pack(see, T).cuda()).double().cpu()
    cache.check()
    u = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -11
    for b, m in enumerate(lens):
        sees = torch.zeros(T, m + T, dtype=torch.bool)
        sees[:, :m] = True
        for t in range(T):
            sees[t, [m + j for j in see[0][t]]] = True
        kk, vv = (torch.cat([x[0, b, :m], x[0, b, S:]]).double().repeat_interleave(H // Hkv, 1).transpose(0, 1) for x in (k, v))      # [H, S, D]
        w = torch.softmax((q[b].double().transpose(0, 1) @ kk.transpose(1, 2) * D ** -0.5).masked_fill(~sees, -math.inf), -1)
        o = w @ vv
        spread = torch.stack([(w[:, t, :, None] * (vv - o[:, t, None]).abs()).sum(1) for t in range(T)], 1)
        small = (m + T) * 2.0 ** -25 * 8 if dtype == torch.float16 else 0                                     # (probabilities below fp16's normal numbers)
        tol = u * o.abs() + u / (1 - u) * spread + 1e-5 * o.abs() + small
        off = (got[b].transpose(0, 1) - o).abs() - tol
        assert (off <= 0).all(), (m, float(off.max()), float((off > 0).double().mean()))


def test_attention_grows_along_the_keys():
    """Scores that rise block by block, by more than a type's range at once: the running maximum is rescaled every time."""
    from paper_2203_16487_b200 import tree
    for dtype in (torch.bfloat16, torch.float16, torch.float32):
        S, D, page = 900, 64, 16
        q = torch.zeros(1, 1, 1, D)
        q[..., 0] = 8
        k, v = torch.zeros(S, 1, D), torch.randn(S, 1, D, generator=torch.Generator().manual_seed(1)).to(dtype).float()
        k[:, 0, 0] = (torch.arange(S) // 100 * 40 - 200).float()
        P = -(-S // page)
        kv = torch.zeros(1, 2, P, page, 1, D)
        kv[0, 0].view(-1, 1, D)[:S], kv[0, 1].view(-1, 1, D)[:S] = k, v
        cache = tree.PagedCache.over(kv.to(dtype).cuda(), torch.arange(P, dtype=torch.int32, device="cuda")[None], ints([S - 1]), ints([P]), ints([1] * P))
        got = tree.attention(q.to(dtype).cuda(), cache, 0, ints([0]), ints([[[1]]]))
        want, mag = R.attention(q[0], k, v, torch.ones(1, S, dtype=torch.bool), D ** -0.5)
        check_attention(got, want[None], mag[None], dtype, S)


def test_attention_far_pages():
    """A page whose elements lie beyond 2^31, of a cache that is larger than that."""
    from paper_2203_16487_b200 import tree
    free, _ = torch.cuda.mem_get_info()
    if free < 12 << 30:
        pytest.skip("needs 12 GB")
    P, page, H, D = 1100, 128, 64, 128
    kv = torch.zeros(1, 2, P, page, H, D, dtype=torch.bfloat16, device="cuda")     # 2.3e9 elements
    x = torch.randn(2, page, H, D, generator=torch.Generator().manual_seed(2)).bfloat16()
    kv[0, :, P - 1] = x.cuda()
    cache = tree.PagedCache.over(kv, ints([[P - 1]]), ints([page - 1]), ints([1]), ints([0] * P))
    q = torch.randn(1, 1, H, D, generator=torch.Generator().manual_seed(3)).bfloat16()
    got = tree.attention(q.cuda(), cache, 0, ints([0]), ints([[[1]]]))
    want, mag = R.attention(q[0], x[0], x[1], torch.ones(1, page, dtype=torch.bool), D ** -0.5)
    check_attention(got, want[None], mag[None], torch.bfloat16, page)


def test_attention_on_another_stream_and_again():
    """The same bits on another stream and on a second call; queries on the default stream's tensors."""
    got, _, _, (cache, q, seqs, bits, nodes) = attention_case(torch.bfloat16, [700, 3, 2000], 13, 8, 2, 64, 16, seed=4)
    from paper_2203_16487_b200 import tree
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        outs = [tree.attention(q, cache, 0, ints(seqs), bits, n_nodes=ints(nodes)) for _ in range(3)]
    side.synchronize()
    assert all(torch.equal(got, o) for o in outs)


def test_attention_refusals():
    from paper_2203_16487_b200 import binding, tree
    cache = tree.PagedCache(1, 2, 64, n_pages=4, n_seqs=2, max_pages=2)
    q, m = torch.randn(1, 3, 4, 64, device="cuda").bfloat16(), ints([[[1]] * 3])
    tree.attention(q, cache, 0, ints([0]), m)
    for bad in (lambda: tree.attention(q.half(), cache, 0, ints([0]), m), lambda: tree.attention(q[..., :32], cache, 0, ints([0]), m),
                lambda: tree.attention(q, cache, 0, ints([0, 1]), m), lambda: tree.attention(q, cache, 0, ints([0]), m.long()),
                lambda: tree.attention(q, cache, 0, ints([0]), ints([[[1]] * 2])), lambda: tree.attention(q, cache, 0, ints([0]), m, out=q[:, :2])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: tree.attention(q, cache, 1, ints([0]), m), lambda: tree.attention(q[:, :, :3], cache, 0, ints([0]), m),
                lambda: tree.attention(q, cache, 0, ints([0]), m, scale=0.0), lambda: tree.attention(q, cache, 0, ints([0]), m, scale=math.nan)):
        with pytest.raises(binding.SpecDecError):
            bad()
    with pytest.raises(binding.SpecDecError):
        tree.attention(q, cache, 0, ints([0]), m, scale=1e300)
    with pytest.raises(ValueError):
        tree.attention(q, cache, 1 << 40, ints([0]), m)
    for bad in (lambda: tree.attention(q, cache, 0, ints([0]).cpu(), m), lambda: tree.attention(q.cpu(), cache, 0, ints([0]), m), lambda: tree.sample(q[0, :, 0], q[0, :, 0, 0].float().cpu())):
        with pytest.raises(ValueError):
            bad()
    out = tree.attention(q, cache, 0, ints([7]), m)            # no such sequence: nothing to see
    assert (out == 0).all()


# ------------------------------------------------------------------ sampling
def check_sample(logits, u, temperature, top_k, top_p, min_p, most_near=None):
    """Tokens exactly, but where the row's own margin is within what fp32 exponentials can move it (1e-6); log probabilities to 1e-5 of their size.
    most_near: how many rows may have such a margin (V boundaries of u and V of top_p, 2e-6 of the row's weight each, and one or two by design)."""
    from paper_2203_16487_b200 import tree
    dev = lambda x, dt: torch.tensor(np.asarray(x), dtype=dt, device="cuda")  # noqa: E731
    R_, V = logits.shape
    token, logp = tree.sample(logits.cuda(), dev(u, torch.float32), dev(temperature, torch.float32), dev(top_k, torch.int32), dev(top_p, torch.float32), dev(min_p, torch.float32))
    token, logp, near = token.cpu().tolist(), logp.cpu().tolist(), 0
    f32 = lambda x: float(np.float32(x))  # noqa: E731
    for r in range(R_):
        want, lp, margin = R.sample_row(logits[r].float().numpy(), f32(u[r]), f32(temperature[r]), int(top_k[r]), f32(top_p[r]), f32(min_p[r]))
        if margin < 1e-6:
            near += 1
            continue
        assert token[r] == want, (r, token[r], want, margin)
        assert logp[r] == lp if math.isinf(lp) else abs(logp[r] - lp) <= 1e-5 * max(1, abs(lp)), (r, logp[r], lp)
    assert near <= (R_ * (0.02 + 4e-6 * V) + 2 if most_near is None else most_near)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("V", [1, 2, 31, 100, 513, 1000, 4097, 32768, 50265])
def test_sample_filters(dtype, V):
    rng = np.random.default_rng(V)
    rows = 60 if V < 5000 else 24
    logits = torch.from_numpy(rng.standard_normal((rows, V)).astype(np.float32) * rng.choice([0.1, 1, 3, 10], (rows, 1)).astype(np.float32)).to(dtype)
    u = rng.random(rows).astype(np.float32)
    u[:2] = 0, 1 - 2.0 ** -24
    check_sample(logits, u, rng.choice([0, 0.1, 0.7, 1, 2], rows), rng.choice([0, 1, 2, 7, 50, V - 1, V, V + 5], rows),
                 rng.choice([0, 0.1, 0.5, 0.9, 0.99, 1], rows), rng.choice([0, 0, 0.05, 0.5, 1], rows))


@pytest.mark.parametrize("what", ["equal", "few values", "two levels", "lowest", "infinities", "nan", "none", "one", "huge", "far"])
@pytest.mark.parametrize("V", [700, 9000])
def test_sample_hard_rows(what, V):
    """Ties beyond any list, masked entries of every kind, rows of nothing."""
    rng = np.random.default_rng(len(what) + V)
    rows = 24
    l = rng.standard_normal((rows, V)).astype(np.float32)
    if what == "equal":
        l[:] = 1.5
    elif what == "few values":
        l = rng.integers(0, 3, (rows, V)).astype(np.float32) * 0.25
    elif what == "two levels":
        l = np.where(rng.random((rows, V)) < 0.5, 0, -1e-6).astype(np.float32)
    elif what == "lowest":
        l[rng.random((rows, V)) < 0.9] = np.finfo(np.float32).min
    elif what == "infinities":
        l[rng.random((rows, V)) < 0.5] = -math.inf
        l[::2, 3] = math.inf
        l[::4, V - 1] = math.inf
    elif what == "nan":
        l[rng.random((rows, V)) < 0.5] = math.nan
    elif what == "none":
        l[:] = -math.inf
        l[::2] = math.nan
    elif what == "one":
        l[:] = -math.inf
        l[np.arange(rows), rng.integers(0, V, rows)] = -3e38
    elif what == "huge":
        l = np.clip(l, -3, 3) * np.float32(1e38)
    elif what == "far":
        l = (l * 1e-3 + 60000).astype(np.float32)
    temperature = rng.choice([0, 0.3, 1, 1.5], rows)
    check_sample(torch.from_numpy(l), rng.random(rows).astype(np.float32), temperature, rng.choice([0, 1, 40, V // 2], rows), rng.choice([1, 0.3, 0.95], rows), rng.choice([0, 0.02], rows),
                 most_near=rows // 2)                        # (few distinct weights: top_p of them is often a whole number of entries)


@pytest.mark.parametrize("V", [700, 50265])
def test_sample_parameters_that_are_no_numbers(V):
    """top_p and min_p of NaN cut nothing, as neither top_p < 1 nor min_p > 0 holds; a temperature of NaN is none above 0.  By every route: top-k small, large or off."""
    rng = np.random.default_rng(V)
    rows = 36
    l = (rng.standard_normal((rows, V)) * 2).astype(np.float32)
    p, m = rng.choice([1, 0.7, math.nan, math.inf], rows), rng.choice([0, 0.05, math.nan, -1], rows)
    p[:3], m[:3] = (math.nan, math.nan, 0.9), (math.nan, 0.1, math.nan)
    check_sample(torch.from_numpy(l), rng.random(rows).astype(np.float32), rng.choice([1, 0.7, math.nan], rows, p=[0.5, 0.4, 0.1]), rng.choice([0, 40, V // 2], rows), p, m)


def test_sample_parameters_and_strides():
    """No parameters, one for a run of rows, rows inside wider tensors that begin anywhere; the same token however the rows lie."""
    from paper_2203_16487_b200 import tree
    g = torch.Generator(device="cuda").manual_seed(1)
    wide = torch.randn(12, 1000, generator=g, device="cuda")
    logits, u = wide[:, 3:970], torch.rand(12, generator=g, device="cuda")
    a = tree.sample(logits, u)
    b = tree.sample(logits.contiguous().view(4, 3, 967), u.view(4, 3), torch.ones(4, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda"))
    assert torch.equal(a[0], b[0].view(-1)) and torch.equal(a[1], b[1].view(-1))
    t = torch.tensor([0.5, 1.0, 0.0, 2.0], device="cuda")
    c = tree.sample(logits.contiguous().view(4, 3, 967), u.view(4, 3), t)
    d = tree.sample(logits, u, t.repeat_interleave(3))
    assert torch.equal(c[0].view(-1), d[0]) and torch.equal(c[1].view(-1), d[1])
    assert tree.sample(logits[:0], u[:0])[0].shape == (0,)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [900, 32768, 50265, 131072, 262144])
def test_sample_is_the_same_by_every_route(V, dtype):
    """Weights are whole numbers, so nothing may depend on how a row is cut: alone (a cluster a row) and among many, and with a top-k that drops one entry of weight 0
    (which is found by other means than top-p alone).  Flat rows, whose cut lies among thousands of nearly equal entries, and steep ones."""
    from paper_2203_16487_b200 import tree
    rows = 160 if V < 100000 else 12
    g = torch.Generator(device="cuda").manual_seed(V)
    scale = torch.tensor([0.0, 1e-3, 0.05, 0.5, 2.0, 6.0], device="cuda").repeat(rows)[:rows, None]
    l = (torch.randn(rows, V, generator=g, device="cuda") * scale).to(dtype)
    l[:, V - 1] = -math.inf
    u = torch.rand(rows, generator=g, device="cuda")
    t = 0.3 + torch.rand(rows, generator=g, device="cuda")
    p = 0.02 + 0.979 * torch.rand(rows, generator=g, device="cuda")
    m = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.5, 0, 0.3 * torch.rand(rows, generator=g, device="cuda"))
    token, logp = tree.sample(l, u, t, None, p, m)
    k = torch.full((rows,), V - 1, dtype=torch.int32, device="cuda")
    again = tree.sample(l, u, t, k, p, m)
    assert torch.equal(token, again[0]) and torch.equal(logp, again[1])
    for r in range(0, rows, 7):
        one = tree.sample(l[r:r + 1], u[r:r + 1], t[r:r + 1], None, p[r:r + 1], m[r:r + 1])
        assert torch.equal(token[r:r + 1], one[0]) and torch.equal(logp[r:r + 1], one[1]), r


def test_sample_frequencies():
    """Many uniform numbers over one row: each token as often as its share, to the grid of the numbers."""
    from paper_2203_16487_b200 import tree
    V, n = 37, 1 << 14
    l = torch.randn(V, generator=torch.Generator().manual_seed(3))
    token, _ = tree.sample(l.cuda().expand(n, V).contiguous(), (torch.arange(n, device="cuda") + 0.5) / n)
    share = torch.bincount(token.cpu().long(), minlength=V) / n
    assert (share - torch.softmax(l.double(), 0)).abs().max() <= 1.0 / n + 1e-6


def test_sample_refusals():
    from paper_2203_16487_b200 import binding, tree
    l, u = torch.randn(4, 50, device="cuda"), torch.rand(4, device="cuda")
    for bad in (lambda: tree.sample(l.double(), u), lambda: tree.sample(l.T, u), lambda: tree.sample(l, u[:3]), lambda: tree.sample(l, u.half()),
                lambda: tree.sample(l, u, torch.ones(3, device="cuda")), lambda: tree.sample(l, u, torch.ones(4, device="cuda"), torch.ones(2, dtype=torch.int32, device="cuda")),
                lambda: tree.sample(l, u, top_k=torch.ones(4, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(binding.SpecDecError, match="262144"):
        tree.sample(torch.zeros(1, 262145, device="cuda"), u[:1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page", [1, 4, 16])
def test_strides_of_dimensions_of_one_do_not_matter(dtype, page):
    """Layers, pages, tokens, heads, sequences and entries of which there is one may come with any stride; the results are those of plain tensors."""
    from paper_2203_16487_b200 import tree
    D, g = 64, torch.Generator(device="cuda").manual_seed(page)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)  # noqa: E731
    def odd(x):
        """x again, with strides of 3, 5, 7, ... where its extent is 1."""
        c = x.clone(memory_format=torch.contiguous_format)
        y = torch.as_strided(c, c.shape, [s if m > 1 else 3 + 2 * i for i, (s, m) in enumerate(zip(c.stride(), c.shape))])
        assert torch.equal(x, y)
        return y
    for P, H in ((1, 1), (3, 1), (1, 2)):
        k, v, q, k1 = n(1, 1, page, H, D), n(1, 1, page, H, D), n(1, 1, 2 * H, D), n(1, 1, H, D)
        outs = []
        for f in (lambda x: x, odd):
            kv = f(torch.zeros(1, 2, P, page, H, D, dtype=dtype, device="cuda"))
            cache = tree.PagedCache.over(kv, ints([[-1]]), ints([0]), ints([0]), ints([0] * P))
            s = ints([0])
            cache.reserve(s, page)
            cache.append(s, f(k), v)                           # (strides of keys and values differ where there is one)
            cache.append(s, k1, f(k1), layer=0)
            if page > 1:                                       # (all but the last token committed; with none, its page would be given back)
                cache.compact(s, torch.arange(page, dtype=torch.int32, device="cuda")[None], ints([page - 1]))
            out = tree.attention(f(q), cache, 0, s, ints([[[1]]]), out=f(torch.zeros_like(q)))
            cache.check()
            outs.append((out, kv))
        assert torch.equal(*(o[0] for o in outs)) and torch.equal(*(o[1] for o in outs))
        assert torch.equal(outs[0][1][0, 0, 0, 0], k1[0, 0]) and not (outs[0][0] == 0).all()
    l, u = n(6, 50), torch.rand(6, generator=g, device="cuda")
    assert torch.equal(tree.sample(odd(l[:, 7:8]), u)[0], torch.zeros_like(u).int())
    assert torch.equal(tree.sample(l.T[7:8].T, u)[0], tree.sample(l[:, 7:8].contiguous(), u)[0])


def test_there_are_no_gradients_and_that_is_said():
    """Tensors that require a gradient give the same values, and an error where the gradient is asked for; without autograd nothing is kept of it."""
    from paper_2203_16487_b200 import tree
    def cache():
        return tree.PagedCache(1, 2, 64, n_pages=4, n_seqs=2, max_pages=2)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, q = torch.randn(1, 3, 2, 64, generator=g, device="cuda").bfloat16(), torch.randn(1, 3, 4, 64, generator=g, device="cuda").bfloat16()
    m, s = ints([[[1], [3], [7]]]), ints([0])
    def run(k, q, out=None):
        c = cache()
        c.reserve(s, 3)
        c.append(s, k, k, layer=0)
        return tree.attention(q, c, 0, s, m, out=out)
    want = run(k, q)
    assert not want.requires_grad
    for a, b in ((k, q.clone().requires_grad_()), (k.clone().requires_grad_(), q)):
        for out in (None, torch.empty_like(q)):
            got = run(a, b, out)
            assert torch.equal(got, want) and got.requires_grad
            with pytest.raises(RuntimeError, match="tree.attention has no gradient"):
                got.float().sum().backward()
        with torch.no_grad():
            got = run(a, b)
        assert torch.equal(got, want) and not got.requires_grad
    l, u, t = torch.randn(4, 50, generator=g, device="cuda"), torch.rand(4, generator=g, device="cuda"), torch.ones(4, device="cuda")
    want = tree.sample(l, u, t)
    for a, b in ((l.clone().requires_grad_(), t), (l, t.clone().requires_grad_())):
        token, logp = tree.sample(a, u, b)
        assert torch.equal(token, want[0]) and torch.equal(logp, want[1]) and logp.requires_grad and not token.requires_grad
        with pytest.raises(RuntimeError, match="tree.sample has no gradient"):
            logp.sum().backward()
        with torch.no_grad():
            assert not tree.sample(a, u, b)[1].requires_grad


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("batch,prompt,tokens", [(1, 1, 20), (5, 12, 48)])
def test_tree_decoding_is_sampling_token_by_token(batch, prompt, tokens):
    """The example: the same text with trees as without, in fewer steps (fp32: a near-tie that rounding decides is rarer than the run is long)."""
    from paper_2203_16487_b200 import tree_decode
    steps, fewer, same = tree_decode.main(["--batch", str(batch), "--prompt", str(prompt), "--tokens", str(tokens)])
    assert same == 1.0 and steps == tokens and fewer < steps


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_step_in_a_graph(dtype):
    """One step's calls, captured once and replayed while the sequences grow: bit for bit what calling them gives."""
    from paper_2203_16487_b200 import tree
    g = torch.Generator(device="cuda").manual_seed(6)
    L, B, T, H, Hkv, D, V, steps = 3, 5, 9, 8, 2, 64, 300, 12
    parents = ints(random_parents(np.random.default_rng(6), B, T))
    def new(*s):
        return torch.randn(*s, generator=g, device="cuda")
    steps = [dict(k=new(L, B, T, Hkv, D).to(dtype), v=new(L, B, T, Hkv, D).to(dtype), q=new(L, B, T, H, D).to(dtype), logits=new(B, T, V) * 3, u=torch.rand(B, T, generator=g, device="cuda"),
                  tokens=torch.randint(0, V, (B, T), generator=g, device="cuda").int()) for _ in range(steps)]
    seqs, k = ints([3, 0, 5, 1, 4]), torch.full((B,), 3, dtype=torch.int32, device="cuda")
    def call(cache, x):
        mask, depth = tree.ancestors(parents)
        cache.reserve(seqs, T)
        outs = [mask, depth]
        for layer in range(L):
            cache.append(seqs, x["k"][layer], x["v"][layer], layer=layer)
            outs.append(tree.attention(x["q"][layer], cache, layer, seqs, mask))
        outs += tree.sample(x["logits"], x["u"], top_k=k)
        outs += tree.accept(parents, x["tokens"], outs[-2])
        cache.compact(seqs, outs[-3], outs[-2])
        return outs
    for x in steps:                                            # drafts that the samples often follow
        sampled, _ = tree.sample(x["logits"], x["u"], top_k=k)
        x["tokens"][:, 1:] = sampled.gather(1, parents[:, 1:].long())
    caches = [tree.PagedCache(L, Hkv, D, n_pages=60, n_seqs=6, max_pages=10, page_tokens=16, dtype=dtype) for _ in range(2)]
    at, warm = {n: t.clone() for n, t in steps[0].items()}, tree.PagedCache(L, Hkv, D, n_pages=60, n_seqs=6, max_pages=10, page_tokens=16, dtype=dtype)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(warm, at)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed = call(caches[0], at)
    for x in steps:
        for n, t in x.items():
            at[n].copy_(t)
        graph.replay()
        for a, b in zip(replayed, call(caches[1], x)):
            assert torch.equal(a, b)
    for c in caches:
        c.check()
    assert torch.equal(caches[0].length, caches[1].length) and torch.equal(caches[0].kv, caches[1].kv) and torch.equal(caches[0].table, caches[1].table)
    assert int(caches[0].length.max()) > 2 * len(steps)


def test_branches_of_a_prompt():
    """Forked sequences continue a shared prompt each its own way, as sequences that hold copies of it would."""
    from paper_2203_16487_b200 import tree
    g = torch.Generator(device="cuda").manual_seed(5)
    H, D, n, ways = 2, 64, 37, 3
    cache = tree.PagedCache(1, H, D, n_pages=40, n_seqs=2 * ways + 1, max_pages=8, page_tokens=16, dtype=torch.float32)
    k, v = (torch.randn(1, n, H, D, generator=g, device="cuda") for _ in "kv")
    chain = torch.arange(n, dtype=torch.int32, device="cuda")[None]
    copies = ints(list(range(ways + 1, 2 * ways + 1)))
    for seqs in [ints([0])] + [copies[i:i + 1] for i in range(ways)]:
        cache.reserve(seqs, n)
        cache.append(seqs, k, v, layer=0)
        cache.compact(seqs, chain, ints([n]))
    branches = ints(list(range(1, ways + 1)))
    cache.fork(ints([0] * ways), branches)
    assert cache.refs.max() == ways + 1
    new = torch.randn(ways, 20, H, D, generator=g, device="cuda")
    q = torch.randn(ways, 20, 4, D, generator=g, device="cuda")
    mask, _ = tree.ancestors(torch.arange(-1, 19, dtype=torch.int32, device="cuda").expand(ways, -1).contiguous())
    outs = []
    for seqs in (branches, copies):
        cache.reserve(seqs, 20)
        cache.append(seqs, new, new, layer=0)
        outs.append(tree.attention(q, cache, 0, seqs, mask))
    cache.check()
    assert torch.equal(outs[0], outs[1])
