"""The cache in 4 bits and the reordering of beams, against plain implementations in 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests import fp4_reference as F
from tests import tree_reference as R
from tests.test_gpu_tree import ints, random_parents

pytestmark = pytest.mark.gpu


def bytes_of(cache):
    """[L, 2, P, page, H, D / 2 + D / 16] on the CPU: codes and scales of a token and head."""
    return torch.cat((cache.codes, cache.scales.view(torch.uint8)), -1).transpose(3, 4).cpu()


def empty(L, H, D, P, page, n_seqs, max_pages, unit=None, fill=None):
    from paper_2203_16487_b200 import fp4
    cache = fp4.Fp4Cache(L, H, D, n_pages=P, n_seqs=n_seqs, max_pages=max_pages, page_tokens=page, unit=unit)
    if fill is not None:
        g = torch.Generator(device="cuda").manual_seed(fill)
        cache.codes.random_(0, 256, generator=g)
        cache.scales.view(torch.uint8).random_(0, 127, generator=g)
    return cache


def hard_numbers(shape, dtype, seed):
    """Blocks of every kind: normal ones, whole multiples (halfway between codes and between scales), tiny and huge ones, zeros, one value alone, infinities, NaN."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(*shape[:-1], shape[-1] // 16, 16, generator=g)
    kind = torch.randint(0, 12, x.shape[:-1], generator=g)[..., None]
    whole = torch.randint(-48, 49, x.shape, generator=g).float()
    x = torch.where(kind == 1, whole / 8, x)
    x = torch.where(kind == 2, whole * 0.21875, x)
    x = torch.where(kind == 3, x * 2.0 ** -9, x)
    x = torch.where(kind == 4, x * 2.0 ** -13, x)
    x = torch.where(kind == 5, x * (1000 if dtype == torch.float16 else 1e5), x)
    x = torch.where(kind == 6, torch.where(whole > 40, x, -0.0), x)
    x = torch.where(kind == 7, whole * 56, x)                  # beyond what the largest scale reaches
    x = torch.where((kind == 8) & (whole > 45), math.inf, x)
    x = torch.where((kind == 9) & (whole > 45), math.nan, x)
    x = torch.where(kind == 10, torch.zeros_like(x), x)
    return x.flatten(-2).to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("L,H,D,page,T,unit", [(1, 1, 64, 16, 1, None), (2, 3, 64, 16, 37, None), (3, 2, 128, 32, 70, None), (1, 12, 128, 16, 5, 0.037), (2, 2, 64, 64, 130, 3.0)])
def test_append_and_read(dtype, L, H, D, page, T, unit):
    """Codes and scales to the bit, what they stand for to the bit, nothing beside them touched."""
    n, spare = 3, 8
    units = None if unit is None else torch.rand(L, 2, H, device="cuda") * unit + unit
    per = -(-(20 + T) // page)
    cache = empty(L, H, D, n * per + 2, page, n + 1, per + 1, unit=units, fill=1)
    ref = F.Pages(bytes_of(cache), n + 1, per + 1)
    seqs, lens = [2, 0, 3], [5, 0, 20]
    for s, m in zip(seqs, lens):
        ref.length[s] = m
    cache.length.copy_(torch.tensor(ref.length))
    cache.reserve(ints(seqs), T)
    assert ref.reserve(seqs, T) == 0
    wide = hard_numbers((2, L, n, T, H, D + 16 * spare), dtype, T).cuda()
    k, v = wide[0, ..., :D], wide[1, ..., 16:16 + D]           # strided rows
    count = [T, max(T - 3, 0), T]
    if L == 2:
        for i in range(L):
            cache.append(ints(seqs), k[i], v[i], layer=i, count=ints(count))
    else:
        cache.append(ints(seqs), k, v, count=ints(count))
    cache.check()
    rows = []
    for side, x in enumerate((k, v)):
        x = x.cpu()
        both = [[torch.cat(F.quantise(x[l, :, :, h], None if units is None else units[l, side, h].item()), -1) for h in range(H)] for l in range(L)]
        rows.append(torch.stack([torch.stack(b, 2) for b in both]))
    ref.append(seqs, rows[0], rows[1], range(L), count)
    got = bytes_of(cache)
    half = D // 2
    scale = ref.kv[..., half:]
    good = ((scale & 127) != 127).repeat_interleave(8, -1)     # the codes of a NaN block do not matter
    assert torch.equal(got[..., half:], scale)
    a, b = got[..., :half][good], ref.kv[..., :half][good]
    zero = ((a ^ b) & 0x77) == 0                               # (a zero of either sign)
    assert ((a == b) | (zero & (((a ^ b) & 0x80 == 0) | (a & 0x70 == 0)) & (((a ^ b) & 0x08 == 0) | (a & 0x07 == 0)))).all()
    for start in (None, [0, 1, 3]):
        for out in (torch.float32, torch.bfloat16, torch.float16):
            kk, vv = cache.read(ints(seqs), T + 2, start=None if start is None else ints(start), dtype=out)
            for side, x in enumerate((kk, vv)):
                for i, s in enumerate(seqs):
                    first = lens[i] if start is None else start[i]
                    for t in range(T + 2):
                        row = torch.zeros(L, H, D, dtype=torch.float64)
                        if (first + t) // page < len(ref.table[s]):
                            p, o = ref.at(s, first + t)
                            row = F.values(ref.kv[:, side, p, o, :, :half], ref.kv[:, side, p, o, :, half:])
                            if units is not None:              # one product in fp32, then the type's rounding
                                row = (row.float() * units[:, side, :, None].cpu()).double()
                        want = row.to(out)
                        y = x[:, i, t].cpu()
                        assert ((y == want) | (y.isnan() & want.isnan())).all(), (side, i, t)
    one = cache.read(ints([3, 3]), 1, layer=L - 1)             # a sequence twice
    assert torch.equal(one[0][0].nan_to_num(7), one[0][1].nan_to_num(7))


def same(cache, ref):
    assert cache.length.tolist() == ref.length and cache.refs.tolist() == ref.refs
    assert cache.held.tolist() == [len(t) for t in ref.table]
    assert cache.table.tolist() == [t + [-1] * (ref.max_pages - len(t)) for t in ref.table]
    assert torch.equal(cache.kv.cpu() if hasattr(cache, "kv") else bytes_of(cache), ref.kv)


@pytest.mark.parametrize("kind,page,H,D,L", [("4", 16, 2, 64, 2), ("4", 32, 3, 128, 1), ("4", 16, 1, 64, 3), ("16", 16, 2, 64, 2), ("16", 4, 3, 24, 1), ("heads first", 8, 2, 16, 2)])
def test_pages_random_walk(kind, page, H, D, L):
    """Every call, in random order, with calls that find too few pages among them: tables, counts and contents as one token at a time gives them."""
    from paper_2203_16487_b200 import tree
    rng = np.random.default_rng(page * 7 + H + D)
    n_seqs, max_pages, n_pages, T = 12, 5, 19, 2 * page + 3
    if kind == "4":
        cache = empty(L, H, D, n_pages, page, n_seqs, max_pages, fill=2)
        ref = F.Pages(bytes_of(cache), n_seqs, max_pages)
    else:
        kv = torch.randn(L, 2, n_pages, H, page, D, device="cuda").half().transpose(3, 4) if kind == "heads first" else torch.randn(L, 2, n_pages, page, H, D, device="cuda").half()
        cache = tree.PagedCache.over(kv, torch.full((n_seqs, max_pages), -1, dtype=torch.int32, device="cuda"), ints([0] * n_seqs), ints([0] * n_seqs), ints([0] * n_pages))
        ref = F.Pages(kv.cpu(), n_seqs, max_pages)
    refused = moved = 0
    for step in range(400):
        if step >= 90 and refused and moved:
            break
        seqs = rng.permutation(n_seqs)[:rng.integers(1, 5)].tolist()
        what = rng.choice(["block", "block", "fork", "beams", "beams", "beams", "reserve", "release"])
        status = 0
        if what == "block":
            t = int(rng.integers(1, T + 1))
            status = ref.reserve(seqs, t)
            cache.reserve(ints(seqs), t)
            if status == 0:
                k, v = (torch.randn(L, len(seqs), t, H, D, device="cuda").half() for _ in "kv")
                cache.append(ints(seqs), k, v)
                if kind == "4":
                    k, v = (torch.cat(F.quantise(x.cpu()), -1) for x in (k, v))
                ref.append(seqs, k.cpu(), v.cpu(), range(L), [t] * len(seqs))
                paths = [sorted(rng.permutation(t)[:rng.integers(0, t + 1)].tolist()) for _ in seqs]
                pad = [p + [-1] * (t - len(p)) for p in paths]
                cache.compact(ints(seqs), ints(pad), ints([len(p) for p in paths]))
                ref.compact(seqs, paths)
        elif what == "reserve":                                # pages behind the committed tokens, which a reordering gives back
            status = ref.reserve(seqs, 3)
            cache.reserve(ints(seqs), 3)
        elif what == "release":
            cache.release(ints(seqs))
            ref.release(seqs)
        elif what == "fork":
            dst = rng.permutation(n_seqs)[:len(seqs)].tolist()
            status = ref.fork(seqs, dst)
            cache.fork(ints(seqs), ints(dst))
        else:
            k = int(rng.choice([1, 2, 3, 4, 6, 12]))
            groups = rng.permutation(n_seqs)[:n_seqs // k * k].reshape(-1, k)[:int(rng.integers(1, n_seqs // k + 1))].tolist()
            parents = rng.integers(0, k, (len(groups), k))
            if rng.random() < 0.3:
                parents[rng.random(parents.shape) < 0.2] = -1
            if rng.random() < 0.2:
                parents[0, -1] = rng.choice([k, -2, 10 ** 6])
            if rng.random() < 0.2:
                groups[-1][0] = int(rng.choice([n_seqs, -1, 10 ** 6]))
            status = ref.reorder(groups, parents.tolist())
            cache.reorder(ints(groups), ints(parents.tolist()))
            moved += status & 1 == 0
        assert int(cache.status.item()) == status, (step, what)
        refused += status & 1
        cache.status.zero_()
        same(cache, ref)
        # a token that can still be written belongs to one sequence alone
        assert all(ref.refs[p] == 1 for s in range(n_seqs) for p in ref.table[s][ref.length[s] // page:])
    assert refused and moved, "the walk should meet a full pool"


def test_reorder_of_many_beams():
    """More entries than a CTA has threads, groups wider than one, permutations that move nothing."""
    from paper_2203_16487_b200 import tree
    rng = np.random.default_rng(3)
    n, K, page = 1500, 1500, 4
    cache = tree.PagedCache(1, 1, 8, n_pages=3 * n, n_seqs=n, max_pages=3, page_tokens=page, dtype=torch.float32)
    cache.kv.normal_()
    ref = F.Pages(cache.kv.cpu(), n, 3)
    seqs = list(range(n))
    lens = [int(x) for x in rng.integers(0, 11, n)]
    for c in (cache, ref):
        c.reserve(ints(seqs) if c is cache else seqs, 10)
    path = [list(range(m)) for m in lens]
    cache.compact(ints(seqs), ints([p + [-1] * (10 - len(p)) for p in path]), ints(lens))
    ref.compact(seqs, path)
    same(cache, ref)
    for K, parents in ((1500, rng.integers(0, 300, (1, 1500))), (1500, rng.permutation(1500)[None]), (30, rng.integers(0, 30, (50, 30))), (1, np.zeros((1500, 1), int))):
        groups = rng.permutation(n).reshape(-1, K).tolist()
        before = cache.kv.clone()
        assert ref.reorder(groups, parents.tolist()) == 0
        cache.reorder(ints(groups), ints(parents.tolist()))
        cache.check()
        same(cache, ref)
        if K == 1 or (K == 1500 and len(set(parents[0])) == K):
            assert torch.equal(cache.kv, before)


@pytest.mark.parametrize("n,K,H,D,page,L", [(1100, 550, 1, 64, 16, 2), (1400, 100, 3, 128, 16, 1), (200, 100, 2, 64, 64, 1)])
def test_reorder_of_many_beams_in_4_bits(n, K, H, D, page, L):
    """Codes and scales of more entries, or wider groups, than one CTA settles."""
    rng = np.random.default_rng(n)
    cache = empty(L, H, D, 2 * n, page, n, 2, fill=n)
    ref = F.Pages(bytes_of(cache), n, 2)
    seqs, top = list(range(n)), 2 * page - 1
    lens = [int(x) for x in rng.integers(0, top + 1, n)]
    cache.reserve(ints(seqs), top)
    ref.reserve(seqs, top)
    path = [list(range(m)) for m in lens]
    cache.compact(ints(seqs), ints([p + [-1] * (top - len(p)) for p in path]), ints(lens))
    ref.compact(seqs, path)
    for _ in range(2):
        groups = rng.permutation(n).reshape(-1, K).tolist()
        parents = rng.integers(0, K, (n // K, K))
        parents[0, ::7] = -1
        assert ref.reorder(groups, parents.tolist()) == 0
        cache.reorder(ints(groups), ints(parents.tolist()))
        cache.check()
        same(cache, ref)


# ------------------------------------------------------------------ attention
def attention_case(dtype, lens, T, H, Hkv, D, page, *, nodes=None, one_mask=False, seed=0, strided=False, mask=None, layer=0, spare=0, unit=None, q_times=2.0):
    """A cache with those lengths (the scales of slots that nobody sees are NaN), queries, masks, and the answer in 64 bits."""
    from paper_2203_16487_b200 import fp4, tree
    rng = np.random.default_rng(seed)
    g = torch.Generator().manual_seed(seed)
    B, L = len(lens), layer + 1
    nodes = [T] * B if nodes is None else nodes
    held = [-(-(n + T) // page) for n in lens]
    P = sum(held) + 2
    codes = torch.randint(0, 256, (L, 2, P, Hkv, page, D // 2), dtype=torch.uint8, generator=g)
    scales = torch.full((L, 2, P, Hkv, page, D // 16), 127, dtype=torch.uint8)
    units = None if unit is None else torch.rand(L, 2, Hkv, generator=g) * unit + unit
    table = torch.full((B + 1, max(held) + spare), -1, dtype=torch.int32)
    seqs = rng.permutation(B + 1)[:B]
    order = rng.permutation(P)[:sum(held)]
    length = torch.zeros(B + 1, dtype=torch.int32)
    parents = random_parents(rng, B, T)
    see_nodes, _ = R.ancestors(parents, [T] * B)
    if one_mask:
        see_nodes = [see_nodes[0]] * B
    if mask is not None:
        see_nodes = [mask(b) for b in range(B)]
    q = torch.randn(B, T, H, D, generator=g).mul(q_times).to(dtype)
    want, mag = torch.zeros(B, T, H, D, dtype=torch.float64), torch.zeros(B, T, H, D, dtype=torch.float64)
    at = 0
    for b in range(B):
        n, s = lens[b], int(seqs[b])
        pages = torch.from_numpy(order[at:at + held[b]])
        at += held[b]
        table[s, :held[b]] = pages.int()
        length[s] = n
        S = n + nodes[b]
        c, z = F.quantise(torch.randn(2, S, Hkv, D, generator=g))
        see = torch.zeros(T, S, dtype=torch.bool)
        for t in range(nodes[b]):
            see[t, :n] = True
            for j in see_nodes[b][t]:
                if j < nodes[b]:
                    see[t, n + j] = True
        j = torch.arange(S)
        j = j[(j < n) | see.any(0)]                            # what nobody sees stays NaN
        codes[layer, :, pages[j // page], :, j % page] = c[:, j].transpose(0, 1)
        scales[layer, :, pages[j // page], :, j % page] = z[:, j].transpose(0, 1)
        x = F.values(c, z)
        if units is not None:
            x = x * units[layer].double()[:, None, :, None]
        want[b], mag[b] = R.attention(q[b], x[0], x[1], see, D ** -0.5)
    hold = torch.zeros_like(length).cuda()
    cache = fp4.Fp4Cache.over(codes.cuda(), scales.cuda().view(torch.float8_e4m3fn), table.cuda(), length.cuda(), hold, ints([0] * P), None if units is None else units.cuda())
    qd, out = q.cuda(), None
    if strided:                                                # rows inside a wider tensor, at odd places
        wide = torch.zeros(B, T, H * D * 3 + 1, dtype=dtype, device="cuda")
        wide[..., 1:1 + H * D] = qd.reshape(B, T, -1)
        qd = wide[..., 1:1 + H * D].unflatten(-1, (H, D))
        out = torch.zeros(B, H, T, D + 3, dtype=dtype, device="cuda")[..., 1:1 + D].transpose(1, 2)
    bits = R.pack([see_nodes[0]] if one_mask else see_nodes, T).cuda()
    got = tree.attention(qd, cache, layer, ints(seqs), bits, n_nodes=ints(nodes), out=out)
    cache.check()
    return got, want, mag, (cache, qd, seqs, bits, nodes)


def check_attention(got, want, mag, dtype, times=1.0):
    """Probabilities are rounded to fp16, by 2^-11 of themselves (fp32: in two parts, 2^-22), and so is their sum's share of each; the output once to its type.  The products are exact, the
    rest is fp32 sums: the 1e-5, as for the other caches, and 1e-6 of the values' size."""
    got = got.double().cpu()
    u = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[dtype]
    p = 2.0 ** -22 if dtype == torch.float32 else 2.0 ** -11
    tol = 2 * p * mag + u * want.abs() + 1e-5 * mag + (1e-7 if dtype == torch.float32 else 1e-6) * times
    off = (got - want).abs() - tol
    assert not got.isnan().any() and (off <= 0).all(), (float((got - want).abs().max()), float(off.max()))


ALL = [torch.bfloat16, torch.float16, torch.float32]


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("H,Hkv,D", [(8, 8, 64), (8, 2, 128), (6, 1, 64), (32, 2, 128), (5, 5, 128)])
@pytest.mark.parametrize("T,page", [(1, 16), (5, 32), (26, 16), (33, 64), (70, 128)])
def test_attention_layouts(dtype, H, Hkv, D, T, page):
    got, want, mag, _ = attention_case(dtype, [0, 1, 63, 130], T, H, Hkv, D, page, seed=T + D)
    check_attention(got, want, mag, dtype)


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("T,H,Hkv,D,lens", [(1, 8, 2, 64, [3000]), (1, 4, 4, 128, [2047, 1, 2048]), (3, 8, 1, 128, [1500, 0]), (64, 8, 4, 64, [1029]), (17, 8, 8, 64, [64, 700]), (17, 4, 4, 128, [900, 5])])
def test_attention_split_keys(dtype, T, H, Hkv, D, lens):
    """Few rows over long caches: keys split over CTAs, also where a sequence of the batch is short."""
    got, want, mag, _ = attention_case(dtype, lens, T, H, Hkv, D, 32, seed=5, spare=200)
    check_attention(got, want, mag, dtype)


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("T,H,Hkv,D,n", [(2, 12, 12, 64, 41), (2, 12, 12, 128, 41), (20, 12, 12, 64, 41), (3, 48, 4, 64, 60), (20, 12, 12, 128, 30), (66, 7, 7, 64, 30), (130, 6, 3, 64, 30),
                                         (66, 7, 7, 128, 30), (40, 12, 12, 64, 41), (11, 12, 12, 64, 41), (4, 48, 12, 128, 41), (13, 16, 16, 128, 61)])
def test_attention_many_short_sequences(dtype, T, H, Hkv, D, n):
    """More sequences and heads than CTAs that run at once, of every number of key blocks: CTAs that take several."""
    lens = [(i * 37) % 331 for i in range(n)]
    got, want, mag, _ = attention_case(dtype, lens, T, H, Hkv, D, 16, seed=T, one_mask=True)
    check_attention(got, want, mag, dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H,Hkv,D", [(1, 4, 2, 64), (9, 2, 2, 128), (12, 4, 2, 64), (40, 2, 1, 64), (100, 2, 2, 128), (90, 3, 1, 64)])
def test_attention_uneven_long_sequences(dtype, T, H, Hkv, D):
    """Sequences of one to thousands of keys: CTAs whose stretch of keys begins and ends inside sequences, or holds several."""
    got, want, mag, _ = attention_case(dtype, [5000, 0, 3, 1900, 64, 65, 0, 700], T, H, Hkv, D, 16, seed=T, one_mask=True, nodes=[T, T, 1, T, 0, T, 0, T])
    check_attention(got, want, mag, dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("H,Hkv,D", [(2, 1, 64), (2, 1, 128), (4, 1, 128)])
def test_attention_many_rows(dtype, H, Hkv, D):
    """Tiles of 128 and 256 rows: none, one, two, three and many blocks of keys, parts of a long sequence, the same bits every time."""
    from paper_2203_16487_b200 import tree
    T, lens = 50, [0, 70, 128 - 50, 206, 300, 1000, 6000]
    got, want, mag, (cache, q, seqs, bits, nodes) = attention_case(dtype, lens, T, H, Hkv, D, 16, seed=11, nodes=[T, T, T, T, 7, T, T])
    check_attention(got, want, mag, dtype)
    for _ in range(20):
        assert torch.equal(got, tree.attention(q, cache, 0, ints(seqs), bits, n_nodes=ints(nodes)))


@pytest.mark.parametrize("T,H,Hkv,D,lens", [(1024, 1, 1, 128, [70]), (970, 2, 1, 128, [0]), (1024, 1, 1, 64, [5, 1]), (300, 3, 1, 128, [129, 0]), (250, 1, 1, 128, [300]), (40, 12, 12, 64, [(i * 53) % 400 for i in range(41)])])
def test_attention_wide_trees(T, H, Hkv, D, lens):
    got, want, mag, _ = attention_case(torch.bfloat16, lens, T, H, Hkv, D, 32, seed=T, one_mask=len(lens) > 5)
    check_attention(got, want, mag, torch.bfloat16)


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("T", [9, 70])
@pytest.mark.parametrize("kw", [dict(nodes=[9, 0, 3]), dict(one_mask=True), dict(strided=True), dict(layer=2), dict(nodes=[1, 9, 8], strided=True), dict(unit=0.02, q_times=50.0), dict(unit=7.0, q_times=0.1, layer=1)])
def test_attention_ragged_shared_strided(dtype, T, kw):
    got, want, mag, _ = attention_case(dtype, [40, 65, 0], T, 8, 4, 64, 16, seed=3, **kw)
    check_attention(got, want, mag, dtype, 2 * kw.get("unit", 0.5))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("size", [1e-30, 1e-6, 1e4, 1e30])
def test_attention_queries_of_any_size(dtype, size):
    """Rows beyond what fp16 holds, among them rows of zeros: a row is scaled by a power of two of its own.  The unit brings the scores back to the usual size."""
    from paper_2203_16487_b200 import tree
    got, want, mag, (cache, q, seqs, bits, nodes) = attention_case(dtype, [100, 3], 20, 4, 2, 64, 16, seed=4)
    rows = torch.where(torch.arange(20, device="cuda") % 3 == 0, 1.0, size)[None, :, None, None]
    q2 = (q.float() * 0.5).to(dtype)
    big = (q2.float() * rows).to(dtype)
    scale = 64 ** -0.5
    g1 = tree.attention(big, cache, 0, ints(seqs), bits, n_nodes=ints(nodes), scale=scale / size)
    g2 = tree.attention((big.double() / size).to(torch.float32).to(dtype), cache, 0, ints(seqs), bits, n_nodes=ints(nodes), scale=scale)
    same_rows = torch.arange(20) % 3 != 0
    u = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -22}[dtype]      # (the division by `size` rounds the query; values are up to 6 in size)
    assert g1.isfinite().all() and ((g1 - g2).abs()[:, same_rows] <= 40 * 6 * u).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H,Hkv,D,page", [(1, 8, 2, 128, 16), (20, 4, 4, 64, 64), (50, 4, 4, 64, 16), (50, 8, 4, 128, 32), (64, 16, 4, 64, 128)])
def test_attention_pages_that_are_none(dtype, T, H, Hkv, D, page):
    """Table entries below zero or beyond the pages read as a page of zeros, whatever else is on its way, and later blocks are as they were."""
    from paper_2203_16487_b200 import tree
    _, _, _, (cache, q, seqs, bits, nodes) = attention_case(dtype, [700, 0, 331], T, H, Hkv, D, page, seed=4)
    free = sorted(set(range(cache.refs.numel())) - set(cache.table.flatten().tolist()))[0]
    cache.codes[:, :, free], cache.scales.view(torch.uint8)[:, :, free] = 0, 0
    at = [(0, 1), (0, 600 // page), (2, 0)]
    out = []
    for fill in (free, -1, cache.refs.numel(), 2 ** 31 - 1, -2 ** 31):
        for b, i in at:
            cache.table[int(seqs[b]), i] = fill
        out.append(tree.attention(q, cache, 0, ints(seqs), bits, n_nodes=ints(nodes)))
    cache.check()
    assert all(torch.equal(x, out[0]) for x in out) and out[0].isfinite().all()


@pytest.mark.parametrize("dtype", ALL)
def test_attention_masks(dtype):
    """Queries that see nothing, nodes that nobody sees (their slots hold NaN), nodes that see later ones."""
    for T, H in ((40, 4), (40, 8)):
        def mask(b):
            return [set() if t % 3 == 0 else {T - 1, t} if t % 3 == 1 else {1, 34} for t in range(T)]
        got, want, mag, _ = attention_case(dtype, [0, 7], T, H, 2, 64, 16, seed=9, mask=mask)
        check_attention(got, want, mag, dtype)
        assert (got[0, ::3] == 0).all()


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("T,H", [(1, 4), (64, 4)])
def test_attention_many_small_weights(dtype, T, H):
    """One key that weighs 2^15 times what each of 30000 others does: what is small must not be lost.  A 1 is held as 6 * 11 / 64 (the scale nearest to 1 / 6 is 11 / 64)."""
    from paper_2203_16487_b200 import fp4, tree
    n, D, page = 30000, 64, 64
    P = -(-(n + T) // page)
    cache = fp4.Fp4Cache(1, 1, D, n_pages=P, n_seqs=1, max_pages=P, page_tokens=page)
    seqs = ints([0])
    cache.reserve(seqs, n + T)
    x = torch.zeros(2, 1, 1, n + T, 1, D, device="cuda")
    x[0, ..., 0] = -6.0                                        # keys: one channel; scores -6 c and 0 for the one
    x[0, 0, 0, 77] = 0
    x[1, ..., 1] = 1.0
    x[1, 0, 0, 77] = 0
    x[1, 0, 0, 77, 0, 2] = 1.0
    cache.append(seqs, x[0], x[1])
    cache.length.fill_(n)
    q = torch.zeros(1, T, H, D, device="cuda", dtype=dtype)
    q[..., 0] = 1.0
    scale = 15 * math.log(2) / 6
    got = tree.attention(q, cache, 0, seqs, torch.zeros(1, T, (T + 31) // 32, dtype=torch.int32, device="cuda"), scale=scale).double().cpu()
    small = (n - 1) * 2.0 ** -15
    u = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[dtype]
    tol = u + 2.0 ** -11 + 1e-5 if dtype != torch.float32 else 2e-5
    held = 6 * 11 / 64
    worst = float((got[..., 1] - held * small / (1 + small)).abs().max()), float((got[..., 2] - held / (1 + small)).abs().max())
    assert max(worst) <= held * tol, worst


def test_operators_say_that_there_is_no_gradient_and_refuse():
    from paper_2203_16487_b200 import binding, fp4, tree
    cache = empty(2, 2, 64, 4, 16, 2, 2, fill=3)
    seqs, one = ints([0]), ints([[[1]]])
    cache.reserve(seqs, 1)
    k = torch.randn(1, 1, 2, 64, device="cuda", requires_grad=True)
    q = torch.randn(1, 1, 2, 64, device="cuda", requires_grad=True)
    with pytest.raises(RuntimeError, match="no gradient"):
        tree.attention(q, cache, 0, seqs, one).sum().backward()
    cache.append(seqs, k, k, layer=0)
    with pytest.raises(RuntimeError, match="no gradient"):
        tree.attention(q.detach(), cache, 0, seqs, one).sum().backward()
    k = k.detach()
    codes, scales = cache.codes, cache.scales
    books = (cache.table, cache.length, cache.held, cache.refs)
    for bad in (lambda: cache.append(seqs, k.double(), k.double(), layer=0), lambda: cache.append(seqs, k, k), lambda: cache.append(seqs, k[..., :32], k[..., :32], layer=0),
                lambda: cache.append(seqs, k, k.half(), layer=0), lambda: cache.read(seqs, 1, dtype=torch.float64), lambda: cache.read(seqs, -1), lambda: cache.read(seqs.long(), 1),
                lambda: cache.reorder(ints([[0, 1]]), ints([0, 1])), lambda: cache.reorder(torch.tensor([[0]]), ints([[0]])), lambda: tree.attention(q.double(), cache, 0, seqs, one),
                lambda: tree.attention(q[..., :32], cache, 0, seqs, one), lambda: fp4.Fp4Cache.over(codes.int(), scales, *books), lambda: fp4.Fp4Cache.over(codes, scales.view(torch.uint8), *books),
                lambda: fp4.Fp4Cache.over(codes[..., :16], scales, *books), lambda: fp4.Fp4Cache.over(codes, scales, *books, unit=torch.ones(2, 2, 3, device="cuda")),
                lambda: fp4.Fp4Cache.over(codes.transpose(3, 4), scales.transpose(3, 4), *books)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: cache.append(seqs, k, k, layer=2), lambda: cache.read(seqs, 1, layer=-1), lambda: cache.reserve(ints([0, 1, 0]), 1), lambda: fp4.Fp4Cache(1, 1, 64, n_pages=2, n_seqs=1, max_pages=1, page_tokens=8).release(seqs),
                lambda: tree.attention(q.detach(), cache, 2, seqs, one)):
        with pytest.raises(binding.SpecDecError):
            bad()
    cache.append(ints([5]), k, k, layer=0)
    with pytest.raises(binding.SpecDecError, match="out of range"):
        cache.check()
    cache.append(ints([1]), k, k, layer=0)
    with pytest.raises(binding.SpecDecError, match="reserved"):
        cache.check()


def test_a_step_captured_and_replayed_while_sequences_grow():
    """reserve, append, attention, compact of one token and a reordering of the beams, captured once; replays equal calls one by one."""
    from paper_2203_16487_b200 import tree
    B, H, D, steps = 4, 2, 64, 40
    a, b = (empty(1, H, D, 24, 16, B, 5, fill=5) for _ in "ab")
    seqs, one = ints([[0, 1, 2, 3]]), ints([[[1]]])
    x = torch.randn(steps, 3, B, 1, H, D, device="cuda").half()
    up = torch.randint(0, B, (steps, 1, B), device="cuda").int()
    now, parents = torch.zeros_like(x[0]), torch.zeros_like(up[0])
    out = torch.zeros(B, 1, H, D, device="cuda").half()
    path, n_path = ints([[0]] * B), ints([1] * B)

    def step(cache):
        flat = seqs.view(-1)
        cache.reserve(flat, 1)
        cache.append(flat, now[0], now[1], layer=0)
        tree.attention(now[2], cache, 0, flat, one, out=out)
        cache.compact(flat, path, n_path)
        cache.reorder(seqs, parents)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        step(b)                                                # (limits and workspaces are set)
        b.release(seqs.view(-1))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step(b)
    torch.cuda.synchronize()
    b.codes.copy_(a.codes), b.scales.view(torch.uint8).copy_(a.scales.view(torch.uint8))
    for i in range(steps):
        now.copy_(x[i]), parents.copy_(up[i])
        step(a)
        first = out.clone()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(first, out), i
    a.check(), b.check()
    assert torch.equal(bytes_of(a), bytes_of(b)) and a.table.tolist() == b.table.tolist() and a.length.tolist() == [steps] * B
