"""Attention whose scores are larger than their own differences, over every kind of cache: with one clear winner a row the answer is the winner's value, however large the scores."""
import math

import numpy as np
import pytest
import torch

from tests import tree_reference as R
from tests.test_gpu_tree import ints

pytestmark = pytest.mark.gpu
KINDS = [("4", torch.bfloat16), ("4", torch.float16), ("4", torch.float32), ("16", torch.bfloat16), ("16", torch.float16), ("16", torch.float32)]
# nodes, heads, K/V heads, width, page, lengths: tiles of 8, 16, 32, 64, 128 and 256 rows; one block of keys, several, sequences that are cut
SHAPES = [(1, 8, 8, 64, 16, [0, 9, 63]), (1, 8, 2, 128, 16, [300, 70]), (1, 2, 2, 64, 16, [5000]), (1, 4, 1, 128, 64, [4000, 3]), (12, 2, 2, 64, 16, [20, 300]), (26, 2, 2, 128, 16, [130, 1900]), (51, 2, 2, 64, 16, [10, 300]),
          (51, 2, 2, 64, 32, [3000]), (40, 4, 2, 128, 16, [7, 400]), (60, 4, 2, 64, 16, [20, 500]), (64, 8, 2, 128, 64, [30, 700]), (64, 4, 1, 64, 64, [3000]), (40, 3, 1, 128, 32, [2500])]
CASES = [(*k, s) for k in KINDS for s in SHAPES] + [(*k, (12, 2, 2, 64, 4, [20, 300])) for k in KINDS if k[0] == "16"]


def filled(kind, dtype, k, v, count, T, page):
    """A cache of tokens k, v [B, S, heads, width], count[b] of them in sequence b and the last T of those a block; and the values that it holds, in 64 bits."""
    from paper_2203_16487_b200 import fp4, tree
    B, S, H, D = k.shape
    per = -(-S // page)
    kw = dict(n_pages=B * per, n_seqs=B, max_pages=per, page_tokens=page)
    cache = fp4.Fp4Cache(1, H, D, **kw) if kind == "4" else tree.PagedCache(1, H, D, dtype=dtype, **kw)
    seqs = torch.arange(B, device="cuda").int()
    cache.reserve(seqs, S)
    cache.append(seqs, k, v, layer=0, count=ints(count))
    held = cache.read(seqs, S, layer=0, dtype=torch.float32) if kind == "4" else (k, v)
    cache.length.copy_(torch.tensor([n - T for n in count]))
    return cache, seqs, *(x.double() for x in held)


def chain(T):
    """Words of a mask in which every node sees itself and the ones ahead of it, and [T, T] of the same."""
    return R.pack([[set(range(t + 1)) for t in range(T)]], T).cuda(), torch.ones(T, T, dtype=torch.bool, device="cuda").tril()


def exact(q, k, v, count, scale, tree):
    """In 64 bits: the answer, the sum of p |v|, and of each query's scores (times log2 e) the best one's lead and the largest sum of |q k|."""
    B, T, H, D = q.shape
    g = H // k.shape[2]
    want, mag = (torch.zeros(B, T, H, D, dtype=torch.float64, device="cuda") for _ in "wm")
    lead, size = (torch.zeros(B, T, H, dtype=torch.float64, device="cuda") for _ in "ls")
    for b, n in enumerate(count):
        see = torch.cat((torch.ones(T, n - T, dtype=torch.bool, device="cuda"), tree), 1)
        for h in range(H):
            kk, vv, qq = k[b, :n, h // g], v[b, :n, h // g], q[b, :, h].double()
            s = (qq @ kk.T * scale).masked_fill(~see, -math.inf)
            p = torch.softmax(s, 1)
            want[b, :, h], mag[b, :, h] = p @ vv, p @ vv.abs()
            best = torch.nn.functional.pad(s, (0, 1), value=-math.inf).topk(2, 1).values
            lead[b, :, h] = (best[:, 0] - best[:, 1]) * math.log2(math.e)
            size[b, :, h] = (qq.abs() @ kk.abs().T).amax(1) * scale * math.log2(math.e)
    return want, mag, lead, size


UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def check_winners(got, want, lead, size, dtype):
    """Scores are sums of at most 128 products in fp32, off by less than 2^-16 of the sum of their sizes with the sum's roundings (an additional one of a product with the scale, and 2^-22 of queries in two
    parts, among them), so two differ by at most 2^-15 more than they should; asked for is twice that and 64, behind which nobody weighs anything.  The winner's weight is divided by itself (sums in fp32, 2^-20
    with the merges), and the answer rounded once."""
    clear = lead > 2.0 ** -14 * size + 64
    assert clear.double().mean() > 0.7
    off = (got.double() - want).abs() - (UNIT[dtype] + 2.0 ** -20) * want.abs() - 1e-15
    wrong = ~(off.amax(-1) <= 0) & clear
    assert not wrong.any(), (int(wrong.sum()), int(clear.sum()), int(got.isnan().any(-1).sum()))


@pytest.mark.parametrize("kind,dtype,shape", CASES)
def test_the_winner_of_large_scores(kind, dtype, shape):
    """Scores of 2^15 to 2^39 (times log2 e), the largest of them positive, negative or either."""
    from paper_2203_16487_b200 import tree
    T, H, Hkv, D, page, lens = shape
    g = torch.Generator(device="cuda").manual_seed(T + D)
    B, S, count = len(lens), max(lens) + T, [n + T for n in lens]
    k, v = (torch.randn(B, S, Hkv, D, generator=g, device="cuda").to(dtype) for _ in "kv")
    k[..., 0] = 6
    cache, seqs, kk, vv = filled(kind, dtype, k, v, count, T, page)
    words, see = chain(T)
    for e in (12, 18, 20, 22, 24, 30, 36):
        for sign in (1, -1, 0):
            inside = min(e, 10) if dtype == torch.float16 else e // 2
            q = torch.randn(B, T, H, D, generator=g, device="cuda")
            if sign:
                q[..., 0] = 8 * sign
            q = (q * 2.0 ** inside).to(dtype)
            scale = D ** -0.5 * 2.0 ** (e - inside)
            got = tree.attention(q, cache, 0, seqs, words, scale=scale)
            want, _, lead, size = exact(q, kk, vv, count, scale, see)
            check_winners(got, want, lead, size, dtype)
    cache.check()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", SHAPES)
def test_queries_up_to_the_largest_number(dtype, shape):
    """Rows whose largest number is the type's, over 4 bits: finite, so they are scaled like any other."""
    from paper_2203_16487_b200 import tree
    T, H, Hkv, D, page, lens = shape
    g = torch.Generator(device="cuda").manual_seed(T + D)
    B, S, count = len(lens), max(lens) + T, [n + T for n in lens]
    k, v = (torch.randn(B, S, Hkv, D, generator=g, device="cuda").to(dtype) for _ in "kv")
    cache, seqs, kk, vv = filled("4", dtype, k, v, count, T, page)
    words, see = chain(T)
    q = torch.randn(B, T, H, D, generator=g, device="cuda").double()
    q = (q / q.abs().amax(-1, keepdim=True) * torch.finfo(dtype).max).to(dtype)
    assert q.isfinite().all()
    for scale in (2.0 ** -121, 2.0 ** -100):
        got = tree.attention(q, cache, 0, seqs, words, scale=scale)
        want, _, lead, size = exact(q, kk, vv, count, scale, see)
        if scale == 2.0 ** -121:                               # scores of some 2^9: winners are rarer
            assert got.isfinite().all()
        else:
            check_winners(got, want, lead, size, dtype)


@pytest.mark.parametrize("kind,dtype,shape", CASES)
def test_later_keys_ahead_by_what_rounding_hides(kind, dtype, shape):
    """Scores that are exact in fp32, 1.125 * 2^27 and, of some keys, 16 and of later ones 32 (of log2) more.  One unit in the last place is 16 there: a maximum's next neighbour weighs 2^16 times as much."""
    from paper_2203_16487_b200 import tree
    T, H, Hkv, D, page, _ = shape
    g = torch.Generator(device="cuda").manual_seed(T + D)
    n = 600
    k = torch.zeros(1, n + T, Hkv, D, device="cuda")
    k[..., :6], k[..., 17] = 768, 6                            # (codes of 6, and scales of 128 and 1)
    k[0, [5, 70, 130, 131], :, 16] = 1
    k[0, [300, 333, 450, 560], :, 16] = 2
    v = torch.randn(1, n + T, Hkv, D, generator=g, device="cuda")
    cache, seqs, kk, vv = filled(kind, dtype, k.to(dtype), v.to(dtype), [n + T], T, page)
    assert torch.equal(kk, k.double())
    q = torch.zeros(1, T, H, D, device="cuda", dtype=dtype)
    q[..., :6], q[..., 16] = 2.0 ** 15, 16
    log2e = np.float32(1.4426950408889634)
    ln2 = np.float32(math.log(2))
    scale = next(float(s) for s in (ln2, np.nextafter(ln2, np.float32(1)), np.nextafter(ln2, np.float32(0))) if s * log2e == 1)
    words, see = chain(T)
    got = tree.attention(q, cache, 0, seqs, words, scale=scale)
    want, mag, _, size = exact(q, kk, vv, [n + T], math.log(2), see)
    assert float(size.max()) < 2.0 ** 28 and float(size.min()) >= 2.0 ** 27
    # probabilities rounded to 16 bits (bf16: 2^-8 of themselves, half of that in the sum), the answer once
    p = 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8 if kind == "16" and dtype == torch.bfloat16 else 2.0 ** -11
    off = (got.double() - want).abs() - (2 * p + 1e-5) * mag - UNIT[dtype] * want.abs()
    assert not got.isnan().any() and (off <= 0).all(), (float(off.max()), int(got.isnan().sum()))
    cache.check()
