"""Beam search's selection against a plain implementation in 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests import beam_reference as F
from tests import fp4_reference
from tests.test_gpu_tree import ints

pytestmark = pytest.mark.gpu
ALL = [torch.float32, torch.bfloat16, torch.float16]


def run(logits, scores, n, finished=None, end_token=0, norm=None):
    """Checks a call; returns (scores, parents, tokens).  Beams and tokens have to be those of the reference, however near two ranks are, unless they are nearer than 64 bits tell (1e-12).
    Scores: the sum of e^x in fp32 is off by less than 2^-20 of itself (products with log2 e and exponentials by some 2^-22 each, sums of at most 64 terms a thread in four parts), the result
    is rounded to fp32."""
    from paper_2203_16487_b200 import beam
    got = beam.select(logits, scores, n, finished=finished, end_token=end_token, norm=norm)
    assert [x.dtype for x in got] == [torch.float32, torch.int32, torch.int32] and all(x.shape == (logits.shape[0], n) for x in got)
    s, parent, token = (x.cpu().numpy() for x in got)
    l, sc = logits.float().cpu().numpy(), scores.cpu().numpy()
    fin, nm = (None if x is None else x.cpu().numpy() for x in (finished, norm))
    for b in range(len(l)):
        want, near = F.select(l[b], sc[b], n, None if fin is None else fin[b], end_token, None if nm is None else nm[b])
        if near > 1e-12 or near == 0:
            assert parent[b].tolist() == [w[1] for w in want] and token[b].tolist() == [w[2] for w in want], (b, near)
        for x, w in zip(s[b], want):
            # (beyond fp32's largest number the nearest one is an infinity)
            assert x == w[0] or abs(x - w[0]) <= 2.0 ** -20 + 2.0 ** -24 * abs(w[0]) or x == (-math.inf if w[0] < -2.0 ** 128 else w[0]), (b, x, w)
    return got


def rows(B, K, V, dtype, seed, spread=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(B, K, V, generator=g, device="cuda") * spread).to(dtype), -30 * torch.rand(B, 1, generator=g, device="cuda") - 3 * torch.rand(B, K, generator=g, device="cuda")


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("B,K,V,n", [(1, 1, 1, 1), (1, 4, 32768, 8), (3, 5, 50265, 5), (2, 12, 1001, 25), (40, 8, 2048, 16), (1, 64, 333, 64), (2, 1, 7, 12), (1, 2, 131071, 3), (300, 1, 100, 2), (1, 3, 4097, 64),
                                     (1, 2, 600000, 9), (64, 8, 9000, 16)])
def test_select(dtype, B, K, V, n):
    for spread in (0.3, 4.0):
        run(*rows(B, K, V, dtype, B + V, spread), n)


@pytest.mark.parametrize("dtype", ALL)
def test_select_finished_dead_normed(dtype):
    B, K, V, n = 6, 6, 3001, 9
    logits, scores = rows(B, K, V, dtype, 5)
    finished = torch.zeros(B, K, dtype=torch.bool, device="cuda")
    finished[0] = True
    finished[1, ::2] = True
    scores[2] = -math.inf
    scores[3, 1:] = -math.inf                                  # the first step: one beam
    scores[4, 0], finished[4, 0] = math.nan, True
    logits[1, 0], logits[2, 0] = math.nan, math.nan            # what does not count is not looked at
    norm = 1 / (1 + torch.rand(B, K, device="cuda") * 3)
    out = run(logits, scores, n, finished, 7, norm)
    assert out[1][2].tolist() == [-1] * n and out[0][2].tolist() == [-math.inf] * n
    assert sorted(out[1][0].tolist()) == [-1, -1, -1] + list(range(K)) and set(out[2][0].tolist()) == {-1, 7}
    run(logits, scores, n, None, 0, norm)
    run(logits, scores, n, finished, V - 1, None)
    run(logits, scores, 1, finished, 0, None)


@pytest.mark.parametrize("dtype", ALL)
def test_select_ties_infinities_nan(dtype):
    """Equal logits, equal beams, rows of nothing, infinite logits, NaN among the largest; runs of equal values longer than any list."""
    V = 5000
    logits, scores = rows(10, 4, V, dtype, 9)
    logits[0] = 1.5                                            # everything alike, in every beam
    scores[0] = -2.0
    logits[1, :, 100:] = logits[1, :, 50:51]                   # thousands of equal ones, small ones among them
    logits[2] = logits[2, 0]                                   # the same row in all beams
    scores[2, :2] = scores[2, 0]
    logits[3, 0], logits[3, 1] = -math.inf, math.nan
    logits[4, 2, 17], logits[4, 2, 4000] = math.inf, math.inf
    logits[5, :, ::2] = math.nan
    logits[6, 1, 3:] = -math.inf
    logits[7, 0, :] = -math.inf
    logits[7, 0, 4999] = 3.0
    logits[8] = (torch.randint(0, 3, (4, V), device="cuda") * 4.0).to(dtype)
    logits[9] = torch.where(logits[9] == 0, 0.0, torch.where(torch.arange(V, device="cuda") % 2 == 0, 0.0, -0.0)).to(dtype)      # zeros of either sign are equal
    for n in (1, 8, 63, 64):
        run(logits, scores, n)
    run(logits[:, :, :40], scores, 64)                         # rows that begin anywhere, evenly spaced


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("V", [90, 32768, 50265])
def test_select_masks_of_the_lowest_value_and_logits_of_any_size(dtype, V):
    """Tokens that a mask has set to the type's lowest value: some, whole stretches, whole rows; logits around numbers of every size, whose sums' shares are whole or gone."""
    low, high = torch.finfo(dtype).min, torch.finfo(dtype).max
    logits, scores = rows(12, 3, V, dtype, V)
    logits[0, :, ::3] = low
    logits[1, :, 40:] = low
    logits[2, :, :-5] = low
    logits[3] = low
    logits[4, 0], logits[4, 1, 7:] = low, -math.inf
    logits[5], logits[5, :, 11], logits[5, 1, 50:] = low, high, math.nan
    logits[6], logits[6, 1] = high, 0.0
    for b, size in zip(range(7, 12), (6e4, 65536.0, 1e6, 1e9, 1e30)):
        logits[b] = (logits[b].float() + (size if b % 2 else -size)).to(dtype).clamp(low, high)
    for n in (1, 7):
        run(logits, scores, n)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("gap", [0.0, 1e-9, 1e-7, 3e-7, 1e-6, 1e-5])
def test_select_is_that_of_exact_sums(dtype, gap):
    """Two beams of unlike rows whose best continuations differ by less than fp32 sums can tell, either way round."""
    B, K, V = 24, 3, 20000
    logits, scores = rows(B, K, V, dtype, 3)
    base = logits.double().cpu().numpy()
    for b in range(B):
        first = [F.log_softmax(base[b, k])[1].max() for k in range(2)]
        want = np.float64(-3.0) + first[0] - first[1] + (gap if b % 2 else -gap)       # beam 1's score that brings its best one there
        scores[b, 0], scores[b, 1], scores[b, 2] = -3.0, float(want), -9.0
        # fp32 cannot hold that score; the nearest ones are some 1e-7 apart, so the gap is what the reference finds
    run(logits, scores, 6)
    flat = torch.tensor([[-3.0, -3.0, -9.0]], device="cuda").expand(B, -1).contiguous()
    norm = torch.ones(B, K, device="cuda")
    norm[:, 1] = (flat.new_tensor([(-3.0 + F.log_softmax(base[b, 0])[1].max()) / (-3.0 + F.log_softmax(base[b, 1])[1].max()) for b in range(B)]) * (1 + gap)).float()
    run(logits, flat, 6, norm=norm)


def test_select_strides_refusals_and_gradients():
    from paper_2203_16487_b200 import beam, binding
    logits, scores = rows(3, 4, 515, torch.bfloat16, 1)
    wide = torch.full((3, 4, 700), 50.0, device="cuda", dtype=torch.bfloat16)
    for at in range(0, 9):                                     # rows that begin at every place of a vector
        wide[..., at:at + 515] = logits
        run(wide[..., at:at + 515], scores, 8)                 # (which thread adds up what goes by where a row begins, so scores may differ by the bound that is checked there)
    run(wide[1:2, ::2, 8:523], scores[1:2, ::2].contiguous(), 4)
    assert all(x.shape == (0, 4) for x in beam.select(logits[:0], scores[:0], 4))
    for bad in (lambda: beam.select(logits[0], scores[0], 4), lambda: beam.select(logits.double(), scores, 4), lambda: beam.select(logits, scores.double(), 4), lambda: beam.select(logits, scores[:, :2], 4),
                lambda: beam.select(logits, scores, 4, finished=torch.zeros(3, 4, device="cuda")), lambda: beam.select(logits, scores, 4, norm=scores[:2]), lambda: beam.select(logits.transpose(0, 1), scores.t().contiguous(), 4),
                lambda: beam.select(logits.cpu(), scores.cpu(), 4), lambda: beam.select(logits.transpose(1, 2), scores, 4)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: beam.select(logits, scores, 0), lambda: beam.select(logits, scores, 65), lambda: beam.select(torch.zeros(1, 65, 3, device="cuda"), torch.zeros(1, 65, device="cuda"), 1)):
        with pytest.raises(binding.SpecDecError):
            bad()
    with pytest.raises(RuntimeError, match="no gradient"):
        beam.select(logits, scores.clone().requires_grad_(), 4)[0].sum().backward()


def test_select_captured_and_replayed_with_others_running():
    """Replays on new logits, another call between them on another stream: workspaces are nobody else's."""
    from paper_2203_16487_b200 import beam
    logits, scores = rows(4, 5, 20001, torch.float32, 2)
    other, more = rows(9, 8, 32768, torch.bfloat16, 3)
    want = [x.clone() for x in beam.select(other, more, 16)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        beam.select(logits, scores, 10)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = beam.select(logits, scores, 10)
    for i in range(5):
        logits.normal_(generator=torch.Generator(device="cuda").manual_seed(i))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        now = beam.select(other, more, 16)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(now, want))
        ref = beam.select(logits, scores, 10)
        assert all(torch.equal(x, y) for x, y in zip(out, ref))


@pytest.mark.parametrize("kind", ["16", "4"])
def test_beams_select_and_reorder_together(kind):
    """What a sequence's cache holds after some steps is what its beam's ancestors have written."""
    from paper_2203_16487_b200 import beam, fp4, tree
    B, K, H, D, page, V, steps = 3, 4, 2, 64, 16, 50, 40
    n = B * K
    kw = dict(n_pages=n * 3 + 2, n_seqs=n, max_pages=3, page_tokens=page)
    cache = fp4.Fp4Cache(1, H, D, **kw) if kind == "4" else tree.PagedCache(1, H, D, dtype=torch.float16, **kw)
    seqs = torch.arange(n, device="cuda").int().view(B, K)
    flat = seqs.view(-1)
    scores = torch.full((B, K), -math.inf, device="cuda")
    scores[:, 0] = 0
    held = [[] for _ in range(n)]
    g = torch.Generator(device="cuda").manual_seed(1)
    for _ in range(steps):
        k, v = (torch.randn(1, n, 1, H, D, device="cuda", generator=g).half() for _ in "kv")
        cache.reserve(flat, 1)
        cache.append(flat, k, v)
        cache.compact(flat, ints([[0]] * n), ints([1] * n))
        logits = torch.randn(B, K, V, device="cuda", generator=g) * 2
        scores, parent, token = beam.select(logits, scores, K)
        cache.reorder(seqs, parent)
        held = [h + [(k[0, i, 0].cpu(), v[0, i, 0].cpu())] for i, h in enumerate(held)]
        held = [held[b * K + p] for b in range(B) for p in parent[b].tolist()]
    cache.check()
    assert cache.length.tolist() == [steps] * n
    assert sum(x > 0 for x in cache.refs.tolist()) == len({p for row in cache.table.tolist() for p in row if p >= 0})
    table = cache.table.tolist()
    for i in range(n):
        want = torch.stack([torch.stack(x) for x in held[i]], 1)                     # [2, steps, H, D]
        if kind == "4":
            got = torch.cat(cache.read(ints([i]), steps, layer=0, start=ints([0]), dtype=torch.float16)).cpu().double()
            want = fp4_reference.values(*fp4_reference.quantise(want))
            assert torch.equal(got, want)
        else:
            for t in range(steps):
                assert torch.equal(cache.kv[0, :, table[i][t // page], t % page].cpu(), want[:, t])
