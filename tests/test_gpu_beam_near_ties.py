"""Beam search's selection where more than two beams lie within the errors of fp32 sums of one another, or hide behind a tie: the choice is still that of exact sums."""
import numpy as np
import pytest
import torch

from tests import beam_reference as F
from tests.test_gpu_beam import ALL, rows, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("B,K,V", [(16, 3, 50265), (40, 5, 5001), (3, 64, 3333), (2, 12, 131071)])
def test_alike_beams_whose_rows_begin_anywhere(dtype, B, K, V):
    """Rows of equal logits, which begin at other places of a vector and so are added up in another order: of ranks alike it is the lowest beam."""
    logits, scores = rows(B, K, V, dtype, K)
    logits[:] = logits[:, :1].clone()
    scores[:] = scores[:, :1].clone()
    for n in (1, 2, K - 1):
        out = run(logits, scores, n)
        top = (logits[:, 0] == logits[:, 0].amax(-1, keepdim=True)).sum(-1)
        if n == 1:
            assert (out[1] == 0).all()
        assert (out[1][:, 0] == 0).all() and (top >= 1).all()


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("copies", [2, 3, 7])
def test_alike_beams_behind_equal_logits(dtype, copies):
    """A beam's best logit several times over, so that its entries fill the last place and those behind it."""
    B, K, V = 24, 4, 50265
    logits, scores = rows(B, K, V, dtype, copies)
    logits[:] = logits[:, :1].clone()
    scores[:] = scores[:, :1].clone()
    at = torch.stack([torch.randperm(V, generator=torch.Generator().manual_seed(b))[:copies] for b in range(B)]).cuda()
    logits.scatter_(2, at[:, None].expand(B, K, copies), 12.0)
    for n in (1, copies - 1, copies, copies + 1, 2 * copies):
        if n:
            out = run(logits, scores, n)
            assert (out[1][:, :min(n, copies)] == 0).all()


@pytest.mark.parametrize("dtype", ALL)
def test_alike_beams_of_thousands_of_equal_logits(dtype):
    """More entries of one rank than any list holds."""
    B, K, V = 6, 8, 20001
    logits, scores = rows(B, K, V, dtype, 1)
    logits[..., ::3] = 9.0
    logits[:] = logits[:, :1].clone()
    scores[:] = scores[:, :1].clone()
    for n in (1, 17, 64):
        out = run(logits, scores, n)                           # (some sentences have a larger logit or two ahead of them, which is then every beam's)
        few = (logits[:, 0] > 9).sum(-1) == 0
        assert (out[1][few] == 0).all() and (out[2][few] == 3 * torch.arange(n, device="cuda")).all()


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("copies", [1, 2, 4])
@pytest.mark.parametrize("normed", [False, True])
def test_several_unlike_beams_nearly_alike(dtype, copies, normed):
    """Six beams whose best continuations lie within what an fp32 score can be set to, some of them several times over, in any order."""
    B, K, V = 16, 6, 20001
    logits, scores = rows(B, K, V, dtype, 7 + copies)
    at = torch.stack([torch.randperm(V, generator=torch.Generator().manual_seed(b))[:copies] for b in range(B * K)]).view(B, K, copies).cuda()
    logits.scatter_(2, at, 11.0)
    norm = torch.ones(B, K, device="cuda")
    base = logits.double().cpu().numpy()
    rng = np.random.default_rng(copies)
    for b in range(B):
        best = np.array([F.log_softmax(base[b, k])[1].max() for k in range(K)])
        f = rng.choice([0.25, 0.5, 1.0], K) if normed else np.ones(K)                   # (powers of two: ranks are as near as scores are)
        norm[b] = torch.from_numpy(f).float()
        want = -3.0 / f - best + rng.integers(-2, 3, K) * 2.0 ** -23
        scores[b] = torch.from_numpy(want).float()
    for n in (1, 2, copies, copies + 1, 3 * copies, 5):
        run(logits, scores, n, norm=norm if normed else None)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ended_beams_between_beams_nearly_alike(dtype):
    """A beam that has ended, whose rank is exact, at the last place; others within the sums' errors of it."""
    B, K, V = 24, 5, 20001
    logits, scores = rows(B, K, V, dtype, 3)
    base = logits.double().cpu().numpy()
    finished = torch.zeros(B, K, dtype=torch.bool, device="cuda")
    for b in range(B):
        finished[b, b % K] = True
        for k in range(K):
            scores[b, k] = -3.0 if k == b % K else float(np.float32(-3.0 - F.log_softmax(base[b, k])[1].max()))
    for n in (1, 2, 3, 5):
        run(logits, scores, n, finished, 7)
