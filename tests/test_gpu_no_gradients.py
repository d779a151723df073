"""Operators without a gradient say so for every argument that could ask for one."""
import pytest
import torch

from tests.test_gpu_tree import ints

pytestmark = pytest.mark.gpu


def test_values_read_from_tokens_that_require_a_gradient():
    from paper_2203_16487_b200 import fp4
    for which in "kv":
        cache = fp4.Fp4Cache(1, 2, 64, n_pages=2, n_seqs=2, max_pages=1, page_tokens=16)
        seqs = ints([0])
        cache.reserve(seqs, 3)
        k, v = (torch.randn(1, 3, 2, 64, device="cuda") for _ in "kv")
        cache.append(seqs, k, v, layer=0)
        assert not any(x.requires_grad for x in cache.read(seqs, 3, layer=0))
        cache.append(seqs, *(x.requires_grad_() if name == which else x for name, x in zip("kv", (k, v))), layer=0)
        for i in range(2):
            with pytest.raises(RuntimeError, match="no gradient"):
                cache.read(seqs, 3, layer=0, dtype=torch.float32)[i].sum().backward()
        with torch.no_grad():
            a, b = cache.read(seqs, 3, layer=0)
        assert not a.requires_grad and not b.requires_grad


def test_selection_by_anything_that_requires_a_gradient():
    from paper_2203_16487_b200 import beam
    make = lambda *s: torch.randn(*s, device="cuda")  # noqa: E731
    for asked in ((0,), (1,), (2,), (0, 1), (0, 1, 2), (1, 2)):
        args = [make(2, 3, 50), make(2, 3), make(2, 3).abs() + 1]
        for i in asked:
            args[i].requires_grad_()
        for i in asked:
            out = beam.select(args[0], args[1], 4, norm=args[2])
            assert out[0].requires_grad and not out[1].requires_grad
            with pytest.raises(RuntimeError, match="no gradient"):
                torch.autograd.grad(out[0].sum(), args[i])
        with torch.no_grad():
            assert not beam.select(args[0], args[1], 4, norm=args[2])[0].requires_grad


def test_sampling_by_logits_and_temperature():
    from paper_2203_16487_b200 import tree
    for asked in ((0,), (1,), (0, 1)):
        logits, temperature = torch.randn(2, 50, device="cuda"), torch.ones(2, device="cuda")
        args = [logits, temperature]
        for i in asked:
            args[i].requires_grad_()
        for i in asked:
            logprob = tree.sample(args[0], torch.rand(2, device="cuda"), args[1])[1]
            with pytest.raises(RuntimeError, match="no gradient"):
                torch.autograd.grad(logprob.sum(), args[i])
