"""The training step with everything in it (examples/rehearse_classes.py), and one of its iterations against plain torch."""
import importlib.util
import os

import pytest
import torch

import paper_2406_03285_amd as rb

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("rehearse_classes", os.path.join(ROOT, "examples", "rehearse_classes.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_rehearsal_keeps_what_was_learnt(example):
    with_it, losses = example.train(True, steps=40)
    without, _ = example.train(False, steps=40)
    assert torch.isfinite(losses).all()
    first, last = slice(0, 40), slice(-10, None)
    assert losses[last].mean() < losses[first][:5].mean()
    assert with_it[0] > 0.6 and with_it[0] > without[0] + 0.2, (with_it, without)      # the first task, three tasks later
    again, _ = example.train(True, steps=40)
    assert again == with_it


def test_gradients_reach_the_weights(example):
    """Weights' gradients of the example's loss against the same loss by log_softmax in binary64."""
    torch.manual_seed(0)
    model = example.Model("cuda")
    x = torch.randn((50, example.FEATURES), device="cuda")
    tokens = torch.randint(-1, example.CLASSES, (50, 1 + example.ALTERNATIVES), device="cuda")
    p = torch.rand((50, 1 + example.ALTERNATIVES), device="cuda")
    scorer = rb.TokenScorer(example.CLASSES, given=1 + example.ALTERNATIVES, top=3)
    s = scorer(model(x), tokens)
    ((p * s.logp).sum() - 0.1 * s.entropy.sum()).backward()
    got = [w.grad.double() for w in (model.hidden, model.classes)]
    w1, w2 = (w.detach().double().requires_grad_() for w in (model.hidden, model.classes))
    logp = torch.log_softmax(torch.relu(x.double() @ w1.t()) @ w2.t(), 1)
    loss = (p.double() * torch.where(tokens >= 0, logp.gather(1, tokens.clamp(min=0)), 0.0)).sum() + 0.1 * (logp.exp() * logp).sum()
    for g, want in zip(got, torch.autograd.grad(loss, (w1, w2))):
        # the products in binary32: sums of at most 256 terms, 2^-24 each, and their inputs' as much again
        assert (g - want).norm() <= 2.0 ** -15 * want.norm()


def test_no_rows_and_changed_weights():
    scorer = rb.TokenScorer(9, given=2, top=2)
    z, t = torch.zeros((0, 9), device="cuda"), torch.zeros((0, 2), dtype=torch.int64, device="cuda")
    assert scorer.score(z, t).top_ids.shape == (0, 2)
    z.requires_grad_()
    scorer(z, t).logp.sum().backward()
    assert z.grad.shape == (0, 9)
    w = torch.randn((8, 8), device="cuda", requires_grad=True)
    y = (w * w).sum()                                   # saves w
    rb.Orthogonalizer(8, 8).step(w.detach(), torch.randn((8, 8), device="cuda"), torch.zeros((8, 8), device="cuda"), lr=0.1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
