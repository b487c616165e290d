"""The language model with everything in it (examples/rehearse_sequences.py): it runs, and its gradients against the same model in 64 bits."""
import importlib.util
import os

import pytest
import torch

import block_reference as ref

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("rehearse_sequences", os.path.join(ROOT, "examples", "rehearse_sequences.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_it_runs_and_repeats_itself(example):
    likelihoods, losses = example.train(True, steps=6)
    assert torch.isfinite(losses).all() and all(v == v for v in likelihoods)
    again, same = example.train(True, steps=6)
    assert again == likelihoods and torch.equal(losses, same)


def test_gradients_reach_the_weights(example):
    """Of the sum of given log probabilities, dropout among it.  On the way lie some 12 roundings to bfloat16 of a block (of two) and as many back: 64 half steps."""
    model = example.Model("cuda")
    rows = example.sequences(1, 2, 5, "cuda")
    rows[3, 0] = 0                                        # a document of no tokens
    tokens, documents, target = example.packed(rows)
    scorer = example.rb.TokenScorer(example.VOCAB)
    logp = scorer(model(tokens, documents, 9), target[:, None]).logp
    logp.sum().backward()
    p = {n: ref.to64(w).requires_grad_() for n, w in model.named_parameters()}
    n, heads, kv, dim = tokens.numel(), example.HEADS, example.KV_HEADS, model.dim
    mask = ref.seen(n, documents.offsets.tolist(), documents.lengths.tolist(), documents.prefixes.tolist())
    some = mask.any(1)
    x = p["tokens"][tokens.cpu()]
    for i in range(example.BLOCKS):
        b = {k: p[f"blocks.{i}.{k}"] for k in ("qkv", "back", "up", "down", "before", "between", "bias")}
        drop = [ref.kept(n, example.WIDTH, example.rb.Drop(model.dropout, 1000 * i + layer, 9)) for layer in range(2)]
        y = ref.norm(x, b["before"], None, 1e-5)[0]
        q, k, v = (z.unflatten(1, (c, dim)) for z, c in zip((y @ b["qkv"].t()).split([heads * dim, kv * dim, kv * dim], 1), (heads, kv, kv)))
        s = torch.einsum("ihd,jhd->hij", q, ref.spread(k, heads)) * dim ** -0.5
        w = torch.softmax(torch.where(mask | ~some[:, None], s, -float("inf")), 2) * some[:, None]
        a = torch.einsum("hij,jhd->ihd", w, ref.spread(v, heads)).flatten(1)
        total = x + (a @ b["back"].t()) * drop[0]
        y = ref.norm(total, b["between"], b["bias"], 1e-5)[0]
        x = total + (torch.relu(y @ b["up"].t()) @ b["down"].t()) * drop[1]
    want = torch.log_softmax(x @ p["tokens"].t(), 1)
    t = target.cpu()
    sum(want[i, t[i]] for i in range(n) if t[i] >= 0).backward()
    for name, w in model.named_parameters():
        d = (ref.to64(w.grad) - p[name].grad).norm() / p[name].grad.norm()
        assert d <= 64 * ref.BF16_HALF, (name, float(d))
