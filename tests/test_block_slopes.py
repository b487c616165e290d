"""Scores that rise with distance (include/rb_block.h: slopes below 0) on the GPU, against a plain statement in 64 bits, in every form of the scores."""
import pytest
import torch

import block_reference as ref
import paper_2406_03285_amd as rb
import test_block_attention as plain

pytestmark = pytest.mark.gpu


def rising(heads):
    return torch.tensor([-0.5 * 0.4 ** h for h in range(heads)], device="cuda")


def of_either_sign(heads):
    return torch.tensor([(-1.0) ** h * 0.7 * 0.5 ** h for h in range(heads)], device="cuda")


@pytest.mark.parametrize("dim", [64, 72, 128])
@pytest.mark.parametrize("cap", [0.0, 3.0, 20.0, 32.0, 50.0])
@pytest.mark.parametrize("slopes", [rising, of_either_sign])
@pytest.mark.parametrize("offsets,causal,prefixes", [([0, 431], True, None), ([0, 420], False, None), ([0, 270, 271, 431], True, [70, 5, 400]), ([3 * i for i in range(144)], True, None)])
def test_scores_that_rise_with_distance(monkeypatch, offsets, causal, prefixes, slopes, cap, dim):
    """Far positions have the largest weights, by e^200 and more: the sums are within binary32's range only behind a maximum.  The last documents are short ones."""
    monkeypatch.setattr(plain, "slopes_of", slopes)
    plain.check(*plain.tensors(431, 4, 2, dim, seed=21), offsets, None, prefixes, causal, cap, True)


@pytest.mark.parametrize("cap", [0.0, 20.0, 50.0])
def test_one_weight_of_many(cap):
    """A slope of -40: the first position has all the weight of every position behind it, so out is its v and lse its score."""
    tokens, dim = 700, 64
    q, k, v, _ = plain.tensors(tokens, 2, 2, dim, seed=22)
    a = rb.DocumentAttention(2, dim, max_tokens=tokens, cap=cap)
    got = a.forward(q, k, v, plain.documents([0, tokens]), slopes=torch.full((2,), -40.0, device="cuda"))
    at = torch.arange(50, tokens)
    s = torch.einsum("ihd,hd->hi", ref.to64(q), ref.to64(k)[0]) * dim ** -0.5
    want = (cap * torch.tanh(s / cap) if cap else s) + 40.0 * torch.arange(tokens)
    # the others' weights are e^-40 a position, times what scores differ by; the score is off by 68 half steps of its terms (of size 9 in the mean), a number of
    # the sum's size is rounded some times
    assert ((ref.to64(got.lse) - want).abs() <= 1e-4 + 8 * ref.F32_HALF * want.abs())[:, at].all()
    assert torch.isfinite(got.out.float()).all() and torch.isfinite(got.lse).all()


@pytest.mark.parametrize("cap", [16.0, 64.0, 4096.0])
def test_capped_scores_are_exact_to_some_of_their_own_half_steps(cap):
    """Documents of one position, whose lse is the score: of any size beside the cap.  The product (of two numbers, with 1 and 2^-8) and its quotient by a power of two
    are exact; tanh is within eight half steps, log2 e times the cap and ln 2 are two of each a constant's and a product's."""
    tokens, dim = 30000, 8
    g = torch.Generator().manual_seed(3)
    x = torch.empty(tokens, dtype=torch.float64).uniform_(0.01, 0.6, generator=g)
    x[20000:] = torch.empty(10000, dtype=torch.float64).uniform_(0.1, 3.0, generator=g)
    x = x * (1 - 2 * (torch.arange(tokens) % 2)) * cap
    q, k = (torch.zeros((tokens, 1, dim), dtype=torch.bfloat16) for _ in range(2))
    q[:, 0, 0] = x.to(torch.bfloat16)
    q[:, 0, 1] = ((x - q[:, 0, 0].double()) * 256).to(torch.bfloat16)
    k[:, 0, 0], k[:, 0, 1] = 1.0, 2.0 ** -8
    a = rb.DocumentAttention(1, dim, max_tokens=tokens, scale=1.0, cap=cap)
    got = a.forward(q.cuda(), k.cuda(), k.cuda(), plain.documents(list(range(tokens + 1))))
    s = ref.to64(q[:, 0, 0]) + ref.to64(q[:, 0, 1]) / 256
    want = cap * torch.tanh(s / cap)
    d = (ref.to64(got.lse)[0] - want).abs() / want.abs()
    assert (d <= 12 * ref.F32_HALF).all(), float(d.max()) / ref.F32_HALF
