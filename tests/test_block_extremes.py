"""Scales and caps at the ends of binary32's range (include/rb_block.h): refused where what the kernels multiply by would leave it, right up to there."""
import pytest
import torch

import paper_2406_03285_amd as rb


@pytest.mark.parametrize("scale,cap", [(3e38, 0.0), (2.4e38, 1e38), (1.0, 3e38), (1.0, 1e-39), (1.0, 8e-39), (1e30, 1e-10), (1.0, 1e38), (1e-10, 1e30), (1e-45, 1.0)])
def test_scales_and_caps_whose_quotients_leave_the_range_are_refused(scale, cap):
    assert rb.rb_attention_create(2, 1, 64, 100, 1, scale, cap) == (rb.RB_EINVAL, None)


@pytest.mark.parametrize("scale,cap", [(2e38, 0.0), (1e-40, 0.0), (2e38, 2e38), (1.0, 1e-38), (1.0, 1e-37), (1.0, 8e37), (1e-8, 1e29), (1e30, 1e-7)])
def test_scales_and_caps_up_to_there_are_taken(scale, cap):
    rc, a = rb.rb_attention_create(2, 1, 64, 100, 1, scale, cap)
    assert rc == rb.RB_OK and rb.rb_attention_destroy(a) == rb.RB_OK


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,count", [(40, 40), (300, 1)])
def test_caps_at_the_ends_of_the_range(tokens, count):
    """A cap that no score comes near leaves the scores as they are; one that is next to nothing makes them all next to nothing."""
    g = torch.Generator("cuda").manual_seed(1)
    q, k, v, d = (torch.randn((tokens, 2, 64), generator=g, device="cuda").to(torch.bfloat16) for _ in range(4))
    docs = rb.Documents(torch.arange(count + 1, device="cuda") * (tokens // count))

    def results(cap, scale):
        a = rb.DocumentAttention(2, 64, max_tokens=tokens, cap=cap, scale=scale)
        o = a.forward(q, k, v, docs)
        return [o.lse.double(), o.out.double(), *(x.double() for x in a.grad(q, k, v, docs, o.out, o.lse, d))]
    plain, wide = results(0.0, 1.0), results(8e37, 1.0)
    # scores of up to some 40 are 12 half steps off at most, which is 3e-5 of a weight; out and gradients are rounded to bfloat16 on either side of a boundary
    assert (plain[0] - wide[0]).abs().max() < 1e-4
    for x, y in zip(plain[1:], wide[1:]):
        assert (x - y).norm() <= 2.0 ** -8 * x.norm() + 1e-30
    flat, small = results(0.0, 1e-30), results(1e-30, 1.0)
    assert (flat[0] - small[0]).abs().max() < 1e-5 and (flat[1] - small[1]).norm() <= 2.0 ** -8 * flat[1].norm()
    assert all(torch.isfinite(x).all() for x in small)
