"""Gradients of attention (include/rb_block.h) on the GPU around a key that is infinite and has no weight: who neither sees it nor is seen by it has the gradients it would have
without it."""
import pytest
import torch

import block_reference as ref
import paper_2406_03285_amd as rb
from test_block_attention import INF, documents, tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 72, 128])
@pytest.mark.parametrize("offsets,prefix", [([0, 100], None), ([0, 300], None), ([0, 20, 320], [0, 7])])
def test_an_infinite_key_without_weight(offsets, prefix, dim):
    """Scores of -inf: the weight is 0, out and lse are what they are without the key.  The positions before it are seen by queries that see it, too, and their gradients need
    these queries' sum of p dp."""
    tokens, at, heads = offsets[-1], 60, 2
    q, k, v, d = tensors(tokens, heads, 1, dim, seed=31, layout="own")
    q[:, :, 3] = q[:, :, 3].abs() + 0.5
    k[at, 0, 3] = -INF
    docs = documents(offsets, None, prefix)
    a = rb.DocumentAttention(heads, dim, 1, max_tokens=tokens)
    got = a.forward(q, k, v, docs)
    _, grad_k, grad_v = a.grad(q, k, v, docs, got.out, got.lse, d)
    mask, scale = ref.seen(tokens, offsets, None, prefix), dim ** -0.5
    saw = mask[:, at].clone()
    mask[:, at] = False
    q64, k64, v64, d64 = (ref.to64(x) for x in (q, k, v, d))
    k64[at] = 0.0                                          # (nobody sees it)
    out, lse, off_out, off_lse = ref.attend(q64, k64, v64, scale, 0.0, None, mask)
    have_out, have_lse = ref.to64(got.out), ref.to64(got.lse)
    assert ((have_out - out).abs() <= off_out).all() and ((have_lse - lse).abs() <= off_lse).all()
    want, off = ref.attend_grad(q64, k64, v64, have_out, have_lse, d64, scale, 0.0, None, mask)
    # of the queries that see it the sum of p dp is grad_out . out of an out that was rounded: half a step of each of its terms, which goes into ds with the weight
    s, _, _ = ref.scores(q64, ref.spread(k64, heads), scale, 0.0, None, mask)
    p = torch.where(mask, (s - have_lse[:, :, None]).exp(), 0.0)
    rounding = ((d64 * have_out).abs().sum(2) * ref.BF16_HALF + (d64.abs() * off_out).sum(2)).t()[:, :, None] * saw[None, :, None]
    more = torch.einsum("hij,ihd->jhd", p * rounding, q64.abs()).unflatten(1, (1, heads)).sum(2) * scale * (1 + 4 * ref.BF16_HALF)
    others = list(range(at))
    assert ((ref.to64(grad_k) - want[1]).abs() <= off[1] + more)[others].all(), ((ref.to64(grad_k) - want[1]).abs() / (off[1] + more))[others].max()
    assert ((ref.to64(grad_v) - want[2]).abs() <= off[2])[others].all()
    # ... as if the key were finite and very negative, but for that rounding
    k2 = k.clone()
    k2[at, 0, 3] = -1e30
    same = a.forward(q, k2, v, docs)
    assert torch.equal(same.out, got.out) and torch.equal(same.lse, got.lse)
    assert torch.equal(a.grad(q, k2, v, docs, got.out, got.lse, d)[2][others], grad_v[others])
