"""Attention of many documents and of long ones (include/rb_block.h) on the GPU against a plain statement in 64 bits, which is made on the GPU as well, some documents at a time."""
import random

import pytest
import torch

import block_reference as ref
import paper_2406_03285_amd as rb
from test_block_attention import INF, documents, slopes_of, tensors

pytestmark = pytest.mark.gpu


def seen(offsets, lengths, prefixes, causal):
    """[positions, positions] of documents that begin at 0, on the GPU."""
    n = offsets[-1]
    i = torch.arange(n, device="cuda")
    begins = torch.tensor(offsets[:-1], device="cuda")
    ends = torch.tensor([min(e, b + max(0, size)) for b, e, size in zip(offsets, offsets[1:], lengths or [n] * (len(offsets) - 1))], device="cuda")
    there = (i[None] >= begins[:, None]) & (i[None] < ends[:, None])                  # [documents, positions]
    where = torch.where(there.any(0), there.to(torch.int32).argmax(0), -1)
    mask = (where[:, None] == where[None]) & (where >= 0)[None]
    if causal:
        limit = begins + torch.tensor(prefixes or [0] * len(begins), device="cuda")
        mask &= (i[None] <= i[:, None]) | (i < limit[where.clamp(min=0)])[None]
    return mask


def check(tokens, offsets, heads, kv, dim, lengths=None, prefixes=None, causal=True, cap=0.0, slopes=False, together=400, padding=0, seed=0):
    """Results and gradients of one call, by pieces of whole documents of about `together` positions; `padding`: empty documents behind the others."""
    q, k, v, d = tensors(tokens, heads, kv, dim, seed=seed, layout="own")
    a = rb.DocumentAttention(heads, dim, kv, max_tokens=tokens, causal=causal, cap=cap)
    more = [0] * padding
    docs = documents(offsets + [offsets[-1]] * padding, None if lengths is None else lengths + more, None if prefixes is None else prefixes + more)
    low, scale = slopes_of(heads) if slopes else None, dim ** -0.5
    into = a.outputs(tokens)
    into.out.fill_(7.0), into.lse.fill_(7.0)
    got = a.forward(q, k, v, docs, slopes=low, out=into)
    grads = tuple(torch.full_like(x, 7.0) for x in (q, k, v))
    a.grad(q, k, v, docs, got.out, got.lse, d, slopes=low, out=grads)
    assert (got.out[offsets[-1]:] == 0).all() and (got.lse[:, offsets[-1]:] == -INF).all() and all((x[offsets[-1]:] == 0).all() for x in grads)
    first = 0
    while first < len(offsets) - 1:
        last = first + 1
        while last < len(offsets) - 1 and offsets[last + 1] - offsets[first] <= together:
            last += 1
        at = slice(offsets[first], offsets[last])
        n = at.stop - at.start
        if n:
            mask = seen([x - at.start for x in offsets[first:last + 1]], lengths and lengths[first:last], prefixes and prefixes[first:last], causal)
            some = mask.any(1)
            args = [x[at].double() for x in (q, k, v)]
            out, lse, off_out, off_lse = ref.attend(*args, scale, cap, None if low is None else low.double(), mask)
            have_out, have_lse = got.out[at].double(), got.lse[:, at].double()
            assert (have_out[~some] == 0).all() and (have_lse[:, ~some] == -INF).all()
            assert ((have_out - out).abs() <= off_out)[some].all(), (at, ((have_out - out).abs() / off_out)[some].max())
            assert ((have_lse - lse).abs() <= off_lse)[:, some].all(), (at, ((have_lse - lse).abs() / off_lse)[:, some].max())
            del out, lse, off_out, off_lse
            want, off = ref.attend_grad(*args, have_out, have_lse, d[at].double(), scale, cap, None if low is None else low.double(), mask)
            for name, x, w, o in zip("qkv", grads, want, off):
                x = x[at].double()
                assert (x[~some] == 0).all(), name
                assert ((x - w).abs() <= o).all(), (at, name, ((x - w).abs() / o).max())
            del want, off, mask
        first = last
    return a, (q, k, v, d), docs, got, grads


def many(count, mean, seed):
    """Offsets of `count` documents of about `mean` positions, some of none; lengths in a padded batch; prefixes."""
    rng = random.Random(seed)
    sizes = [rng.choice((0, 1, mean // 2, mean, mean, 2 * mean - 1, 2 * mean)) for _ in range(count)]
    offsets = [0]
    for n in sizes:
        offsets.append(offsets[-1] + n)
    return offsets, [n - rng.randrange(0, n // 3 + 1) for n in sizes], [rng.randrange(0, n + 2) for n in sizes]


@pytest.mark.parametrize("count", [255, 256, 2047, 2048, 3001])
@pytest.mark.parametrize("kind", ["plain", "all", "not causal"])
def test_many_short_documents(count, kind):
    """Offsets that fit a workgroup's LDS and ones that do not, forward (2048) and backward (256)."""
    offsets, lengths, prefixes = many(count, 4, count)
    tokens = offsets[-1] + 5
    if kind == "plain":
        check(tokens, offsets, 2, 1, 16)
    elif kind == "all":
        check(tokens, offsets, 4, 2, 64, lengths, prefixes, cap=10.0, slopes=True)
    else:
        check(tokens, offsets, 1, 1, 128, lengths, causal=False)


@pytest.mark.parametrize("count", [255, 256, 300])
@pytest.mark.parametrize("cap,slopes", [(0.0, False), (25.0, False), (50.0, True)])
def test_many_documents_that_are_not_short(count, cap, slopes):
    """More than 128 positions in the mean: the other forms, with offsets in LDS and without, tiles in turn by length (up to 256) and as they lie."""
    offsets, lengths, prefixes = many(count, 150, count + 1)
    while offsets[-1] < 128 * count:
        offsets[-1] += 128
    tokens = offsets[-1]
    lengths[-1] = offsets[-1] - offsets[-2]
    check(tokens, offsets, 2, 1, 64, lengths, prefixes, cap=cap, slopes=slopes, together=1500)


@pytest.mark.parametrize("dim,heads,kv", [(16, 2, 1), (72, 1, 1), (128, 2, 2)])
@pytest.mark.parametrize("cap,slopes,causal", [(0.0, False, True), (0.0, False, False), (30.0, False, True), (30.0, True, False), (100.0, True, True)])
def test_one_long_document(dim, heads, kv, cap, slopes, causal):
    check(6001, [0, 5990], heads, kv, dim, causal=causal, cap=cap, slopes=slopes, prefixes=[1000])


def test_a_few_long_documents():
    """More than 256 tiles; keys' queries in parts."""
    check(34000, [0, 9000, 9001, 9001, 20000, 24000, 33900], 1, 1, 16, prefixes=[5, 1, 0, 3000, 0, 100], together=1)
    check(34000, [0, 9000, 9001, 9001, 20000, 24000, 33900], 1, 1, 64, lengths=[8000, 1, 0, 10999, 4000, 9000], causal=False, together=1)


@pytest.mark.parametrize("cap", [0.0, 30.0])
@pytest.mark.parametrize("padding", [10, 30, 300, 2500])
def test_offsets_that_are_padded_with_empty_documents(padding, cap):
    """Empty documents count among the documents that forms are chosen by, and nothing else knows of them."""
    offsets, lengths, prefixes = [0, 1700, 1701, 2900], [1650, 1, 1199], [30, 0, 2000]
    a, (q, k, v, d), docs, got, grads = check(3000, offsets, 4, 2, 64, lengths, prefixes, cap=cap, padding=padding, together=1)
    few = documents(offsets, lengths, prefixes)
    same = a.forward(q, k, v, few)
    if padding + 3 <= 3000 // 128:                      # the same forms: the same bits
        assert torch.equal(same.out, got.out) and torch.equal(same.lse, got.lse)
    # what either form is off by is in both: 2^-8 of the results' size and 2^-8 of their terms'
    assert (same.out.double() - got.out.double()).norm() <= 2.0 ** -7 * got.out.double().norm()
    assert (same.lse - got.lse)[:, :1650].abs().max() <= 1e-4
    # a forward of one form and gradients of the other are still each other's
    mixed = a.grad(q, k, v, few, got.out, got.lse, d)
    for x, y in zip(mixed, grads):
        assert (x.double() - y.double()).norm() <= 2.0 ** -6 * y.double().norm()
