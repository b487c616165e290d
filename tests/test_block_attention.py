"""Attention of packed documents and its gradients (include/rb_block.h) on the GPU against a plain statement in 64 bits."""
import numpy as np
import pytest
import torch

import block_reference as ref
import paper_2406_03285_amd as rb

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
INF, NAN = float("inf"), float("nan")


def tensors(tokens, heads, kv, dim, seed=0, layout="one", size=1.3):
    """q, k, v, grad_out: views of one tensor, tensors of their own, or heads before positions."""
    g = torch.Generator().manual_seed(seed + 1000 * tokens + dim)

    def new(n, scale=size):
        return (torch.randn((tokens, n, dim), generator=g) * scale).to(BF16)
    q, k, v, d = new(heads), new(kv), new(kv), new(heads, 1.0)
    if layout == "one":
        whole = torch.cat([x.flatten(1) for x in (q, k, v)], 1).cuda()
        q, k, v = (x.unflatten(1, (n, dim)) for x, n in zip(whole.split([heads * dim, kv * dim, kv * dim], 1), (heads, kv, kv)))
        return q, k, v, d.cuda()
    if layout == "heads":
        return tuple(x.transpose(0, 1).contiguous().cuda().transpose(0, 1) for x in (q, k, v, d))
    return tuple(x.cuda() for x in (q, k, v, d))


def documents(offsets, lengths=None, prefixes=None):
    def on(x):
        return None if x is None else torch.tensor(x, dtype=torch.int64, device="cuda")
    return rb.Documents(on(offsets), on(lengths), on(prefixes))


def slopes_of(heads):
    return torch.tensor([0.9 * 2.0 ** -h for h in range(heads)], device="cuda")


def check(q, k, v, d, offsets, lengths=None, prefixes=None, causal=True, cap=0.0, slopes=False, scale=None, grads=True):
    tokens, heads, dim = q.shape
    kv = k.shape[1]
    a = rb.DocumentAttention(heads, dim, kv, max_tokens=max(tokens, 1), causal=causal, scale=scale, cap=cap)
    scale = dim ** -0.5 if scale is None else scale
    docs, low = documents(offsets, lengths, prefixes), slopes_of(heads) if slopes else None
    into = a.outputs(tokens)
    into.out.fill_(7.0)
    into.lse.fill_(7.0)
    got = a.forward(q, k, v, docs, slopes=low, out=into)
    mask = ref.seen(tokens, offsets, lengths, prefixes, causal)
    some = mask.any(1)
    q64, k64, v64, d64, low64 = (ref.to64(x) for x in (q, k, v, d, low))
    out, lse, off_out, off_lse = ref.attend(q64, k64, v64, scale, cap, low64, mask)
    have_out, have_lse = ref.to64(got.out), ref.to64(got.lse)
    assert (have_out[~some] == 0).all() and (have_lse[:, ~some] == -INF).all()
    assert ((have_out - out).abs() <= off_out)[some].all(), ((have_out - out).abs() / off_out)[some].max()
    assert ((have_lse - lse).abs() <= off_lse)[:, some].all(), ((have_lse - lse).abs() / off_lse)[:, some].max()
    again = a.forward(q, k, v, docs, slopes=low)
    assert torch.equal(again.out, got.out) and torch.equal(again.lse, got.lse)
    if not grads:
        return got
    into = tuple(torch.full((tokens, n, dim), 7.0, dtype=BF16, device="cuda") for n in (heads, kv, kv))
    have = a.grad(q, k, v, docs, got.out, got.lse, d, slopes=low, out=into)
    want, off = ref.attend_grad(q64, k64, v64, have_out, have_lse, d64, scale, cap, low64, mask)
    for name, x, w, o in zip("qkv", have, want, off):
        x = ref.to64(x)
        assert (x[~some] == 0).all(), name
        assert ((x - w).abs() <= o).all(), (name, ((x - w).abs() / o).max())
    for x, y in zip(have, a.grad(q, k, v, docs, got.out, got.lse, d, slopes=low)):
        assert torch.equal(x, y)
    return got


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("tokens", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 321])
def test_one_document_of_any_length(tokens, dim):
    check(*tensors(tokens, 2, 1, dim), [0, tokens])
    check(*tensors(tokens, 1, 1, dim, layout="own"), [0, tokens], causal=False)


@pytest.mark.parametrize("dim", [8, 16, 24, 40, 56, 64, 72, 80, 96, 120, 128])
def test_heads_of_any_size(dim):
    check(*tensors(150, 3, 3, dim, layout="heads"), [0, 70, 150])
    check(*tensors(97, 2, 1, dim, layout="one"), [0, 33, 97], cap=5.0, slopes=True)


MANY = [0, 1, 1, 3, 40, 40, 40, 100, 164, 165, 230, 300, 300]


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("cap,slopes", [(0.0, False), (3.0, False), (0.0, True), (3.0, True)])
@pytest.mark.parametrize("causal,prefix,gaps", [(True, False, False), (True, True, False), (True, True, True), (False, False, True), (True, False, True)])
def test_documents_prefixes_and_gaps(causal, prefix, gaps, cap, slopes, dim):
    """Documents of 0, 1, 2, 37, .. positions, positions behind the last one, prefixes of nothing, some, more than all."""
    lengths = [max(0, b - a - (7 if i % 2 else 1)) for i, (a, b) in enumerate(zip(MANY, MANY[1:]))] if gaps else None
    prefixes = [(0, 5, 1000, 33, 64)[i % 5] for i in range(len(MANY) - 1)] if prefix else None
    check(*tensors(317, 4, 2, dim, seed=5), MANY, lengths, prefixes, causal, cap, slopes)


@pytest.mark.parametrize("dim", [40, 64, 72, 128])
@pytest.mark.parametrize("slopes", [False, True])
@pytest.mark.parametrize("causal,prefixes,lengths", [(True, None, None), (False, None, [260, 0, 150]), (True, [70, 5, 400], None)])
def test_capped_scores_of_long_documents(causal, prefixes, lengths, slopes, dim):
    """Documents of 128 positions and more in the mean have a form of capped scores of their own (up to a cap of 32)."""
    for cap in (3.0, 32.0):
        check(*tensors(431, 4, 2, dim, seed=6), [0, 270, 271, 431], lengths, prefixes, causal, cap, slopes)


@pytest.mark.parametrize("dim", [64, 72, 128])
@pytest.mark.parametrize("cap,slopes", [(0.0, False), (0.0, True), (4.0, True), (50.0, False)])
@pytest.mark.parametrize("causal,prefix,gaps", [(True, False, False), (True, True, True), (False, False, True), (False, False, False)])
def test_longer_documents(causal, prefix, gaps, cap, slopes, dim):
    """Documents of more than 160 positions in the mean, one of them of one position and one of none: tiles take turns by length."""
    offsets = [0, 1, 330, 330, 690]
    check(*tensors(700, 4, 2, dim, seed=8), offsets, [1, 300, 0, 355] if gaps else None, [0, 100, 7, 1000] if prefix else None, causal, cap, slopes)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 2.0, 30.0, 100.0])
def test_one_key_is_taken_as_it_is(cap, dim):
    """Where a position sees nothing but itself, out is v and lse is the score: a few roundings of the score away, not of the cap."""
    tokens, heads, scale = 41, 2, dim ** -0.5
    q, k, v, _ = tensors(tokens, heads, heads, dim, seed=9)
    a = rb.DocumentAttention(heads, dim, max_tokens=tokens, cap=cap)
    got = a.forward(q, k, v, documents(list(range(tokens + 1))))
    assert torch.equal(got.out, v)
    mask = torch.eye(tokens, dtype=torch.bool)
    q64, k64 = ref.to64(q), ref.to64(k)
    plain, _, off = ref.scores(q64, k64, scale, 0.0, None, mask)
    at = range(tokens)
    s, off = plain[:, at, at], off[:, at, at]
    want = cap * torch.tanh(s / cap) if cap else s
    # (the cap's slope is at most 1; tanh and its factors: 16 roundings)
    assert ((ref.to64(got.lse) - want).abs() <= off + 16 * ref.F32_HALF * want.abs()).all()


@pytest.mark.parametrize("dim,heads,kv,cap", [(16, 4, 2, 0.0), (64, 2, 2, 30.0), (128, 3, 1, 0.0)])
def test_short_documents_are_as_exact_as_their_results_rounding(dim, heads, kv, cap):
    """In the mean: what p and ds are off by, 2^-17 of themselves, is nothing beside the results' 2^-9 (one in 2^15 of its square, and rounded to the other side
    for as many); with p and ds in bfloat16 errors would be 1.4 times as large."""
    offsets = [0, 2, 4, 9, 10, 26, 29, 60]
    q, k, v, d = tensors(60, heads, kv, dim, seed=12)
    a = rb.DocumentAttention(heads, dim, kv, max_tokens=60, cap=cap)
    docs, mask, scale = documents(offsets), ref.seen(60, offsets), dim ** -0.5
    got = a.forward(q, k, v, docs)
    grads = a.grad(q, k, v, docs, got.out, got.lse, d)
    q64, k64, v64, d64 = (ref.to64(x) for x in (q, k, v, d))
    out, lse, _, _ = ref.attend(q64, k64, v64, scale, cap, None, mask)
    want, _ = ref.attend_grad(q64, k64, v64, out, lse, d64, scale, cap, None, mask)
    for name, have, exact in zip(("out", *"qkv"), (got.out, *grads), (out, *want)):
        assert (ref.to64(have) - exact).norm() <= 1.05 * (exact.to(BF16).double() - exact).norm(), name


@pytest.mark.parametrize("slopes", [False, True])
@pytest.mark.parametrize("heads,kv", [(2, 2), (8, 2)])
def test_one_key_has_no_gradient(heads, kv, slopes):
    """Documents of one position: its weight is 1 whatever its score is, so q and k have gradients of 0, and v that of out."""
    tokens, dim = 9, 128
    q, k, v, d = tensors(tokens, heads, kv, dim, seed=2)
    a = rb.DocumentAttention(heads, dim, kv, max_tokens=tokens)
    docs, low = documents(list(range(tokens + 1))), slopes_of(heads) if slopes else None
    got = a.forward(q, k, v, docs, slopes=low)
    grad_q, grad_k, grad_v = a.grad(q, k, v, docs, got.out, got.lse, d, slopes=low)
    assert (grad_q == 0).all() and (grad_k == 0).all()
    want = ref.to64(d).unflatten(1, (kv, heads // kv)).sum(2)
    # (weights of 1 within what lse is off by, a sum of some heads, a rounding)
    size = ref.to64(d).abs().unflatten(1, (kv, heads // kv)).sum(2)
    assert ((ref.to64(grad_v) - want).abs() <= want.abs() * ref.BF16_HALF + size * (ref.BF16_HALF + 2.0 ** -16)).all()
    q[4, 1, 5] = NAN
    got = a.forward(q, k, v, docs, slopes=low)
    grad_q, grad_k, _ = a.grad(q, k, v, docs, got.out, got.lse, d, slopes=low)
    assert grad_q[4, 1].isnan().all() and (grad_q[[0, 3, 5, 8]] == 0).all() and (grad_k[[0, 3, 5, 8]] == 0).all()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("small", [1, 8])
def test_infinities_in_tiles_that_are_seen_whole(small, dim):
    """One long document, alone or with some of one position behind it (the forms for short ones): who sees an infinity has it, and nothing else is changed."""
    tokens = 256 + small
    q, k, v, _ = tensors(tokens, 2, 2, dim, seed=4, layout="own")
    a = rb.DocumentAttention(2, dim, max_tokens=tokens, causal=False)
    docs = documents([0] + list(range(256, tokens + 1)))
    want = a.forward(q, k, v, docs).out.clone()
    v[5, 0, 3] = INF
    v[70, 1, 4] = -INF
    v[71, 1, 5] = NAN
    got = a.forward(q, k, v, docs).out
    want[:256, 0, 3] = INF
    want[:256, 1, 4] = -INF
    assert got[:256, 1, 5].isnan().all()
    got[:256, 1, 5] = want[:256, 1, 5]
    assert torch.equal(got, want)


def test_no_documents_and_documents_that_are_all_empty():
    q, k, v, d = tensors(70, 2, 2, 64)
    check(q, k, v, d, [0])
    check(q, k, v, d, [5, 5, 5])
    check(q, k, v, d, [0, 70], lengths=[0])
    check(q, k, v, d, [30, 60])                          # (the first 30 belong to none)


@pytest.mark.parametrize("heads,kv", [(1, 1), (5, 5), (6, 2), (7, 1), (12, 3)])
def test_shared_heads(heads, kv):
    check(*tensors(140, heads, kv, 64, seed=heads), [0, 90, 140])
    check(*tensors(140, heads, kv, 128, seed=heads), [0, 90, 130], prefixes=[20, 3])


@pytest.mark.parametrize("scale,cap,size", [(1.0, 0.0, 2.0), (0.01, 0.0, 1.0), (1.0, 0.5, 2.0), (1e-3, 1e4, 1.0), (3.0, 50.0, 3.0), (1e-30, 0.0, 1.0)])
def test_large_and_small_scores(scale, cap, size):
    q, k, v, d = tensors(130, 2, 2, 64, size=size)
    check(q, k, v, d, [0, 100, 130], scale=scale, cap=cap)


@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("times", [1, 4])
@pytest.mark.parametrize("dim", [64, 72, 128])
def test_what_lies_in_masked_places_does_not_matter(dim, times, cap):
    """NaN and infinities behind the documents, in gaps, in other documents and in positions to come; results as if they were 0."""
    n = times                                        # (documents of less and of more than 128 positions in the mean)
    offsets, lengths = [0, 50 * n, 130 * n, 190 * n], [40 * n, 80 * n, 55 * n]
    q, k, v, d = tensors(200 * n, 2, 1, dim, layout="own")
    a = rb.DocumentAttention(2, dim, 1, max_tokens=200 * n, cap=cap)
    docs = documents(offsets, lengths)
    nobody = ~ref.seen(200 * n, offsets, lengths).any(1)
    want = a.forward(q, k, v, docs)
    grads = a.grad(q, k, v, docs, want.out, want.lse, d)
    for bad in (NAN, INF, -INF):
        q2, k2, v2, d2, o2 = (x.clone() for x in (q, k, v, d, want.out))
        for x in (q2, k2, v2, d2, o2):
            x[nobody] = bad
        got = a.forward(q2, k2, v2, docs)
        assert torch.equal(got.out, want.out) and torch.equal(got.lse, want.lse)
        for x, y in zip(a.grad(q2, k2, v2, docs, o2, want.lse, d2), grads):
            assert torch.equal(x, y)
        # the second document is not a number: the others do not know
        others = torch.ones(200 * n, dtype=torch.bool)
        others[50 * n:130 * n] = False
        q2, k2, v2, d2, o2 = (x.clone() for x in (q, k, v, d, want.out))
        for x in (q2, k2, v2, d2, o2):
            x[50 * n:130 * n] = bad
        got = a.forward(q2, k2, v2, docs)
        assert torch.equal(got.out[others], want.out[others]) and torch.equal(got.lse[:, others], want.lse[:, others])
        for x, y in zip(a.grad(q2, k2, v2, docs, o2, want.lse, d2), grads):
            assert torch.equal(x[others], y[others])
        # one position of it: what lies before does not know, what lies behind and sees it does
        v2 = v.clone()
        v2[100 * n, 0, 3] = bad
        got = a.forward(q, k, v2, docs).out
        assert torch.equal(got[:100 * n], want.out[:100 * n]) and torch.equal(got[130 * n:], want.out[130 * n:])
        column = got[100 * n:130 * n, :, 3]
        assert torch.isnan(column).all() if bad != bad else (column == bad).all()
        keep = [c for c in range(dim) if c != 3]
        assert torch.equal(got[:, :, keep], want.out[:, :, keep])
        q2, d2 = q.clone(), d.clone()                    # a query's row: the keys behind it do not know
        q2[70 * n, 1] = bad
        d2[70 * n, 1] = bad
        g = a.grad(q2, k, v, docs, want.out, want.lse, d2)
        for x, y in zip(g, grads):
            assert torch.equal(x[70 * n + 1:], y[70 * n + 1:]) and torch.equal(x[:50 * n], y[:50 * n])
        assert torch.equal(g[0][50 * n:70 * n], grads[0][50 * n:70 * n]) and not torch.isfinite(g[2][50 * n:70 * n + 1].float()).any()


def test_rows_that_are_not_numbers():
    """A key that is NaN makes NaN of every row that sees it, an infinite score too."""
    q, k, v, d = tensors(90, 2, 2, 64, layout="own")
    k[40, 1, 5] = NAN
    a = rb.DocumentAttention(2, 64, max_tokens=90)
    got = a.forward(q, k, v, documents([0, 90]))
    assert torch.isnan(got.out[40:, 1]).all() and torch.isfinite(got.out[:, 0].float()).all() and torch.isfinite(got.out[:40].float()).all()
    assert torch.isnan(got.lse[1, 40:]).all() and torch.isfinite(got.lse[0]).all()


def definition(q, k, v, mask, scale, cap, slopes):
    out, _, _, _ = ref.attend(q, k, v, scale, cap, slopes, mask)
    return out


@pytest.mark.parametrize("cap,slopes,prefixes", [(0.0, False, None), (2.0, True, [4, 0])])
def test_gradient_against_differences(cap, slopes, prefixes):
    """Autograd through the call against central differences of the definition in 64 bits."""
    tokens, heads, kv, dim = 23, 2, 1, 8
    offsets = [0, 14, 22]
    q, k, v, d = tensors(tokens, heads, kv, dim, layout="own", size=1.0)
    low = slopes_of(heads) if slopes else None
    a = rb.DocumentAttention(heads, dim, kv, max_tokens=tokens, cap=cap)
    leaves = [x.clone().requires_grad_() for x in (q, k, v)]
    out = a(*leaves, documents(offsets, None, prefixes), low)
    out.backward(d)
    mask = ref.seen(tokens, offsets, None, prefixes)
    at = [ref.to64(x) for x in (q, k, v)]
    d64, low64, scale = ref.to64(d), ref.to64(low), dim ** -0.5
    exact, lse, _, _ = ref.attend(*at, scale, cap, low64, mask)
    _, off = ref.attend_grad(*at, exact, lse, d64, scale, cap, low64, mask)
    # (the bound is of an out that is exact: the call's is off by the weights' and its own half steps, which go on as `aside` does)
    some = torch.einsum("ihd->hi", (d64 * exact).abs() + d64.abs() * 0.5 * exact.abs().max()) * 4 * ref.BF16_HALF
    reach = 4 * ref.BF16_HALF * scale * some.max() * max(float(x.abs().max()) for x in at)
    g = np.random.RandomState(0)
    for n, (x, leaf, o) in enumerate(zip(at, leaves, off)):
        for _ in range(60):
            i = tuple(g.randint(0, s) for s in x.shape)
            e = torch.zeros_like(x)
            e[i] = 1e-5
            up, down = (definition(*[y + f * e if m == n else y for m, y in enumerate(at)], mask, scale, cap, low64) for f in (1, -1))
            slope = ((up - down) * d64).sum() / 2e-5
            assert abs(float(slope) - float(leaf.grad[i])) <= float(o[i]) + (0.0 if n == 2 else float(reach)) + 1e-7, (n, i)
            if n == 2:
                assert abs(float(slope)) < 50


def test_offsets_that_cannot_be():
    """Such calls read and write nothing else; what they give is not specified."""
    q, k, v, d = tensors(100, 2, 2, 64, layout="own")
    a = rb.DocumentAttention(2, 64, max_tokens=100)
    big = 2 ** 62
    for offsets, lengths, prefixes in (([60, 20, 90, 10], None, None), ([-50, 40, 400], None, None), ([0, 50, 100], [-3, big], [big, -big]),
                                       ([-big, big], [big], [big]), ([big, big], None, None), ([0, 100, 0, 100], None, [50, 50, 50])):
        whole = torch.full((102, 2, 64), 7.0, dtype=BF16, device="cuda")
        docs = documents(offsets, lengths, prefixes)
        o = rb.Attended(whole[1:101], torch.empty((2, 100), device="cuda"))
        a.forward(q, k, v, docs, out=o)
        grads = [torch.full((102, 2, 64), 7.0, dtype=BF16, device="cuda") for _ in range(3)]
        a.grad(q, k, v, docs, o.out, o.lse, d, out=tuple(x[1:101] for x in grads))
        for x in (whole, *grads):
            assert (x[0] == 7.0).all() and (x[101] == 7.0).all()


def test_positions_far_apart():
    """Offsets beyond 32 bits: positions as far apart as they may be, 2^26 elements, heads 2^32 and more apart."""
    tokens, heads, dim = 70, 2, 64
    q, k, v, d = tensors(tokens, heads, heads, dim, layout="own")
    a = rb.DocumentAttention(heads, dim, max_tokens=tokens)
    docs = documents([0, 17, 70])
    near = a.forward(q, k, v, docs)
    grads = a.grad(q, k, v, docs, near.out, near.lse, d)
    stride, head = 1 << 26, (1 << 32) + (1 << 31) + 8
    store = torch.empty((tokens - 1) * stride + head + dim, dtype=BF16, device="cuda")
    far = store.as_strided((tokens, heads, dim), (stride, head, 1))
    for which in range(3):
        far.copy_((q, k, v)[which])
        args = [far if i == which else x for i, x in enumerate((q, k, v))]
        assert torch.equal(a.forward(*args, docs).out, near.out)
        for x, y in zip(a.grad(*args, docs, near.out, near.lse, d), grads):
            assert torch.equal(x, y)
        a.grad(q, k, v, docs, near.out, near.lse, d, out=[far if i == which else torch.empty_like(x) for i, x in enumerate((q, k, v))])
        assert torch.equal(far, grads[which])
    a.forward(q, k, v, docs, out=rb.Attended(far, None))
    assert torch.equal(far, near.out)
