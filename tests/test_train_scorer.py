"""Scores of tokens and their gradient (include/rb_train.h) on the GPU against a plain statement in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2406_03285_amd as rb
import train_reference as ref

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
NEG = -float("inf")


def make(rows, vocab, dtype, pad=0, offset=0, seed=0, spread=3.0):
    """[rows, vocab] logits in rows of vocab + pad, the first one `offset` elements behind a 16-byte boundary."""
    g = torch.Generator().manual_seed(seed)
    z = (torch.randn((rows, vocab), generator=g) * spread).to(dtype)
    whole = torch.full((rows * (vocab + pad) + offset + 16,), 7.0, dtype=dtype, device="cuda")
    view = whole[offset:offset + rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab]
    view.copy_(z)
    return view


def tokens_for(rows, vocab, given, seed=0):
    g = torch.Generator().manual_seed(seed + 99)
    t = torch.randint(0, vocab, (rows, given), generator=g)
    if rows > 2:
        t[1] = -1                                   # left out
    if given > 2:
        t[0, 1] = t[0, 0]                           # the same token twice
        t[0, 2] = vocab                             # outside
    return t.cuda()


def check_score(z, tokens, top):
    rows, vocab = z.shape
    given = 0 if tokens is None else tokens.shape[1]
    s = rb.TokenScorer(vocab, z.dtype, given=given, top=top)
    got = s.score(z, tokens)
    want = ref.score(ref.to64(z), np.zeros((rows, 0), dtype=np.int64) if tokens is None else tokens.cpu().numpy(), top)
    bounds = ref.score_bounds(want)
    for name in ("lse", "entropy", "logp", "top_logp"):
        have = getattr(got, name)
        if have is None:
            continue
        have, w = ref.to64(have), want[name]
        assert np.array_equal(np.isnan(have), np.isnan(w)), name
        fine = np.isfinite(w)
        assert np.array_equal(have[~fine & ~np.isnan(w)], w[~fine & ~np.isnan(w)]), name
        assert (np.abs(have - w)[fine] <= bounds[name][fine]).all(), (name, np.abs(have - w)[fine].max())
    if top:
        assert np.array_equal(got.top_ids.cpu().numpy(), want["top_ids"])
    again = s.score(z, tokens)
    for a, b in zip(got, again):
        assert (a is None and b is None) or torch.equal(a.nan_to_num(7.5), b.nan_to_num(7.5))
    return got


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,vocab,given,top", [
    (1, 1, 1, 1), (3, 2, 3, 2), (5, 7, 1, 7), (2, 8, 0, 3), (4, 9, 2, 0), (7, 64, 64, 64), (3, 1000, 1, 5), (65, 1000, 17, 16),
    (1, 2047, 1, 33), (2, 2048, 1, 64), (3, 2049, 9, 1), (1, 8192, 1, 20), (1, 8193, 1, 20), (2, 50001, 17, 16), (1, 131075, 3, 64),
    (600, 4099, 1, 4), (1030, 2500, 1, 0), (4, 32000, 0, 0), (9, 300007, 1, 7),
])
def test_scores(rows, vocab, given, top, dtype):
    z = make(rows, vocab, dtype, seed=vocab)
    check_score(z, tokens_for(rows, vocab, given) if given else None, top)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (3, 2), (5, 7), (8, 3), (40, 0)])
def test_scores_of_rows_that_lie_anyhow(pad, offset, dtype):
    for vocab in (5, 11, 2051, 10007):
        check_score(make(4, vocab, dtype, pad, offset), tokens_for(4, vocab, 3), 5)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [40, 2048, 5003, 40961])
def test_equal_and_ordered_logits(vocab, dtype):
    """The lowest index wins: rows of one value, of few values, of zeros of both signs, ascending, descending."""
    i = torch.arange(vocab, dtype=torch.float32)
    rows = [torch.zeros(vocab), torch.full((vocab,), -3.5), i % 3, torch.where(i % 2 == 0, 0.0, -0.0), i / 64, -i / 64, (i * 7919 % 101) / 8,
            torch.where(i == vocab - 1, 9.0, 0.0), torch.where(i == 0, 9.0, 9.0 - i.clamp(max=1))]
    z = torch.stack(rows).to(dtype).cuda()
    for top in (1, 20, min(64, vocab)):
        check_score(z, tokens_for(len(rows), vocab, 2), top)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [3, 70, 2100, 20011])
def test_masks_and_what_is_not_a_number(vocab, dtype):
    lowest = torch.finfo(dtype).min
    base = torch.randn((14, vocab), generator=torch.Generator().manual_seed(5)).to(dtype)
    base[0] = NEG                                    # nothing left
    base[1] = NEG
    base[1, vocab - 1] = 2.0                         # one left
    base[2, : vocab // 2] = NEG
    base[3] = lowest
    base[4] = lowest
    base[4, 1] = 0.5
    base[5, vocab // 2:] = lowest
    base[6, vocab // 3] = float("nan")
    base[7, 0] = float("inf")
    base[8] = float("nan")
    base[9] = float("inf")
    base[10] = torch.finfo(dtype).max
    base[11, 1:] = NEG
    base[12] = base[12] * 1e4
    base[13, 0] = NEG
    base[13, vocab - 1] = float("nan")
    z = base.cuda()
    t = torch.tensor([[0, vocab - 1]] * 14).cuda()
    s = check_score(z, t, min(3, vocab))
    scorer = rb.TokenScorer(vocab, dtype, given=2)
    w, h = torch.full((14, 2), 0.25, device="cuda"), torch.full((14,), -0.5, device="cuda")
    got = ref.to64(scorer.grad(z, t, s.lse, s.entropy, w, h))
    assert (got[0] == 0).all() and np.isnan(got[[6, 7, 8, 9, 13]]).all()
    fine = [1, 2, 3, 4, 5, 10, 11, 12]
    want, off = ref.grad(ref.to64(z)[fine], t.cpu().numpy()[fine], ref.to64(s.lse)[fine], ref.to64(s.entropy)[fine], ref.to64(w)[fine], ref.to64(h)[fine])
    off += np.abs(want) * (2.0 ** -8 if dtype == BF16 else 2.0 ** -23)
    assert np.isfinite(got[fine]).all() and (np.abs(got[fine] - want) <= off).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,vocab,given,entropy,pad,out_pad,offset", [
    (1, 1, 1, True, 0, 0, 0), (3, 2, 3, True, 0, 0, 0), (5, 13, 1, False, 3, 3, 1), (4, 1000, 17, True, 0, 0, 0), (2, 8197, 64, True, 0, 0, 0),
    (3, 50001, 9, True, 47, 47, 0), (3, 5001, 9, True, 47, 0, 3), (2, 1003, 0, True, 0, 0, 0), (1, 131075, 1, False, 0, 0, 0), (300, 2048, 2, True, 0, 0, 0),
    (2, 70001, 64, True, 0, 1, 5),
])
def test_gradient_of_the_formula(rows, vocab, given, entropy, pad, out_pad, offset, dtype):
    z = make(rows, vocab, dtype, pad, offset, seed=given)
    t = tokens_for(rows, vocab, given) if given else None
    if given == 64:                                  # neighbours within one vector, and at both ends of the row
        t[1] = torch.arange(64) % 11 + 4
        t[1, 60:] = torch.tensor([0, vocab - 1, vocab - 2, 1])
    scorer = rb.TokenScorer(vocab, dtype, given=given)
    s = scorer.score(z, t)
    g = torch.Generator().manual_seed(3)
    w = torch.randn((rows, given), generator=g).cuda() if given else None
    h = torch.randn((rows,), generator=g).cuda() if entropy else None
    out = torch.full((rows, vocab + out_pad), 3.0, dtype=dtype, device="cuda")
    got = scorer.grad(z, t, s.lse, s.entropy, w, h, out=out[:, :vocab])
    want, off = ref.grad(ref.to64(z), np.zeros((rows, 0), dtype=np.int64) if t is None else t.cpu().numpy(), ref.to64(s.lse), ref.to64(s.entropy),
                         np.zeros((rows, 0)) if w is None else ref.to64(w), None if h is None else ref.to64(h))
    off += np.abs(want) * (2.0 ** -8 if dtype == BF16 else 2.0 ** -23)
    assert (np.abs(ref.to64(got) - want) <= off).all()
    assert (out[:, vocab:] == 3.0).all()
    inplace = scorer.grad(z, t, s.lse, s.entropy, w, h, out=z)
    assert inplace.data_ptr() == z.data_ptr() and torch.equal(z, got)


def test_gradient_against_differences():
    """Central differences of a loss of the 64-bit statement, and autograd through the call."""
    rows, vocab, given = 3, 37, 3
    z = make(rows, vocab, F32, seed=8, spread=1.5)
    z[2, 5] = NEG
    t = torch.tensor([[1, 1, 36], [0, -1, 5], [7, 8, 37]]).cuda()
    scorer = rb.TokenScorer(vocab, F32, given=given, top=2)
    w = torch.randn((rows, given), generator=torch.Generator().manual_seed(1)).cuda()
    h = torch.tensor([0.3, -0.7, 1.1]).cuda()

    def loss(z64):
        s = ref.score(z64, t.cpu().numpy(), 0)
        return (s["logp"] * ref.to64(w)).sum() + (s["entropy"] * ref.to64(h)).sum()

    z.requires_grad_()
    s = scorer(z, t)
    assert not s.lse.requires_grad and not s.top_logp.requires_grad
    ((s.logp * w).sum() + (s.entropy * h).sum()).backward()
    z64 = ref.to64(z)
    for i in range(rows):
        for j in range(vocab):
            if np.isneginf(z64[i, j]):
                continue
            d = np.zeros_like(z64)
            d[i, j] = 1e-5
            slope = (loss(z64 + d) - loss(z64 - d)) / 2e-5
            # differences are off by the third derivative (under 10 here) times 1e-10 / 6 and by 1e-15 * |loss| / 1e-5; binary32 by some 2^-20
            assert abs(slope - float(z.grad[i, j])) < 2.0 ** -18, (i, j)
    # one of the two alone, and derivatives that are broadcast
    z.grad = None
    scorer(z, t).entropy.sum().backward()
    alone = z.grad.clone()
    want, off = ref.grad(z64, np.full((rows, given), -1), ref.to64(s.lse), ref.to64(s.entropy), np.zeros((rows, given)), np.ones(rows))
    assert (np.abs(ref.to64(alone) - want) <= off + np.abs(want) * 2.0 ** -23).all()


@pytest.mark.parametrize("rows", [1, 700])
def test_on_a_stream_of_its_own_and_in_a_graph(rows):
    vocab = 33000
    z, t = make(rows, vocab, BF16), tokens_for(rows, vocab, 2)
    scorer = rb.TokenScorer(vocab, BF16, given=2, top=9)
    first = scorer.score(z, t)
    w, h = torch.randn((rows, 2), device="cuda"), torch.randn((rows,), device="cuda")
    dz = scorer.grad(z, t, first.lse, first.entropy, w, h)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = scorer.score(z, t)
        dz2 = scorer.grad(z, t, again.lse, again.entropy, w, h)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, again)) and torch.equal(dz, dz2)
    out, into = scorer.outputs(rows), torch.empty_like(dz)
    graph = torch.cuda.CUDAGraph()
    scorer.score(z, t, out=out)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        scorer.score(z, t, out=out)
        scorer.grad(z, t, out.lse, out.entropy, w, h, out=into)
    for k in range(4):
        z.copy_(make(rows, vocab, BF16, seed=k + 50))
        graph.replay()
        want = rb.TokenScorer(vocab, BF16, given=2, top=9).score(z, t)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), k
        assert torch.equal(into, scorer.grad(z, t, want.lse, want.entropy, w, h)), k


def test_rows_far_apart():
    """Offsets beyond 32 bits: rows 2^31 + 5 elements apart."""
    vocab, stride = 3001, (1 << 31) + 5
    whole = torch.empty(2 * stride + vocab, dtype=BF16, device="cuda")
    z = whole.as_strided((3, vocab), (stride, 1))
    z.copy_(torch.randn((3, vocab), generator=torch.Generator().manual_seed(2)).to(BF16))
    got = check_score(z, tokens_for(3, vocab, 1), 4)
    scorer = rb.TokenScorer(vocab, BF16)
    t, w = tokens_for(3, vocab, 1), torch.ones((3, 1), device="cuda")
    near = scorer.grad(z.contiguous(), t, got.lse, got.entropy, w)
    assert torch.equal(scorer.grad(z, t, got.lse, got.entropy, w, out=z), near)


@pytest.mark.parametrize("rows,vocab", [(1, 200000), (3, 131075), (100, 70000), (2, 66000)])
def test_rows_shared_by_workgroups(rows, vocab):
    """What the parts of an earlier call left does not matter, and the counters are back at nothing."""
    z, t = make(rows, vocab, BF16, seed=rows), tokens_for(rows, vocab, 2)
    scorer = rb.TokenScorer(vocab, BF16, given=2, top=40)
    first = scorer.score(z, t)
    counters = scorer.workspace[:1024].view(torch.int32)
    assert (counters == 0).all()
    scorer.workspace[1024:].fill_(0xFF)
    for a, b in zip(first, scorer.score(z, t)):
        assert torch.equal(a, b)
    assert (counters == 0).all()
    check_score(z, t, 40)
