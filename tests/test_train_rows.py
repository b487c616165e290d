"""Scores of many rows (include/rb_train.h) on the GPU, at the numbers of rows where a row's share of the chip changes, against binary64."""
import numpy as np
import pytest
import torch

import paper_2406_03285_amd as rb
import train_reference as ref

pytestmark = pytest.mark.gpu


def check(z, t, top):
    rows, vocab = z.shape
    s = rb.TokenScorer(vocab, z.dtype, given=t.shape[1], top=top).score(z, t)
    want = {k: [] for k in ("lse", "entropy", "logp", "top_logp", "top_ids", "spread")}
    for z64, tokens in zip(z.double().split(512), t.split(512)):
        logp = torch.log_softmax(z64, 1)
        ids = torch.sort(z64, dim=1, descending=True, stable=True).indices[:, :top]
        want["lse"].append(torch.logsumexp(z64, 1))
        want["spread"].append(want["lse"][-1] - z64.amax(1))
        want["entropy"].append(-(logp.exp() * logp).sum(1))
        want["logp"].append(logp.gather(1, tokens))
        want["top_ids"].append(ids)
        want["top_logp"].append(logp.gather(1, ids))
    want = {k: torch.cat(v).cpu().numpy() for k, v in want.items()}
    for name, bound in ref.score_bounds(want).items():
        have = getattr(s, name)
        if have is not None:
            assert (np.abs(ref.to64(have) - want[name]) <= bound).all(), name
    if top:
        assert np.array_equal(s.top_ids.cpu().numpy(), want["top_ids"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("top", [0, 3, 40])
@pytest.mark.parametrize("rows,vocab", [(511, 9001), (1600, 9001), (1700, 9001), (2049, 9001), (2049, 70001), (4097, 9001), (4097, 17001)])
def test_rows_on_both_sides_of_every_line(rows, vocab, top, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows + vocab)
    z = (3.0 * torch.randn((rows, vocab), generator=g, device="cuda")).to(dtype)
    check(z, torch.randint(0, vocab, (rows, 2), generator=g, device="cuda"), top)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab", [(700, 9001), (1700, 9001), (4097, 9001)])
def test_rows_that_are_in_order_or_equal(rows, vocab, dtype):
    """Every element of a rising row is a candidate when it comes; a falling row's first ones are the last; equal ones go by index."""
    i = torch.arange(vocab, device="cuda").float()
    kinds = torch.stack([i * (20.0 / vocab), -i * (20.0 / vocab), torch.zeros_like(i), (i * 7919) % 101 / 8]).to(dtype)
    z = kinds[torch.arange(rows, device="cuda") % 4]
    check(z, torch.zeros((rows, 1), dtype=torch.int64, device="cuda"), 20)
