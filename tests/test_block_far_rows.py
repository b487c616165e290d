"""Gradients of layer norm for rows that lie far from 0 (include/rb_block.h) on the GPU, against 64 bits from the rows themselves, not from the statistics that were returned."""
import pytest
import torch

import block_reference as ref
import paper_2406_03285_amd as rb

pytestmark = pytest.mark.gpu
F32 = torch.float32
EPS = 1e-5


def far_rows(width, rows=7):
    """Means up to 10^8 deviations away; the mean as one number of binary32 is off by up to half of a deviation."""
    g = torch.Generator().manual_seed(width)
    x = torch.randn((rows, width), generator=g, dtype=torch.float64)
    mean = torch.tensor([1e4, -1e4, 333.3, 77777.7, -0.01, 0.0, 1.5e3], dtype=torch.float64)[:rows]
    spread = torch.tensor([1e-3, 2e-3, 1e-4, 1e-2, 1.0, 1.0, 1e-4], dtype=torch.float64)[:rows]
    return (x * spread[:, None] + mean[:, None]).to(F32).cuda(), torch.randn((rows, width), generator=g).cuda(), torch.randn((rows, width), generator=g).cuda()


def gradients(x, gy, gt, w):
    """(of x, of the weight) in 64 bits by differentiation, and bounds on what the calls may be off by.

    Differences from the mean are exact, or off by half a step of themselves; `rest`, what the mean leaves, is a sum of at most 64 of them in a lane and 10 steps
    between lanes (100 half steps u of their mean size, which is the deviation's and the mean's half step); rstd has 60 half steps.  The sum of g h is made without
    rest and put right: 100 half steps of its terms with a shift of u |mean| rstd in h, and of the shift times the sum of g."""
    u = ref.F32_HALF
    x, w = ref.to64(x).requires_grad_(), ref.to64(w).requires_grad_()
    gy, gt = ref.to64(gy), ref.to64(gt)
    y, mean, rstd = ref.norm(x, w, None, EPS)
    want = torch.autograd.grad((y * gy).sum() + (x * gt).sum(), (x, w))
    x, w, mean, rstd = (t.detach() for t in (x, w, mean, rstd))
    h = ((x - mean[:, None]) * rstd[:, None]).abs()
    shift = u * mean.abs() * rstd
    off_h = h * 70 * u + (110 * u * ((x - mean[:, None]).abs().mean(1) * rstd + shift))[:, None]
    g = (gy * w).abs()
    c0, c1 = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    off_c1 = 110 * u * (c1 + 2 * shift[:, None] * c0) + (g * off_h).mean(1, keepdim=True)
    off = rstd[:, None] * (110 * u * c0 + h * off_c1 + off_h * c1 + 70 * u * (g + c0 + h * c1)) + 2 * u * gt.abs() + ref.F32_HALF * want[0].abs()
    off_w = (gy.abs() * off_h).sum(0) + (x.shape[0] + 64) * u * (gy.abs() * h).sum(0) + ref.F32_HALF * want[1].abs()
    return want, (off, off_w)


@pytest.mark.parametrize("width", [1, 7, 50, 129, 300, 700, 1500, 2048, 5000, 8192, 12000, 16384, 16385, 20000, 32763])
def test_gradients_of_rows_that_lie_far_from_0(width):
    x, gy, gt = far_rows(width)
    w = (1 + 0.3 * torch.randn(width, generator=torch.Generator().manual_seed(1))).cuda()
    n = rb.LayerNorm(width, F32, eps=EPS)
    o = n.forward(x, w)
    g = n.grad(gy, x, w, o.mean, o.rstd, grad_total=gt, bias=False)
    want, off = gradients(x, gy, gt, w)
    for name, have, exact, bound in (("x", g.total, want[0], off[0]), ("weight", g.weight, want[1], off[1])):
        d = (ref.to64(have) - exact).abs()
        assert (d <= bound).all(), (name, (d / bound).max())
    # in place of the gradient that arrives: the same
    gy2 = gy.clone()
    into = rb.NormGrads(gy2, None, torch.empty_like(w), None)
    n.grad(gy2, x, w, o.mean, o.rstd, grad_total=gt, bias=False, out=into)
    assert torch.equal(gy2, g.total) and torch.equal(into.weight, g.weight)


@pytest.mark.parametrize("width", [300, 20000])
def test_gradients_of_many_far_rows_with_dropout(width):
    """More rows than workgroups, in one call as in many of one row."""
    rows = 700
    x = far_rows(width)[0].repeat(rows // 7, 1)
    gy, gt = (torch.randn(x.shape, generator=torch.Generator("cuda").manual_seed(s), device="cuda") for s in (1, 2))
    w = torch.ones(width, device="cuda")
    n = rb.LayerNorm(width, F32, eps=EPS)
    d = rb.Drop(0.3, 5, 6)
    o = n.forward(x, w)
    g = n.grad(gy, x, w, o.mean, o.rstd, grad_total=gt, drop=d)
    want, off = gradients(x, gy, gt, w)
    assert ((ref.to64(g.total) - want[0]).abs() <= off[0]).all() and ((ref.to64(g.weight) - want[1]).abs() <= off[1]).all()
    gy2, gt2 = gy.clone(), gt.clone()
    into = rb.NormGrads(gt2, gy2, torch.empty_like(w), torch.empty_like(w))
    n.grad(gy2, x, w, o.mean, o.rstd, grad_total=gt2, drop=d, out=into)
    assert all(torch.equal(a, b) for a, b in zip(into, g))


@pytest.mark.parametrize("width", [2000, 20000])
def test_captured_gradients_of_far_rows_are_the_eager_ones(width):
    """Apart from the gradient that arrives and in its place, several replays, the program's own work between them."""
    x, gy, gt = far_rows(width)
    w = torch.ones(width, device="cuda")
    n = rb.LayerNorm(width, F32, eps=EPS)
    o = n.forward(x, w)
    kept, gy2, gw2 = n.gradients(7), torch.empty_like(gy), torch.empty_like(w)

    def step():
        n.grad(gy, x, w, o.mean, o.rstd, grad_total=gt, out=kept)
        gy2.copy_(gy)
        n.grad(gy2, x, w, o.mean, o.rstd, grad_total=gt, out=rb.NormGrads(gy2, None, gw2, None))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(4):
        gy.copy_(torch.randn(gy.shape, generator=torch.Generator("cuda").manual_seed(turn), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (kept.total, kept.weight, kept.bias, gy2, gw2)]
        want = n.grad(gy, x, w, o.mean, o.rstd, grad_total=gt)
        for a, b in zip(got, (want.total, want.weight, want.bias, want.total, want.weight)):
            assert torch.equal(a, b), turn
        torch.cuda.synchronize()
