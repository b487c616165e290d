"""Orthogonalised updates (include/rb_train.h) on the GPU against a plain statement in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2406_03285_amd as rb
import train_reference as ref

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
FIVE = (rb.NEWTON_SCHULZ,) * 5


def update(batch, m, n, dtype, seed=0, size=1e-3):
    g = torch.Generator().manual_seed(seed)
    low = torch.randn((batch, m, 4), generator=g) @ torch.randn((batch, 4, n), generator=g)
    return (size * (torch.randn((batch, m, n), generator=g) + low)).to(dtype).cuda()


def check(got, u, coefficients=FIVE, eps=1e-7):
    got, u = ref.to64(got), ref.to64(u)
    dtype_off = 2.0 ** -9
    for x, g in zip(got, u):
        want = ref.orthogonal(g, coefficients, eps)
        norm = np.linalg.norm(want)
        assert np.linalg.norm(x - want) <= (ref.orthogonal_bound(coefficients) + dtype_off) * norm, np.linalg.norm(x - want) / norm


def check_f32(got, u, coefficients=FIVE, eps=1e-7):
    for x, g in zip(ref.to64(got), ref.to64(u)):
        want = ref.orthogonal(g, coefficients, eps)
        norm = np.linalg.norm(want)
        assert np.linalg.norm(x - want) <= ref.orthogonal_bound(coefficients) * norm, np.linalg.norm(x - want) / norm


SHAPES = [(1, 1, 1), (1, 1, 70), (1, 70, 1), (3, 2, 3), (2, 16, 16), (1, 31, 33), (2, 64, 64), (1, 65, 64), (5, 100, 60), (1, 128, 128), (2, 129, 40),
          (1, 127, 300), (2, 300, 127), (1, 256, 256), (1, 257, 513), (3, 200, 333), (1, 640, 512), (1, 40, 3000), (1, 3001, 50), (40, 48, 96)]


@pytest.mark.parametrize("batch,m,n", SHAPES)
@pytest.mark.parametrize("dtype,out_dtype", [(F32, F32), (BF16, BF16), (BF16, F32)])
def test_orthogonalized(batch, m, n, dtype, out_dtype):
    u = update(batch, m, n, dtype, seed=m * n)
    o = rb.Orthogonalizer(m, n, batch=batch, dtype=dtype, out_dtype=out_dtype)
    kept = u.clone()
    got = o.orthogonalize(u)
    assert torch.equal(u, kept) and got.dtype == out_dtype
    (check_f32 if out_dtype == F32 else check)(got, u)
    assert torch.equal(o.orthogonalize(u), got)
    if dtype == out_dtype:
        assert torch.equal(o.orthogonalize(u, out=u), got) and torch.equal(u, got)


@pytest.mark.parametrize("m,n", [(96, 96), (130, 260), (300, 140)])
def test_other_coefficients_and_steps(m, n):
    for coefficients in ([(1.5, -0.5, 0.0)], [(1.875, -1.25, 0.375)] * 3, [(3.0, -3.2, 1.1), (2.0, -1.5, 0.5)], [(1.5, -0.5, 0.0)] * 12):
        u = update(1, m, n, F32, seed=len(coefficients))
        check_f32(rb.Orthogonalizer(m, n, coefficients=coefficients).orthogonalize(u), u, coefficients)


@pytest.mark.parametrize("batch", [1, 3])
def test_strided_matrices(batch):
    """Matrices within a larger tensor: columns of a wider one, matrices side by side, rows at odd places."""
    for m, n in ((33, 65), (140, 70), (130, 200)):
        wide = torch.full((batch, m, n + 7), 5.0, device="cuda")
        u = wide[:, :, 3:3 + n]
        u.copy_(update(batch, m, n, F32, seed=m))
        o = rb.Orthogonalizer(m, n, batch=batch)
        plain = o.orthogonalize(u.contiguous())
        assert torch.equal(o.orthogonalize(u), plain)
        beside = torch.full((m, batch * n), 5.0, device="cuda")
        into = beside.view(m, batch, n).transpose(0, 1)
        assert torch.equal(o.orthogonalize(u, out=into), plain)
        o.orthogonalize(u, out=u)
        assert torch.equal(u, plain) and (wide[:, :, :3] == 5.0).all() and (wide[:, :, 3 + n:] == 5.0).all()


@pytest.mark.parametrize("m,n", [(20, 30), (160, 140)])
def test_sizes_of_the_update_and_what_is_not_a_number(m, n):
    for dtype in (F32, BF16):
        o = rb.Orthogonalizer(m, n, batch=6, dtype=dtype, out_dtype=F32, eps=0.0)
        u = update(6, m, n, F32)
        u[0] = 0.0
        u[1] *= 1e30 / u[1].abs().max()
        u[2] *= 1e-30 / u[2].abs().max()
        u[3, 1, 1] = float("nan")
        u[4, 0, 2] = float("inf")
        u = u.to(dtype)
        got = o.orthogonalize(u)
        assert (got[0] == 0).all()
        assert torch.isnan(got[3]).any() and torch.isnan(got[4]).any()
        check_f32(got[[1, 2, 5]], u[[1, 2, 5]], eps=0.0)


@pytest.mark.parametrize("dtype,weights", [(F32, F32), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("batch,m,n", [(1, 7, 5), (2, 64, 48), (1, 300, 130), (3, 130, 257)])
@pytest.mark.parametrize("nesterov", [True, False])
def test_optimiser_step(batch, m, n, dtype, weights, nesterov):
    o = rb.Orthogonalizer(m, n, batch=batch, dtype=dtype, out_dtype=weights)
    w = update(batch, m, n, weights, seed=1, size=0.05)
    mom = update(batch, m, n, F32, seed=2)
    lr, beta, decay, scale = 0.02, 0.9, 0.1, 1.25
    for k in range(2):
        g = update(batch, m, n, dtype, seed=10 + k)
        w64, m64, g64 = ref.to64(w), ref.to64(mom), ref.to64(g)
        o.step(w, g, mom, lr=lr, beta=beta, nesterov=nesterov, weight_decay=decay, scale=scale)
        new = np.float32(beta).astype(np.float64) * m64 + g64
        assert (np.abs(ref.to64(mom) - new) <= 2.0 ** -23 * (np.abs(m64) + np.abs(g64))).all()
        used = g64 + beta * new if nesterov else new
        for i in range(batch):
            step = lr * scale * ref.orthogonal(used[i], FIVE, 1e-7)
            want = (1 - lr * decay) * w64[i] - step
            rounding = (2.0 ** -9 if weights == BF16 else 2.0 ** -22) * np.linalg.norm(np.abs(w64[i]) + np.abs(step))
            assert np.linalg.norm(ref.to64(w)[i] - want) <= rounding + 1.5 * ref.orthogonal_bound(FIVE) * np.linalg.norm(step)


def test_default_scale_and_momentum_shape():
    o = rb.Orthogonalizer(90, 10)
    w, mom = torch.zeros((90, 10), device="cuda"), torch.zeros((90, 10), device="cuda")
    g = update(1, 90, 10, F32)[0]
    o.step(w, g, mom, lr=1.0, beta=0.0)
    torch.testing.assert_close(w, -3.0 * o.orthogonalize(g), rtol=2e-6, atol=2e-6)
    assert torch.equal(mom, g)


@pytest.mark.parametrize("m,n", [(60, 60), (260, 300)])
def test_on_a_stream_of_its_own_and_in_a_graph(m, n):
    o = rb.Orthogonalizer(m, n, batch=2)
    u = update(2, m, n, F32)
    first = o.orthogonalize(u)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = o.orthogonalize(u)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(first, again)
    out = torch.empty_like(u)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o.orthogonalize(u, out=out)
    for k in range(4):
        u.copy_(update(2, m, n, F32, seed=k + 7))
        graph.replay()
        want = rb.Orthogonalizer(m, n, batch=2).orthogonalize(u)
        torch.cuda.synchronize()
        assert torch.equal(out, want), k


def test_one_matrix_of_a_batch_does_not_touch_another():
    u = update(4, 150, 90, F32)
    whole = rb.Orthogonalizer(150, 90, batch=4).orthogonalize(u)
    one = rb.Orthogonalizer(150, 90)
    for i in range(4):
        assert torch.equal(one.orthogonalize(u[i]), whole[i])


def on_the_gpu(g, coefficients, eps):
    """ref.orthogonal for large matrices: the same products in binary64 on the GPU."""
    x = (g.t() if g.shape[0] > g.shape[1] else g).double().contiguous()
    x = x / (torch.linalg.vector_norm(x) + eps)
    for a, b, c in coefficients:
        p = x @ x.t().contiguous()
        x = a * x + (b * p + c * (p @ p)) @ x
    return x.t() if g.shape[0] > g.shape[1] else x


@pytest.mark.parametrize("batch,m,n", [
    (1, 1000, 1100), (3, 520, 777), (1, 2048, 2048), (1, 1700, 3000), (2, 1100, 1300), (1, 2048, 10016), (1, 6000, 1500), (1, 4096, 4096), (1, 3900, 4200),
    (1, 260, 20000), (70, 130, 150), (300, 129, 140)])
def test_every_tile_and_slicing(batch, m, n):
    """Sizes on both sides of where larger tiles, and slices of a long summed index, are the faster ones."""
    g = torch.Generator(device="cuda").manual_seed(m)
    u = torch.randn((batch, m, n), generator=g, device="cuda") + torch.randn((batch, m, 4), generator=g, device="cuda") @ torch.randn((batch, 4, n), generator=g, device="cuda")
    o = rb.Orthogonalizer(m, n, batch=batch)
    got = o.orthogonalize(u)
    assert torch.equal(o.orthogonalize(u), got)
    for i in {0, batch // 2, batch - 1}:
        want = on_the_gpu(u[i], FIVE, 1e-7)
        assert torch.linalg.vector_norm(got[i] - want) <= ref.orthogonal_bound(FIVE) * torch.linalg.vector_norm(want)
    if batch == 1:
        w = torch.randn((m, n), generator=g, device="cuda").to(BF16)
        mom = torch.zeros((m, n), device="cuda")
        before = w.double()
        rb.Orthogonalizer(m, n, out_dtype=BF16).step(w, u[0], mom, lr=0.5, beta=0.5, nesterov=False, weight_decay=0.5, scale=1.0)
        want = 0.75 * before - 0.5 * on_the_gpu(u[0], FIVE, 1e-7)
        off = torch.linalg.vector_norm(w.double() - want)
        assert off <= 2.0 ** -9 * torch.linalg.vector_norm(want) + ref.orthogonal_bound(FIVE) * torch.linalg.vector_norm(want - 0.75 * before)


@pytest.mark.parametrize("batch,m,n", [(2, 40, 50), (1, 100, 128), (1, 33, 70), (3, 50, 700), (2, 97, 300), (1, 130, 140), (2, 200, 333), (1, 300, 2500), (1, 1999, 1700)])
def test_what_the_workspace_held_does_not_matter(batch, m, n):
    """Room beyond the last row and column is never read into a sum: the workspace starts full of NaN."""
    u = update(batch, m, n, F32, seed=3)
    o = rb.Orthogonalizer(m, n, batch=batch)
    o.workspace.fill_(0xFF)
    got = o.orthogonalize(u)
    assert torch.isfinite(got).all()
    o.workspace.random_(0, 256)
    assert torch.equal(o.orthogonalize(u), got)
    for i in range(batch):
        want = on_the_gpu(u[i], FIVE, 1e-7)
        assert torch.linalg.vector_norm(got[i] - want) <= ref.orthogonal_bound(FIVE) * torch.linalg.vector_norm(want)


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6, 7])
@pytest.mark.parametrize("m,n", [(60, 2000), (2100, 110), (200, 3000)])
def test_blocks_of_steps(m, n, steps):
    """A long side: steps are made on the short side's square in pairs."""
    u = update(1, m, n, F32, seed=steps)[0]
    coefficients = (rb.NEWTON_SCHULZ,) * steps
    got = rb.Orthogonalizer(m, n, coefficients=coefficients).orthogonalize(u)
    want = on_the_gpu(u, coefficients, 1e-7)
    assert torch.linalg.vector_norm(got - want) <= ref.orthogonal_bound(coefficients) * torch.linalg.vector_norm(want)


@pytest.mark.parametrize("m,n", [(40, 1000), (621, 63), (128, 8000), (5000, 200)])
@pytest.mark.parametrize("strong", [1.0, 4.0, 20.0])
def test_strong_directions_cost_the_weak_ones_no_precision(m, n, strong):
    """A few directions much stronger than the rest.  Where two steps are made on A, what is rounded in A is carried through P A P: in a weak
    direction that is a (3.44) times the strong ones' gain, near 1, more than in the plain form in binary32, whose own error is the scale."""
    rng = np.random.default_rng(m + int(strong))
    u = rng.standard_normal((m, n)) + 0.5 * strong * rng.standard_normal((m, 8)) @ rng.standard_normal((8, n))
    u = torch.tensor(u.astype(np.float32), device="cuda")
    got = rb.Orthogonalizer(m, n, coefficients=FIVE).orthogonalize(u)
    want, plain = on_the_gpu(u, FIVE, 1e-7), u / torch.linalg.vector_norm(u)
    plain = plain if m <= n else plain.t().contiguous()
    for a, b, c in FIVE:
        s = plain @ plain.t().contiguous()
        plain = a * plain + (b * s + c * (s @ s)) @ plain
    plain = plain if m <= n else plain.t()
    assert torch.linalg.vector_norm(got - want) <= 4.0 * torch.linalg.vector_norm(plain - want)


@pytest.mark.parametrize("coefficients", [((4.0, -10.2, 7.1),) * 3, ((19.5, -78.0, 62.4), (5.0, -1.3149, 0.069157))])
def test_blocks_that_would_not_fit_are_not_made(coefficients):
    """Steps that raise small values much, by 4 each and by 19.5 and 5: pairs that raise them by more than 60 are not made."""
    u = update(1, 48, 3000, F32, seed=5)[0]
    got = rb.Orthogonalizer(48, 3000, coefficients=coefficients).orthogonalize(u)
    want = on_the_gpu(u, coefficients, 1e-7)
    assert torch.linalg.vector_norm(got - want) <= ref.orthogonal_bound(coefficients) * torch.linalg.vector_norm(want)
