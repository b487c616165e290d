"""Precision of orthogonalised updates, by what the same iteration in binary32 is off by.

A product of include/rb_train.h takes operands as sums of two binary16 numbers.  What that puts in is, per product, 2^-24 for either operand's low
half and 2^-24 for the product of low halves that is left out, where binary32 puts in 2^-24 for rounding each stored result; both sum in binary32, and
both multiply what was put in by the same slopes.  So a result may be off by some 3 times binary32's where sums are short, and 4 is the bound.
Without a low half the operand is off by 2^-12: a thousand times as much.
"""
import numpy as np
import pytest
import torch

import paper_2406_03285_amd as rb

FIVE = (rb.NEWTON_SCHULZ,) * 5


def iteration(u, dtype, coefficients, eps=1e-7):
    """The definition in that type, the update's larger side last."""
    x = (u.t() if u.shape[0] > u.shape[1] else u).to(dtype).contiguous()
    x = x / (torch.linalg.vector_norm(x) + eps)
    for a, b, c in coefficients:
        s = x @ x.t().contiguous()
        x = a * x + (b * s + c * (s @ s)) @ x
    return (x.t() if u.shape[0] > u.shape[1] else x).double()


def errors(got, u, coefficients):
    want = iteration(u, torch.float64, coefficients)
    return torch.linalg.vector_norm(got.double() - want), torch.linalg.vector_norm(iteration(u, torch.float32, coefficients) - want)


# ---- a statement of the format on the CPU: what the bound below notices --------

def halves(x, scale):
    s = (x * np.float32(scale)).astype(np.float32)
    hi = s.astype(np.float16).astype(np.float32)
    return hi, (s - hi).astype(np.float16).astype(np.float32)


def product(p, q, low, scale):
    """p q^T with the low halves of "both", "left", "right" or "none" of the operands."""
    (ph, pl), (qh, ql) = p, q
    out = ph @ qh.T
    if low in ("both", "left"):
        out = out + pl @ qh.T
    if low in ("both", "right"):
        out = out + ph @ ql.T
    return out * np.float32(scale)


def in_halves(u, coefficients, low, pairs):
    x = (u / np.linalg.norm(u.astype(np.float64))).astype(np.float32)
    SX, SA, SB = 4096.0, 2048.0, 1024.0
    def square(p, q, sp, sq):
        return product(halves(p, sp), halves(q, sq), low, 1 / (sp * sq))
    step = 0
    while step < len(coefficients):
        a, b, c = (np.float32(v) for v in coefficients[step])
        s = square(x, x, SX, SX)
        if pairs and step + 1 < len(coefficients):
            eye = np.eye(len(s), dtype=np.float32)
            first = a * eye + b * s + c * square(s, s, SA, SA)
            s = square(first, square(first, s, SB, SA), SB, SA)
            a, b, c = (np.float32(v) for v in coefficients[step + 1])
            second = a * eye + b * s + c * square(s, s, SA, SA)
            x = square(square(second, first, SB, SB), x.T.copy(), SB, SX)
            step += 2
        else:
            x = a * x + square(b * s + c * square(s, s, SA, SA), x.T.copy(), SB, SX)
            step += 1
    return torch.tensor(x)


@pytest.mark.parametrize("m,n,pairs", [(50, 64, False), (128, 128, False), (130, 260, False), (60, 1000, True), (200, 900, True)])
def test_the_bound_holds_for_the_format_and_not_without_a_low_half(m, n, pairs):
    u = torch.tensor(np.random.default_rng(m).standard_normal((m, n)).astype(np.float32))
    for low in ("both", "left", "right", "none"):
        off, plain = errors(in_halves(u.numpy(), FIVE, low, pairs), u, FIVE)
        assert (off <= 4.0 * plain) if low == "both" else (off > 40.0 * plain), (low, off / plain)


# ---- the kernels ---------------------------------------------------------------

def updates(batch, m, n, dtype=torch.float32, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + m + n)
    return (1e-3 * torch.randn((batch, m, n), generator=g, device="cuda")).to(dtype)


FORMS = [
    (2, 40, 50), (1, 64, 64), (3, 33, 60),                                          # one workgroup, up to 64
    (1, 100, 128), (5, 128, 128), (2, 128, 40), (1, 65, 70),                        # one workgroup, up to 128
    (1, 130, 140), (1, 256, 256), (3, 200, 333), (24, 333, 200), (1, 1000, 1100),   # tiles of 64
    (1, 1900, 2100), (1, 2560, 2600), (4, 1000, 1000), (16, 700, 700),              # ... of 128, and of 192 for the last product
    (1, 3000, 3100), (1, 3500, 3500), (1, 4096, 4096),                              # ... of 192 and 256, with slices and without
    (1, 40, 1000), (40, 100, 400), (1, 2000, 60), (1, 1500, 200), (2, 260, 5000),   # pairs of steps
    (1, 6000, 1500), (1, 2048, 10016), (1, 3900, 4200),
]


@pytest.mark.gpu
@pytest.mark.parametrize("batch,m,n", FORMS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_results_are_as_near_as_those_of_binary32(batch, m, n, dtype):
    u = updates(batch, m, n, dtype)
    got = rb.Orthogonalizer(m, n, batch=batch, dtype=dtype, out_dtype=torch.float32).orthogonalize(u)
    for i in sorted({0, batch // 2, batch - 1}):
        off, plain = errors(got[i], u[i], FIVE)
        assert off <= 4.0 * plain, off / plain


@pytest.mark.gpu
@pytest.mark.parametrize("batch,m,n", [(1, 50, 64), (1, 128, 100), (2, 300, 256), (1, 2100, 1900), (1, 4096, 4000), (1, 60, 2000), (1, 3000, 250)])
def test_updates_of_a_step_are_as_near_as_those_of_binary32(batch, m, n):
    """Weights of 0 become the update itself (times -1); the momentum's rounding is the plain iteration's input too."""
    g, mom, w = updates(batch, m, n, torch.bfloat16), 5.0 * updates(batch, m, n, seed=1), torch.zeros((batch, m, n), device="cuda")
    rb.Orthogonalizer(m, n, batch=batch, dtype=torch.bfloat16, out_dtype=torch.float32).step(w, g, mom, lr=1.0, beta=0.9, nesterov=False, scale=1.0)
    for i in range(batch):
        off, plain = errors(-w[i], mom[i], FIVE)
        assert off <= 4.0 * plain, off / plain


@pytest.mark.gpu
@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6, 7])
@pytest.mark.parametrize("m,n", [(100, 90), (300, 257), (60, 2000), (2100, 200)])
def test_any_number_of_steps(m, n, steps):
    u = updates(1, m, n, seed=steps)[0]
    coefficients = (rb.NEWTON_SCHULZ,) * steps
    off, plain = errors(rb.Orthogonalizer(m, n, coefficients=coefficients).orthogonalize(u), u, coefficients)
    assert off <= 4.0 * plain, off / plain


@pytest.mark.gpu
@pytest.mark.parametrize("coefficients", [((1.5, -0.5, 0.0),), ((1.875, -1.25, 0.375),) * 3, ((3.0, -3.2, 1.1), (2.0, -1.5, 0.5)), ((1.5, -0.5, 0.0),) * 12])
@pytest.mark.parametrize("m,n", [(96, 96), (130, 260), (300, 140), (50, 1500)])
def test_other_coefficients(m, n, coefficients):
    u = updates(1, m, n)[0]
    off, plain = errors(rb.Orthogonalizer(m, n, coefficients=coefficients).orthogonalize(u), u, coefficients)
    assert off <= 4.0 * plain, off / plain


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,smallest", [(100, 100, 1e-8), (256, 256, 1e-8), (300, 256, 1e-8), (1000, 1100, 1e-8), (200, 1500, 1e-8), (1500, 200, 1e-8),
                                          (5000, 100, 1e-8), (2048, 3500, 1e-6), (4096, 4096, 1e-6)])
def test_small_rows_are_off_by_what_the_header_says(m, n, smallest):
    """Rows whose sizes fall evenly.  X is kept in steps of 2^-36 of the norm, so a row of n elements whose norm is r of the whole's is off by
    2^-36 sqrt(n / 12) / r of itself when it is kept first (later it is larger, and what is put in then less of it); A and P are kept in steps of 2^-35
    and 2^-34, which P A P and P2 P1 carry into a row of A and R as at most 64 times 2^-36 of each element, and X has a norm of 1 then."""
    u = updates(1, m, n)[0] * torch.logspace(0, np.log10(smallest), m, device="cuda")[:, None]
    got = rb.Orthogonalizer(m, n, coefficients=FIVE).orthogonalize(u).double()
    want = iteration(u, torch.float64, FIVE)
    size = torch.linalg.vector_norm(want, dim=1)
    off = torch.linalg.vector_norm(got - want, dim=1) / size
    plain = (torch.linalg.vector_norm(iteration(u, torch.float32, FIVE) - want, dim=1) / size).max()
    r = torch.linalg.vector_norm(u.double(), dim=1) / torch.linalg.vector_norm(u.double())
    assert (off <= 4.0 * plain + 2.0 ** -36 * (n ** 0.5 + 64) / r).all()


@pytest.mark.gpu
@pytest.mark.parametrize("m,n", [(30, 40), (120, 128), (200, 333), (60, 1000), (1500, 250)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_what_is_not_a_number_is_in_all_of_its_matrix_and_in_no_other(m, n, value):
    u = updates(3, m, n)
    o = rb.Orthogonalizer(m, n, batch=3)
    want = o.orthogonalize(u)
    u[1, m // 2, n - 1] = value
    got = o.orthogonalize(u)
    assert torch.isnan(got[1]).all() and torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])


# ---- pairs of steps of other coefficients --------------------------------------

MADE, NOT_MADE = ((4.0, -10.2, 7.1),) * 3, ((19.5, -78.0, 62.4), (5.0, -1.3149, 0.069157))


def workspace(coefficients, m=200, n=3000):
    rc, o = rb.rb_ortho_create(1, m, n, rb.RB_F32, rb.RB_F32, coefficients, 0.0)
    assert rc == rb.RB_OK
    rc, size = rb.rb_ortho_query(o)
    rb.rb_ortho_destroy(o)
    return size


def test_which_pairs_are_made():
    """A pair wants room for two more squares.  4 * 4 = 16 is kept, 19.5 * 5 = 97.5 would be beyond what a square's scale leaves (60)."""
    one = workspace(FIVE[:1])
    assert workspace(FIVE) > one and workspace(MADE) > one
    assert workspace(NOT_MADE) == one


@pytest.mark.gpu
@pytest.mark.parametrize("m,n", [(48, 3000), (200, 3000), (3000, 110)])
@pytest.mark.parametrize("coefficients", [MADE, NOT_MADE])
def test_steep_steps_are_as_near_as_those_of_binary32(m, n, coefficients):
    u = updates(1, m, n)[0]
    off, plain = errors(rb.Orthogonalizer(m, n, coefficients=coefficients).orthogonalize(u), u, coefficients)
    assert off <= 4.0 * plain, off / plain


@pytest.mark.gpu
@pytest.mark.parametrize("m,n", [(100, 100), (256, 256), (1500, 200), (1000, 1100)])
@pytest.mark.parametrize("norm", [1.0, 1e-7, 1e-9, 1e-11])
def test_updates_smaller_than_eps(m, n, norm):
    """X is G / (|G| + eps), and its steps are those of |G| + eps: a small update is like small rows of a larger one."""
    u = updates(1, m, n)[0]
    u *= norm / torch.linalg.vector_norm(u)
    got = rb.Orthogonalizer(m, n, coefficients=FIVE, eps=1e-7).orthogonalize(u).double()
    want = iteration(u, torch.float64, FIVE)
    size = torch.linalg.vector_norm(want, dim=1)
    off = torch.linalg.vector_norm(got - want, dim=1) / size
    plain = (torch.linalg.vector_norm(iteration(u, torch.float32, FIVE) - want, dim=1) / size).max()
    r = torch.linalg.vector_norm(u.double(), dim=1) / (torch.linalg.vector_norm(u.double()) + 1e-7)
    assert (off <= 4.0 * plain + 2.0 ** -36 * (n ** 0.5 + 64) / r).all()
