"""Plain statements in 64 bits of what include/rb_block.h computes, and bounds on what the results may be off by."""
import numpy as np
import torch

BF16_HALF, F32_HALF = 2.0 ** -8, 2.0 ** -24        # half a step, relative to the value
HALF = {torch.float32: F32_HALF, torch.bfloat16: BF16_HALF}


def to64(t):
    return None if t is None else t.detach().cpu().to(torch.float64)


# ---- dropout -------------------------------------------------------------------

def philox(counter, key):
    """Philox4x32-10 as published, on whole arrays of counters."""
    x = [np.asarray(c, dtype=np.uint64) for c in counter]
    k0, k1 = key
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(b >> np.uint64(32)) ^ x[1] ^ np.uint64(k0), b & low, (a >> np.uint64(32)) ^ x[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) % 2 ** 32, (k1 + 0xBB67AE85) % 2 ** 32
    return x


def kept(rows, width, drop):
    """The factor of every element: 0 or the scale."""
    least = round(drop.p * 65536)
    j, i = np.meshgrid(np.arange(width), np.arange(rows))
    seed, step = drop.seed % 2 ** 64, drop.step % 2 ** 64
    words = philox([i, 2 ** 31 + j // 8, np.full_like(i, step % 2 ** 32), np.full_like(i, step >> 32)], (seed % 2 ** 32, seed >> 32))
    word = np.choose(j % 8 // 2, words)
    half = (word >> (16 * (j % 2)).astype(np.uint64)) & np.uint64(0xFFFF)
    scale = 0.0 if least == 65536 else float(np.float32(65536.0 / (65536 - least)))
    return torch.from_numpy(np.where(half >= least, scale, 0.0))


def drop(x, d):
    if d is None:
        return x
    f = kept(*x.shape, d)
    return torch.where(f > 0, x * f, torch.zeros_like(x))


# ---- layer norm ------------------------------------------------------------------

def norm(total, weight, bias, eps):
    """(y, mean, rstd) of rows."""
    mean = total.mean(1)
    var = (total - mean[:, None]).square().mean(1)
    rstd = 1.0 / torch.sqrt(var + eps)
    y = (total - mean[:, None]) * rstd[:, None] * weight
    return (y if bias is None else y + bias), mean, rstd


def norm_bounds(total, weight, bias, eps, dtype):
    """Of y, mean, rstd.  The mean is a sum of at most 64 numbers in a lane, 10 steps between lanes, two products: under 80 half steps of the mean size of its terms -
    and what it is off by is summed a second time, over the differences, so that 3 half steps of the mean itself and 80 of the deviation's half steps stay.
    The sum of squares is off by 80 half steps and 3 of its terms; h by the mean's error over the deviation, rstd's and three roundings."""
    u = F32_HALF
    mean = total.mean(1).abs()
    spread = (total - total.mean(1, keepdim=True)).abs().mean(1)
    _, _, rstd = norm(total, weight, bias, eps)
    off_mean = 4 * u * mean + 100 * u * spread + 1e-40
    rel_rstd = 60 * u + off_mean.square() * rstd.square() + 4 * u * mean * rstd       # (differences are rounded to half a step of the numbers subtracted)
    h = ((total - total.mean(1, keepdim=True)) * rstd[:, None]).abs()
    off_h = h * (rel_rstd[:, None] + 4 * u) + (off_mean * rstd)[:, None] + 2 * u * (total.abs() + mean[:, None]) * rstd[:, None]
    y = (h * weight).abs() + (0 if bias is None else bias.abs())
    return off_h * weight.abs() + y * (2 * u + HALF[dtype]), off_mean, rstd * rel_rstd


def norm_grad(grad_y, total, grad_total, mean, rstd, weight):
    """(of the sum, of weight, of bias) by the formula, from given statistics."""
    h = (total - mean[:, None]) * rstd[:, None]
    g = grad_y * weight
    d = rstd[:, None] * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    return (d if grad_total is None else d + grad_total), (grad_y * h).sum(0), grad_y.sum(0)


def norm_grad_bounds(grad_y, total, grad_total, mean, rstd, weight, dtype, weight_dtype):
    """h is off by 3 half steps of itself and of what is subtracted; a row's sums by 100 half steps of their terms' sizes; the weights' sums have one term a
    row in a workgroup (rows / 512 or all, 512 at most behind each other in the join, 16 rows): rows + 64 half steps of the terms' sizes."""
    u = F32_HALF
    rows = total.shape[0]
    h = ((total - mean[:, None]) * rstd[:, None]).abs()
    off_h = 3 * u * h + u * (total.abs() + mean.abs()[:, None]) * rstd[:, None]
    g = (grad_y * weight).abs()
    c0, c1 = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    off_c1 = 100 * u * c1 + (g * off_h).mean(1, keepdim=True)
    d = rstd[:, None] * (g + c0 + h * c1)
    off = rstd[:, None] * (100 * u * c0 + h * off_c1 + off_h * c1) + 6 * u * d
    exact, _, _ = norm_grad(grad_y, total, grad_total, mean, rstd, weight)
    off = off + exact.abs() * HALF[dtype] + (0 if grad_total is None else 2 * u * grad_total.abs())
    many = (min(rows, 1200) + 64) * u
    gw = (grad_y.abs() * h).sum(0) * many + (grad_y.abs() * off_h).sum(0)
    gb = grad_y.abs().sum(0) * many
    w = HALF[weight_dtype]
    return off, gw * (1 + w) + (grad_y * (total - mean[:, None]) * rstd[:, None]).sum(0).abs() * w, gb * (1 + w) + grad_y.sum(0).abs() * w


# ---- attention -------------------------------------------------------------------

def seen(tokens, offsets, lengths=None, prefixes=None, causal=True):
    """[tokens, tokens]: whether position i sees position j."""
    m = torch.zeros((tokens, tokens), dtype=torch.bool)
    for d in range(len(offsets) - 1):
        begin, end = offsets[d], offsets[d + 1]
        if lengths is not None:
            end = min(end, begin + lengths[d])
        prefix = begin + min(prefixes[d], end - begin) if prefixes is not None and end > begin else begin
        for i in range(begin, end):
            m[i, begin:end] = True
            if causal:
                m[i, max(i + 1, prefix):end] = False
    return m


def scores(q, k, scale, cap, slopes, mask):
    """[heads, tokens, tokens] of q, k [tokens, heads, dim] (as many heads each); the cap's slope; a bound on the scores' error: dim products summed in binary32,
    and some roundings of what comes of it."""
    u = F32_HALF
    p = torch.einsum("ihd,jhd->hij", q, k)
    size = torch.einsum("ihd,jhd->hij", q.abs(), k.abs())
    off = scale * size * (q.shape[2] + 4) * u
    s, slope = p * scale, torch.ones_like(p)
    if cap:
        t = torch.tanh(s / cap)
        s, slope = cap * t, 1 - t * t
        off = off + 8 * cap * u
    if slopes is not None:
        i = torch.arange(q.shape[0], dtype=torch.float64, device=q.device)
        b = slopes[:, None, None] * (i[:, None] - i[None]).abs()
        off = off + 4 * u * b.abs()
        s = s - b
    off = off + 6 * u * (s.abs() + 1)
    return torch.where(mask, s, -np.inf), slope, torch.where(mask, off, 0.0)


def spread(x, heads):
    return x.repeat_interleave(heads // x.shape[1], 1)


def attend(q, k, v, scale, cap, slopes, mask):
    """(out, lse) of the definition and their bounds."""
    u, heads, tokens = F32_HALF, q.shape[1], q.shape[0]
    k, v = spread(k, heads), spread(v, heads)
    s, _, off = scores(q, k, scale, cap, slopes, mask)
    lse = torch.logsumexp(s, 2)
    p = torch.where(mask, (s - torch.where(mask.any(1), lse, 0.0)[:, :, None]).exp(), 0.0)
    out = torch.einsum("hij,jhd->ihd", p, torch.where(mask.any(0)[:, None, None], v, 0.0))
    worst = off.amax(2) + (tokens + 16) * u
    size = torch.einsum("hij,jhd->ihd", p, torch.where(mask.any(0)[:, None, None], v.abs(), 0.0))
    off_out = size * (BF16_HALF + 2 * worst.t()[:, :, None] + (tokens + 16) * u) * (1 + BF16_HALF) + out.abs() * BF16_HALF
    return out, lse, off_out, 2 * worst + 8 * u * (torch.where(mask.any(1), lse, 0.0).abs() + 1)


def attend_grad(q, k, v, out, lse, grad_out, scale, cap, slopes, mask):
    """Gradients of q, k, v by the formula from given lse, and their bounds.  Out is where the sum of p dp begins: what that is off by (`away`) takes part in what is
    rounded on the way."""
    u, heads, tokens, dim = F32_HALF, q.shape[1], q.shape[0], q.shape[2]
    kv = k.shape[1]
    k, v = spread(k, heads), spread(v, heads)
    some = mask.any(1)[:, None, None]
    q, k, v, out, grad_out = (torch.where(some, x, 0.0) for x in (q, k, v, out, grad_out))
    s, slope, off_s = scores(q, k, scale, cap, slopes, mask)
    lse = torch.where(mask.any(1), lse, 0.0)
    p = torch.where(mask, (s - lse[:, :, None]).exp(), 0.0)
    # what is less than binary32's least normal number, 2^-126, may be 0: a weight, ds, and what they were rounded to
    least = torch.where(mask, 2.0 ** -126, 0.0)
    off_p = p * (2 * off_s + 4 * u * (lse.abs()[:, :, None] + 1)) + least
    dp, dp_size = torch.einsum("ihd,jhd->hij", grad_out, v), torch.einsum("ihd,jhd->hij", grad_out.abs(), v.abs())
    first, first_size = (grad_out * out).sum(2).t()[:, :, None], (grad_out * out).abs().sum(2).t()[:, :, None]
    # sum of p (dp - first) over what is seen, p as it was computed: the weights add up to 1 only within the bound of lse, which makes of `first` no more than that
    away = (p * (dp - first)).sum(2, keepdim=True)
    delta = first + away
    off_dp = (dim + 4) * u * (dp_size + first_size)
    off_delta = (off_p * (dp - first).abs() + p * off_dp + (tokens + 8) * u * p * (dp - first).abs()).sum(2, keepdim=True) + 4 * u * delta.abs()
    ds = p * (dp - delta) * slope
    # the cap's slope 1 - t^2 is off by some 2^-22 where it is of size 1, and by that much of 1 where it is small
    off_slope = 16 * u if cap else 0.0
    off_ds = off_p * (dp - delta).abs() * slope + p * slope * (off_dp + off_delta) + off_slope * p * (dp - delta).abs() + 4 * u * ds.abs()
    aside = p * away.abs() * slope                     # what is added to ds before it is rounded, and taken away again
    off_aside = (off_p * slope + off_slope * p) * away.abs() + 4 * u * aside
    def rounded(x, off):           # x was rounded to bfloat16
        return off * (1 + BF16_HALF) + x.abs() * BF16_HALF + least
    off_w = rounded(p, off_p)
    off_of_q = rounded(ds.abs() + aside, off_ds + off_aside) + rounded(aside, off_aside)
    off_of_k = rounded(ds, off_ds)
    # ... as the sum of what was rounded, which the roundings move by no more than all of them, times p k
    off_of_q = off_of_q + (1 + BF16_HALF) * rounded(p * slope, off_p * slope + off_slope * p + p * slope) * (rounded(ds.abs() + aside, off_ds + off_aside) - off_ds).sum(2, keepdim=True)
    many = (tokens * heads + 16) * u
    def joined(x):
        return x.unflatten(1, (kv, heads // kv)).sum(2)
    dq = torch.einsum("hij,jhd->ihd", ds, k) * scale
    dk = joined(torch.einsum("hij,ihd->jhd", ds, q)) * scale
    dv = joined(torch.einsum("hij,ihd->jhd", p, grad_out))
    b_q = torch.einsum("hij,jhd->ihd", off_of_q + many * (ds.abs() + 2 * aside), k.abs()) * scale
    b_k = joined(torch.einsum("hij,ihd->jhd", off_of_k + many * ds.abs(), q.abs())) * scale
    b_v = joined(torch.einsum("hij,ihd->jhd", off_w + many * p, grad_out.abs()))
    return (dq, dk, dv), tuple(b * (1 + BF16_HALF) + x.abs() * BF16_HALF * (1 + BF16_HALF) + 2.0 ** -130 for x, b in ((dq, b_q), (dk, b_k), (dv, b_v)))
