"""Plain statements in 64 bits (numpy) of what include/rb_train.h computes, and bounds on what binary32 may be off by."""
import numpy as np
import torch


def to64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def score(z, tokens, top):
    """Scores of rows z [rows, vocab] (float64), as rb_train.h defines them: dict of arrays."""
    rows, vocab = z.shape
    out = {"logp": np.zeros(tokens.shape), "lse": np.zeros(rows), "entropy": np.zeros(rows), "top_logp": np.zeros((rows, top)),
           "top_ids": np.zeros((rows, top), dtype=np.int64), "spread": np.zeros(rows)}
    for i in range(rows):
        r = z[i]
        there = (tokens[i] >= 0) & (tokens[i] < vocab)
        ids = np.argsort(-r, kind="stable")[:top] if not np.isnan(r).any() else np.zeros(top, dtype=np.int64)
        if np.isnan(r).any() or np.isposinf(r).any():
            out["lse"][i] = out["entropy"][i] = out["spread"][i] = np.nan
            out["logp"][i] = np.where(there, np.nan, 0.0)
            out["top_logp"][i], out["top_ids"][i] = np.nan, -1
            continue
        m = r.max()
        if np.isneginf(m):
            out["lse"][i], out["logp"][i], out["top_logp"][i], out["top_ids"][i] = -np.inf, np.where(there, -np.inf, 0.0), -np.inf, ids
            continue
        e = np.exp(r - m)
        s = e.sum()
        lse = m + np.log(s)
        live = e > 0
        out["lse"][i] = lse
        out["entropy"][i] = np.log(s) - (e[live] * (r[live] - m)).sum() / s
        out["spread"][i] = np.log(s)
        out["logp"][i] = np.where(there, r[np.where(there, tokens[i], 0)] - lse, 0.0)
        out["top_logp"][i], out["top_ids"][i] = r[ids] - lse, ids
    return out


def score_bounds(ref):
    """What the binary32 results may be off by.  A term e^(z-m) is off by its argument's rounding (|z-m| 2^-23: two roundings, times ln 2 log2 e) and
    the exponential's (2^-23); s is off by the terms' average of that - |z-m| weighted by probability is at most entropy - and by
    the sums' roundings (32 in a tile, one per tile, 8 joins: under 128 of 2^-24 for the rows here).  64 2^-23 (1 + entropy) covers these."""
    u = 2.0 ** -23
    h = np.nan_to_num(ref["entropy"], nan=0.0, posinf=0.0, neginf=0.0)
    base = 64 * u * (1 + h)
    lse = np.nan_to_num(ref["lse"], nan=0.0, posinf=0.0, neginf=0.0)
    at = base + 2 * u * (np.abs(lse) + np.nan_to_num(ref["spread"]))
    def wide(v):
        return at[:, None] + u * np.abs(np.nan_to_num(v, nan=0.0, posinf=0.0, neginf=0.0))
    return {"lse": at, "entropy": base * (2 + h), "logp": wide(ref["logp"]), "top_logp": wide(ref["top_logp"])}


def grad(z, tokens, lse, entropy, grad_logp, grad_entropy):
    """The gradient by its formula, from given lse and entropy; and its bound for binary32 results: the exponential's argument is off by
    |log p| 2^-23, the factors by some 2^-23."""
    rows, vocab = z.shape
    out, off = np.zeros_like(z), np.zeros_like(z)
    u = 2.0 ** -23
    for i in range(rows):
        if np.isneginf(lse[i]):
            continue
        there = (tokens[i] >= 0) & (tokens[i] < vocab)
        w = np.where(there, grad_logp[i], 0.0)
        with np.errstate(invalid="ignore"):
            logp = z[i] - lse[i]
        p = np.exp(logp)
        finite = np.where(np.isneginf(logp), 0.0, logp)
        h = 0.0 if grad_entropy is None else grad_entropy[i]
        inner = w.sum() + (0.0 if grad_entropy is None else h * (finite + entropy[i]))
        size = np.abs(w).sum() + abs(h) * (np.abs(finite) + (0.0 if grad_entropy is None else abs(entropy[i])))
        out[i] = -p * inner
        off[i] = p * size * u * (8 + 2 * np.abs(finite)) + 2.0 ** -140
        for g in range(tokens.shape[1]):
            if there[g]:
                out[i, tokens[i, g]] += w[g]
                off[i, tokens[i, g]] += 64 * u * np.abs(w).sum()
    return out, off


def orthogonal(g, coefficients, eps):
    """One matrix, as the definition reads."""
    tall = g.shape[0] > g.shape[1]
    x = g.T if tall else g
    norm = np.sqrt((x * x).sum()) + eps
    x = x / norm if norm > 0 else x * 0.0
    for a, b, c in coefficients:
        p = x @ x.T
        x = a * x + (b * p + c * p @ p) @ x
    return x.T if tall else x


def orthogonal_bound(coefficients):
    """Error of the result over the result's norm: in every step operands of 22 bits and binary32 sums put in some 2^-20 of the norm, and
    every later step may multiply that by the steepest of its polynomial on [0, 1.3] - |a|, or where the slope is steeper - so the whole is
    2^-20 times the sum of the products of the slopes."""
    total, growth = 0.0, 1.0
    s = np.linspace(0, 1.3, 400)
    for a, b, c in reversed(coefficients):
        total += growth
        growth *= np.abs(a + 3 * b * s ** 2 + 5 * c * s ** 4)[s <= 1.25].max()
    return 2.0 ** -20 * (total + growth)
