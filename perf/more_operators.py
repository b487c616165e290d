"""The operators between the matrix products of a block that is trained on the augmented mini-batch, as measurable cases.

  norm         layer norm of rows, alone or of the sum of a residual row and a row that went through dropout; that sum is an output too
  norm_grad    its gradients: of the sum, of what went through dropout, of weight and bias
  drop         dropout from a counter-based generator: the mask is a function of (seed, step, row, column)
  attend       attention of packed documents (fresh and rehearsed sequences behind one another): a position sees its own document, of that what is
               not behind it (causal) and the document's prefix; scores may be capped by a tanh and lowered with distance
  attend_grad  its gradients

`run` with `own` false states each in elementary operations in binary32; with `own` true it makes the calls that a training program makes of the
framework.  Positions that belong to no document get results and gradients of 0 and a log-sum of -inf.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5
SEED, STEP = 0x1234567890ABCDEF, (3 << 32) + 17        # of the dropout's generator


def _norm(name, op, rows, width, dtype, weights, residual=False, p=0.0, bias=True):
    return {"name": name, "op": op, "rows": rows, "width": width, "dtype": dtype, "weights": weights, "residual": residual, "p": p, "bias": bias}


def _drop(name, rows, width, dtype, p, pad=0):
    return {"name": name, "op": "drop", "rows": rows, "width": width, "dtype": dtype, "p": p, "pad": pad}


def _attend(name, op, tokens, docs, heads, kv_heads, dim, causal=True, cap=0.0, slopes=False, prefix=False, gaps=False):
    return {"name": name, "op": op, "tokens": tokens, "docs": docs, "heads": heads, "kv_heads": kv_heads, "dim": dim, "causal": causal, "cap": cap,
            "slopes": slopes, "prefix": prefix, "gaps": gaps}


def listed():
    return [
        # one token's row in an evaluation: nothing but latency
        _norm("norm_one_row", "norm", 1, 4096, "bf16", "f32"),
        # 4096 fresh + 1024 rehearsed feature rows, all in binary32
        _norm("norm_features", "norm", 5120, 2048, "f32", "f32"),
        # the sum of the residual stream and a dropped-out branch, normalised, for a large mini-batch
        _norm("norm_residual", "norm", 8192, 8192, "bf16", "f32", residual=True, p=0.1),
        # the gradient in a small hidden layer: 96 fresh + 32 rehearsed rows
        _norm("norm_grad_small", "norm_grad", 128, 192, "f32", "f32", residual=True, p=0.1),
        # the gradient for a large mini-batch, weights and bias among it
        _norm("norm_grad_large", "norm_grad", 16384, 4096, "bf16", "f32", residual=True, p=0.1),
        # dropout of the small hidden layer: latency
        _drop("drop_small", 128, 192, "f32", 0.1),
        # dropout of odd rows that lie apart
        _drop("drop_odd", 8191, 10007, "bf16", 0.2, pad=9),
        # a handful of short sequences: latency
        _attend("attend_short", "attend", 160, 9, 4, 4, 64),
        # fresh and rehearsed sequences of any length, packed
        _attend("attend_packed", "attend", 8192, 24, 16, 8, 128),
        # one long document, capped scores
        _attend("attend_long", "attend", 16384, 1, 8, 4, 128, cap=30.0),
        # the gradient for prompts that are seen whole, in a padded batch, scores lowered with distance, eight heads to one of keys and values
        _attend("attend_grad_packed", "attend_grad", 8000, 40, 16, 2, 64, slopes=True, prefix=True, gaps=True),
        # the gradient of a long document
        _attend("attend_grad_long", "attend_grad", 8192, 1, 16, 8, 128),
    ]


def _log_between(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(("norm", "norm_grad", "drop", "attend", "attend_grad"))
    if op in ("norm", "norm_grad"):
        width = _log_between(rng, 32, 16384)
        rows = _log_between(rng, 1, min(65536, (1 << 26) // width))
        residual = rng.random() < 0.6
        case = _norm("", op, rows, width, rng.choice(("f32", "bf16")), rng.choice(("f32", "bf16")), residual, rng.choice((0.0, 0.1, 0.5)) if residual else 0.0,
                     rng.random() < 0.7)
    elif op == "drop":
        width = _log_between(rng, 32, 16384)
        case = _drop("", _log_between(rng, 1, min(65536, (1 << 26) // width)), width, rng.choice(("f32", "bf16")), rng.choice((0.1, 0.25, 0.5)), rng.choice((0, 0, 1, 8)))
    else:
        tokens = _log_between(rng, 1, 16384 if op == "attend" else 8192)
        docs = _log_between(rng, 1, min(64, tokens))
        kv = rng.choice((1, 2, 3, 4, 8))
        case = _attend("", op, tokens, docs, kv * rng.choice((1, 1, 2, 4)), kv, rng.choice((16, 32, 64, 64, 72, 128, 128)), rng.random() < 0.8,
                       rng.choice((0.0, 0.0, 30.0)), rng.random() < 0.3, rng.random() < 0.3, rng.random() < 0.3)
        largest = max(work(c)["flops"] for c in listed() if c["op"] == op)
        longest = max(_documents(case)[1])
        if work(case)["flops"] > largest or docs * longest * longest * case["heads"] > 1 << 31:      # as many heads as are paid for
            case["kv_heads"] = case["heads"] = 1
    return {k: v for k, v in case.items() if k != "name"}


def _documents(case):
    """(begins, lengths, prefixes) of a case's documents, and where the last one ends: of the case alone."""
    tokens, docs = case["tokens"], case["docs"]
    rng = random.Random(tokens * 1000 + docs)
    last = tokens - tokens // 50 if docs > 1 else tokens                       # a few positions behind the last document
    cuts = sorted(rng.randrange(0, last + 1) for _ in range(docs - 1))         # (some documents may be empty)
    ends = [*cuts, last]
    begins = [0, *cuts]
    lengths = [e - b for b, e in zip(begins, ends)]
    if case["gaps"]:
        lengths = [n - rng.randrange(0, n // 3 + 1) for n in lengths]
    prefixes = [rng.randrange(0, n // 2 + 1) for n in lengths]
    return begins, lengths, prefixes, last


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _inputs(case, seed):
    """The tensors of a case, from the seed alone."""
    g = _generator(seed)

    def normal(*shape, dtype="f32", scale=1.0, mean=0.0):
        return torch.empty(shape, dtype=DTYPES[dtype], device="cuda").normal_(mean, scale, generator=g)

    op = case["op"]
    if op in ("norm", "norm_grad"):
        rows, width, dtype = case["rows"], case["width"], case["dtype"]
        # a residual stream grows with depth and has a mean that is not 0
        s = {"weight": normal(width, dtype=case["weights"], scale=0.2, mean=1.0), "bias": normal(width, dtype=case["weights"], scale=0.1) if case["bias"] else None}
        if op == "norm":
            s["x"] = normal(rows, width, dtype=dtype, mean=0.3)
            s["residual"] = normal(rows, width, dtype=dtype, scale=4.0, mean=-0.5) if case["residual"] else None
            return s
        s["total"] = normal(rows, width, dtype=dtype, scale=4.0, mean=-0.5)
        s["grad_y"] = normal(rows, width, dtype=dtype, scale=1e-2)
        s["grad_total"] = normal(rows, width, dtype=dtype, scale=1e-2) if case["residual"] else None
        return s
    if op == "drop":
        return {"x": normal(case["rows"], case["width"] + case["pad"], dtype=case["dtype"])[:, :case["width"]]}
    heads, kv, dim, tokens = case["heads"], case["kv_heads"], case["dim"], case["tokens"]
    # one product's output holds queries, keys and values
    def split(t):
        return (t[:, :heads * dim].view(tokens, heads, dim), t[:, heads * dim:(heads + kv) * dim].view(tokens, kv, dim),
                t[:, (heads + kv) * dim:].view(tokens, kv, dim))
    q, k, v = split(normal(tokens, (heads + 2 * kv) * dim, dtype="bf16", scale=1.3))
    s = {"q": q, "k": k, "v": v, "slopes": None}
    if case["slopes"]:
        s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)], device="cuda")
    begins, lengths, prefixes, last = _documents(case)
    s["offsets"] = torch.tensor([*begins, last], dtype=torch.int64, device="cuda")
    s["lengths"] = torch.tensor(lengths, dtype=torch.int64, device="cuda") if case["gaps"] else None
    s["prefixes"] = torch.tensor(prefixes, dtype=torch.int64, device="cuda") if case["prefix"] else None
    if op == "attend_grad":
        s["grad_out"] = normal(tokens, heads, dim, dtype="bf16", scale=1e-2)
        s["grads"] = split(torch.empty((tokens, (heads + 2 * kv) * dim), dtype=torch.bfloat16, device="cuda"))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    op = case["op"]
    if op == "norm_grad":               # the forward pass has been made: its statistics are at hand
        s["mean"], s["rstd"] = _row_statistics(s["total"].float())
    if op in ("attend", "attend_grad"):
        begins, lengths, _, _ = _documents(case)
        s["longest"] = max(lengths)
        s["begins"] = torch.tensor(begins, device="cuda")
        if op == "attend_grad":         # ... and its output
            done = _plain_attend(s)
            s["out"], s["lse"] = done["out"], done["lse"]
    if own:
        import paper_2406_03285_amd as rb
        if op in ("norm", "norm_grad"):
            s["norm"] = rb.LayerNorm(case["width"], DTYPES[case["dtype"]], weight_dtype=DTYPES[case["weights"]], eps=EPS)
            s["drop"] = rb.Drop(case["p"], SEED, STEP) if case["p"] else None
            s["into"] = s["norm"].outputs(case["rows"], total=case["residual"]) if op == "norm" else \
                s["norm"].gradients(case["rows"], bias=case["bias"], drop=s["drop"] is not None)
        elif op == "drop":
            s["drop"], s["into"] = rb.Drop(case["p"], SEED, STEP), torch.empty_strided(s["x"].shape, s["x"].stride(), dtype=s["x"].dtype, device="cuda")
        else:
            s["attention"] = rb.DocumentAttention(case["heads"], case["dim"], kv_heads=case["kv_heads"], max_tokens=case["tokens"], causal=case["causal"], cap=case["cap"])
            s["documents"] = rb.Documents(s["offsets"], s["lengths"], s["prefixes"])
            s["into"] = s["attention"].outputs(case["tokens"]) if op == "attend" else None
    return s


def run(state):
    case = state["case"]
    op = case["op"]
    if not own:
        return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "drop": _plain_drop, "attend": _plain_attend, "attend_grad": _plain_attend_grad}[op](state)
    if op == "norm":
        o = state["norm"].forward(state["x"], state["weight"], state["bias"], residual=state["residual"], drop=state["drop"], out=state["into"])
        return {"y": o.y, "total": o.total, "mean": o.mean, "rstd": o.rstd}
    if op == "norm_grad":
        g = state["norm"].grad(state["grad_y"], state["total"], state["weight"], state["mean"], state["rstd"], grad_total=state["grad_total"],
                               drop=state["drop"], bias=case["bias"], out=state["into"])
        return {"total": g.total, "x": g.x, "weight": g.weight, "bias": g.bias}
    if op == "drop":
        import paper_2406_03285_amd as rb
        return {"y": rb.dropout(state["x"], state["drop"], out=state["into"])}
    if op == "attend":
        o = state["attention"].forward(state["q"], state["k"], state["v"], state["documents"], slopes=state["slopes"], out=state["into"])
        return {"out": o.out, "lse": o.lse}
    g = state["attention"].grad(state["q"], state["k"], state["v"], state["documents"], state["out"], state["lse"], state["grad_out"], slopes=state["slopes"],
                                out=state["grads"])
    return {"q": g[0], "k": g[1], "v": g[2]}


# ---- plain forms ---------------------------------------------------------------

def _multiple(a, x):
    """The two halves of the 64-bit product of 32-bit numbers."""
    y = a * x                          # (wraps; the bits are those of the product)
    return (y >> 32) & 0xFFFFFFFF, y & 0xFFFFFFFF


def _kept(rows, width, p):
    """Which elements dropout keeps, and what these are multiplied by: an element's 16 bits are a piece of Philox4x32-10's output for its row and its
    group of eight columns; p is held in 16 bits."""
    least = int(round(p * 65536))
    row = torch.arange(rows, device="cuda", dtype=torch.int64)[:, None].expand(rows, (width + 7) // 8)
    group = torch.arange((width + 7) // 8, device="cuda", dtype=torch.int64)[None, :].expand(rows, (width + 7) // 8)
    x = [row, group + 0x80000000, torch.full_like(row, STEP & 0xFFFFFFFF), torch.full_like(row, STEP >> 32)]
    ka, kb = SEED & 0xFFFFFFFF, SEED >> 32
    for _ in range(10):
        ah, al = _multiple(0xD2511F53, x[0])
        bh, bl = _multiple(0xCD9E8D57, x[2])
        x = [bh ^ x[1] ^ ka, bl, ah ^ x[3] ^ kb, al]
        ka, kb = (ka + 0x9E3779B9) & 0xFFFFFFFF, (kb + 0xBB67AE85) & 0xFFFFFFFF
    halves = torch.stack([h for w in x for h in (w & 0xFFFF, w >> 16)], 2).reshape(rows, -1)[:, :width]
    return halves >= least, 65536.0 / (65536 - least)


def _through_dropout(x, p):
    keep, scale = _kept(*x.shape, p)
    return torch.where(keep, x * scale, 0.0)


def _row_statistics(t):
    mean = t.mean(1)
    return mean, 1.0 / ((t - mean[:, None]).square().mean(1) + EPS).sqrt()


def _plain_norm(state):
    case = state["case"]
    total, kept = state["x"].float(), None
    if case["residual"]:
        if case["p"]:
            total = _through_dropout(total, case["p"])
        kept = (state["residual"].float() + total).to(state["x"].dtype)       # the row that the statistics are of
        total = kept.float()
    mean, rstd = _row_statistics(total)
    y = (total - mean[:, None]) * rstd[:, None] * state["weight"].float()
    if state["bias"] is not None:
        y = y + state["bias"].float()
    return {"y": y.to(state["x"].dtype), "total": kept, "mean": mean, "rstd": rstd}


def _plain_norm_grad(state):
    case, dtype, weights = state["case"], state["total"].dtype, state["weight"].dtype
    gy, rstd = state["grad_y"].float(), state["rstd"][:, None]
    hat = (state["total"].float() - state["mean"][:, None]) * rstd
    g = gy * state["weight"].float()
    total = rstd * (g - g.mean(1, keepdim=True) - hat * (g * hat).mean(1, keepdim=True))
    if state["grad_total"] is not None:
        total = total + state["grad_total"].float()
    return {"total": total.to(dtype), "x": _through_dropout(total, case["p"]).to(dtype) if case["p"] else None, "weight": (gy * hat).sum(0).to(weights),
            "bias": gy.sum(0).to(weights) if case["bias"] else None}


def _plain_drop(state):
    return {"y": _through_dropout(state["x"].float(), state["case"]["p"]).to(state["x"].dtype)}


def _rows_of_documents(state):
    """Places [docs, longest] of every document's positions and whether they are there; the first of them to be used where not."""
    at = torch.arange(state["longest"], device="cuda")
    lengths = state["lengths"] if state["lengths"] is not None else state["offsets"][1:] - state["offsets"][:-1]
    there = at[None] < lengths[:, None]
    return torch.where(there, state["begins"][:, None] + at, 0), there


def _by_document(x, places, heads):
    """[tokens, some heads, dim] -> [docs, heads, longest, dim] in binary32."""
    x = x[places].float().transpose(1, 2)
    return x.repeat_interleave(heads // x.shape[1], 1).contiguous()


def _scores(state, q, k, there):
    """Scores [docs, heads, longest, longest], -inf where a position is not seen; and the derivative of the cap."""
    case = state["case"]
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(case["dim"]))
    slope = None
    if case["cap"]:
        t = torch.tanh(s / case["cap"])
        s, slope = case["cap"] * t, 1.0 - t * t
    at = torch.arange(state["longest"], device="cuda")
    if state["slopes"] is not None:
        s = s - state["slopes"][:, None, None] * (at[:, None] - at[None]).abs()
    seen = there[:, None, :, None] & there[:, None, None, :]
    if case["causal"]:
        before = (at[None] <= at[:, None])[None]
        if state["prefixes"] is not None:
            before = before | (at[None, None, :] < state["prefixes"][:, None, None])
        seen = seen & before[:, None]
    return s.masked_fill(~seen, -math.inf), slope


def _plain_attend(state):
    case = state["case"]
    places, there = _rows_of_documents(state)
    q, k, v = (_by_document(state[n], places, case["heads"]) for n in ("q", "k", "v"))
    s, _ = _scores(state, q, k, there)
    m = s.amax(3, keepdim=True).clamp(min=-1e30)
    e = (s - m).exp()
    z = e.sum(3, keepdim=True)
    o = torch.matmul(e, v) / z
    out = torch.zeros((case["tokens"], case["heads"], case["dim"]), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((case["tokens"], case["heads"]), -math.inf, device="cuda")
    out[places[there]] = o.transpose(1, 2)[there].to(torch.bfloat16)
    lse[places[there]] = (m + z.log())[..., 0].transpose(1, 2)[there]
    return {"out": out, "lse": lse.t().contiguous()}


def _plain_attend_grad(state):
    case, heads, kv = state["case"], state["case"]["heads"], state["case"]["kv_heads"]
    places, there = _rows_of_documents(state)
    q, k, v, do = (_by_document(state[n], places, heads) for n in ("q", "k", "v", "grad_out"))
    s, slope = _scores(state, q, k, there)
    lse = state["lse"].t()[places].transpose(1, 2)[..., None]
    p = (s - lse.clamp(min=-1e30)).exp()
    p = torch.where(there[:, None, :, None], p, 0.0)
    do = torch.where(there[:, None, :, None], do, 0.0)
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    dp = torch.matmul(do, v.transpose(2, 3).contiguous())
    ds = p * (dp - (p * dp).sum(3, keepdim=True)) * (1.0 / math.sqrt(case["dim"]))
    if slope is not None:
        ds = ds * slope
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q)
    got = []
    for x, n in ((dq, heads), (dk, kv), (dv, kv)):
        x = x.unflatten(1, (n, heads // n)).sum(2)
        full = torch.zeros((case["tokens"], n, case["dim"]), dtype=torch.bfloat16, device="cuda")
        full[places[there]] = x.transpose(1, 2)[there].to(torch.bfloat16)
        got.append(full)
    return {"q": got[0], "k": got[1], "v": got[2]}


# ---- work ----------------------------------------------------------------------

def _pairs(case):
    """How many pairs of positions a head has to look at."""
    _, lengths, prefixes, _ = _documents(case)
    if not case["causal"]:
        return sum(n * n for n in lengths)
    if not case["prefix"]:
        prefixes = [0] * len(lengths)
    return sum(n * (n + 1) // 2 + p * (p - 1) // 2 for n, p in zip(lengths, prefixes))


def work(case):
    op = case["op"]
    if op in ("norm", "norm_grad", "drop"):
        elems, size = case["rows"] * case["width"], DTYPES[case["dtype"]].itemsize
        if op == "drop":
            return {"bytes": 2.0 * elems * size, "flops": 2.0 * elems}
        weights = case["width"] * DTYPES[case["weights"]].itemsize * (2 if case["bias"] else 1)
        if op == "norm":        # the row (and the residual one, and their sum), the result, the statistics
            return {"bytes": (4.0 if case["residual"] else 2.0) * elems * size + weights + 8 * case["rows"], "flops": 8.0 * elems}
        # the row, the gradient that arrives (both of them), the gradient of the sum, that of what went through dropout
        return {"bytes": (3.0 + case["residual"] + (case["p"] > 0)) * elems * size + 2.0 * weights + 8 * case["rows"], "flops": 14.0 * elems}
    row = case["dim"] * 2.0
    products, rows = (2, 2 * case["heads"] + 2 * case["kv_heads"]) if op == "attend" else (5, 4 * case["heads"] + 4 * case["kv_heads"])
    return {"bytes": case["tokens"] * (rows * row + 4 * case["heads"]), "flops": 2.0 * products * case["dim"] * case["heads"] * _pairs(case)}


# ---- in 64 bits ----------------------------------------------------------------

def _kept_exact(rows, width, p):
    """The same mask from Philox4x32-10's definition on the host."""
    mask, groups = np.uint64(0xFFFFFFFF), -(-width // 8)
    words = np.empty((4, rows, groups), dtype=np.uint64)
    words[0] = np.arange(rows, dtype=np.uint64)[:, None]
    words[1] = np.arange(groups, dtype=np.uint64)[None] | np.uint64(1 << 31)
    words[2], words[3] = STEP % 2 ** 32, STEP // 2 ** 32
    key = [SEED % 2 ** 32, SEED // 2 ** 32]
    for n in range(10):
        left, right = words[0] * np.uint64(0xD2511F53), words[2] * np.uint64(0xCD9E8D57)
        k = [np.uint64((key[0] + n * 0x9E3779B9) % 2 ** 32), np.uint64((key[1] + n * 0xBB67AE85) % 2 ** 32)]
        words = np.stack([(right >> np.uint64(32)) ^ words[1] ^ k[0], right & mask, (left >> np.uint64(32)) ^ words[3] ^ k[1], left & mask])
    bits = np.ascontiguousarray(words.transpose(1, 2, 0).astype("<u4")).view("<u2").reshape(rows, groups * 8)[:, :width]
    least = int(round(p * 65536))
    return torch.from_numpy(bits >= least).cuda(), 1.0 / (1.0 - least / 65536.0)


def _dropped_exact(x, p):
    if not p:
        return x
    keep, scale = _kept_exact(*x.shape, p)
    return x * keep * scale


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "drop":
        return {"y": _dropped_exact(s["x"].double(), case["p"])}
    if op in ("norm", "norm_grad"):
        weight = s["weight"].double()
        if op == "norm":
            total = s["x"].double()
            if case["residual"]:
                total = s["residual"].double() + _dropped_exact(total, case["p"])
            of = total.to(s["x"].dtype).double()
        else:
            of = s["total"].double()
        var, mean = torch.var_mean(of, 1, correction=0)
        rstd = torch.rsqrt(var + EPS)
        hat = (of - mean[:, None]) * rstd[:, None]
        if op == "norm":
            return {"y": hat * weight + (s["bias"].double() if case["bias"] else 0.0), "total": total if case["residual"] else None, "mean": mean, "rstd": rstd}
        gy, n = s["grad_y"].double(), case["width"]
        # the projection of g / deviation away from the two directions that the normalisation takes out
        g = gy * weight
        g = g - g.sum(1, keepdim=True) / n - hat * ((g * hat).sum(1, keepdim=True) / n)
        g = g * rstd[:, None] + (s["grad_total"].double() if case["residual"] else 0.0)
        return {"total": g, "x": _dropped_exact(g, case["p"]) if case["p"] else None, "weight": torch.einsum("rc,rc->c", gy, hat),
                "bias": gy.sum(0) if case["bias"] else None}
    return _exact_attend(case, s)


def _exact_attend(case, s):
    """Document by document, a few heads at a time; gradients by differentiation."""
    heads, group, tokens, dim = case["heads"], case["heads"] // case["kv_heads"], case["tokens"], case["dim"]
    grads = case["op"] == "attend_grad"
    out = torch.zeros((tokens, heads, dim), dtype=torch.float64, device="cuda")
    lse = torch.full((heads, tokens), -math.inf, dtype=torch.float64, device="cuda")
    found = {n: torch.zeros(s[n].shape, dtype=torch.float64, device="cuda") for n in ("q", "k", "v")}
    for begin, length, prefix in zip(*_documents(case)[:3]):
        if not length:
            continue
        at, i = slice(begin, begin + length), torch.arange(length, device="cuda")
        seen = torch.ones((length, length), dtype=torch.bool, device="cuda")
        if case["causal"]:
            seen = (i[:, None] >= i[None]) | (i[None] < (prefix if case["prefix"] else 0))
        most = max(1, (1 << 27) // (length * length))
        for h in range(0, heads, most):
            hs = list(range(h, min(heads, h + most)))
            of = [x // group for x in hs]
            q, k, v = (s[n][at][:, c].double().transpose(0, 1).contiguous().requires_grad_(grads) for n, c in (("q", hs), ("k", of), ("v", of)))
            z = torch.bmm(q, k.transpose(1, 2).contiguous()) / math.sqrt(dim)
            if case["cap"]:
                z = case["cap"] * torch.tanh(z / case["cap"])
            if case["slopes"]:
                z = z - s["slopes"][hs].double()[:, None, None] * (i[:, None] - i[None]).abs()
            z = torch.where(seen, z, -math.inf)
            o = torch.bmm(torch.softmax(z, 2), v)
            if not grads:
                out[at, hs], lse[hs, at] = o.transpose(0, 1), torch.logsumexp(z, 2)
                continue
            d = torch.autograd.grad(o, (q, k, v), s["grad_out"][at][:, hs].double().transpose(0, 1))
            for n, c, x in zip(("q", "k", "v"), (hs, of, of), d):
                found[n][at] = found[n][at].index_add(1, torch.tensor(c, device="cuda"), x.transpose(0, 1))
    return found if grads else {"out": out, "lse": lse}
