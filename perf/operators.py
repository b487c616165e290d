"""The operators of the training step that the rehearsal buffer feeds, as measurable cases.

  score   log probabilities of given tokens (or classes) under a row of logits, its entropy, its top alternatives
  grad    the gradient of those log probabilities and of the entropy with respect to the logits
  ortho   an update matrix orthogonalised by Newton-Schulz products
  step    the optimiser step around it: momentum, orthogonalised update, weight decay, weights

`run` with `own` false states each in elementary operations in binary32; with `own` true it makes the calls that a
training program makes of the framework.  In a step the weights and the momentum are the state's own tensors.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)      # of one Newton-Schulz step; five steps
STEPS = 5
EPS = 1e-7
LR, BETA, DECAY = 0.02, 0.95, 0.01


def _score(name, rows, vocab, dtype, given=1, top=0, pad=0, masked=0):
    return {"name": name, "op": "score", "rows": rows, "vocab": vocab, "dtype": dtype, "given": given, "top": top, "pad": pad, "masked": masked}


def _grad(name, rows, vocab, dtype, given=1, pad=0, masked=0, entropy=True):
    return {"name": name, "op": "grad", "rows": rows, "vocab": vocab, "dtype": dtype, "given": given, "pad": pad, "masked": masked, "entropy": entropy}


def _ortho(name, batch, m, n, dtype):
    return {"name": name, "op": "ortho", "batch": batch, "m": m, "n": n, "dtype": dtype}


def _step(name, batch, m, n, dtype, weights):
    return {"name": name, "op": "step", "batch": batch, "m": m, "n": n, "dtype": dtype, "weights": weights}


def listed():
    return [
        # serving: the log probability of one decoded token, with what else it might have been; nothing but latency
        _score("score_one_token", 1, 32000, "bf16", top=20),
        # 4096 fresh + 1024 rehearsed feature rows under a classifier of 10000 classes, the best five kept
        _score("score_classes", 5120, 10000, "f32", top=5),
        # what is stored beside 2048 tokens for later rehearsal: 16 alternatives each; odd vocabulary, rows without any alignment
        _score("score_alternatives", 2048, 50001, "bf16", top=16),
        # the loss of a large mini-batch over a large vocabulary padded at its end: 2.1 GB of logits read once
        _score("score_large", 8192, 131072, "bf16", masked=500),
        # the gradient for 512 fresh + 64 rehearsed images under 1000 classes: small
        _grad("grad_classes", 576, 1000, "f32"),
        # rehearsal of 1024 tokens against 16 stored alternatives and the token itself; odd vocabulary in padded rows
        _grad("grad_alternatives", 1024, 50001, "bf16", given=17, pad=47),
        # the gradient of the large mini-batch: 2.1 GB read, 2.1 GB written
        _grad("grad_large", 8192, 131072, "bf16", masked=500),
        # one small weight matrix: latency
        _ortho("ortho_small", 1, 128, 128, "f32"),
        # the same projection of 24 layers at once, odd sizes
        _ortho("ortho_layers", 24, 333, 200, "bf16"),
        # a large square projection
        _ortho("ortho_large", 1, 4096, 4096, "bf16"),
        # a hidden layer's whole step: gradients in bfloat16, weights in binary32
        _step("step_hidden", 1, 1024, 1024, "bf16", "f32"),
        # the classifier of 10000 classes on 2048 features: a tall matrix, all in binary32
        _step("step_classes", 1, 10000, 2048, "f32", "f32"),
    ]


def _log_between(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(("score", "grad", "ortho", "step"))
    if op in ("score", "grad"):
        vocab = _log_between(rng, 1000, 131072)
        rows = _log_between(rng, 1, min(8192, (1 << 29) // vocab))
        dtype = rng.choice(("f32", "bf16"))
        pad, masked = rng.choice((0, 0, 1, 40)), rng.choice((0, 0, 100))
        if op == "score":
            return {k: v for k, v in _score("", rows, vocab, dtype, rng.choice((1, 1, 9)), rng.choice((0, 1, 5, 20, 33)), pad, masked).items() if k != "name"}
        return {k: v for k, v in _grad("", rows, vocab, dtype, rng.choice((1, 1, 17)), pad, masked, rng.random() < 0.7).items() if k != "name"}
    m, n = _log_between(rng, 48, 4096), _log_between(rng, 48, 4096)
    batch = _log_between(rng, 1, max(1, min(32, (1 << 22) // (m * n))))
    dtype = rng.choice(("f32", "bf16"))
    if op == "ortho":
        return {k: v for k, v in _ortho("", batch, m, n, dtype).items() if k != "name"}
    return {k: v for k, v in _step("", batch, m, n, dtype, rng.choice(("f32", "bf16"))).items() if k != "name"}


def _inputs(case, seed):
    """The tensors of a case, from the seed alone."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if case["op"] in ("score", "grad"):
        rows, vocab, given = case["rows"], case["vocab"], case["given"]
        # logits of a model that knows something: a spread of 2.5, and for the row's token a few units more, by row
        z = torch.empty((rows, vocab + case["pad"]), dtype=DTYPES[case["dtype"]], device="cuda")
        z.normal_(0.0, 2.5, generator=g)
        z = z[:, :vocab]
        live = vocab - case["masked"]
        tokens = torch.randint(0, live, (rows, given), generator=g, device="cuda")
        lift = 12.0 * torch.rand((rows,), generator=g, device="cuda")
        at = torch.arange(rows, device="cuda")
        z[at, tokens[:, 0]] = (z[at, tokens[:, 0]].float() + lift).to(z.dtype)
        z[:, live:] = -math.inf
        ignored = torch.rand((rows,), generator=g, device="cuda") < 0.03      # padding, prompts: no token to score
        if rows > 8:
            tokens[ignored] = -1
        s = {"logits": z, "tokens": tokens}
        if case["op"] == "grad":
            w = torch.rand((rows, given), generator=g, device="cuda")
            s["grad_logp"] = -w / w.sum(1, keepdim=True) / rows               # a distillation loss (one token: the likelihood's), mean over rows
            s["grad_entropy"] = torch.full((rows,), -0.01 / rows, device="cuda") if case["entropy"] else None
        return s
    shape = (case["batch"], case["m"], case["n"])
    # gradients of a layer: a few strong directions over noise
    u = torch.randn((*shape[:2], 8), generator=g, device="cuda")
    v = torch.randn((shape[0], 8, shape[2]), generator=g, device="cuda")
    noise = torch.randn(shape, generator=g, device="cuda")
    grad = (1e-3 * (noise + 0.5 * torch.bmm(u, v))).to(DTYPES[case["dtype"]])
    if case["op"] == "ortho":
        return {"update": grad}
    w = torch.randn(shape, generator=g, device="cuda") / math.sqrt(shape[2])
    return {"grad": grad, "weight": w.to(DTYPES[case["weights"]]), "momentum": 5e-3 * torch.randn(shape, generator=g, device="cuda")}


def _scale(case):
    return math.sqrt(max(1.0, case["m"] / case["n"]))


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["op"] == "grad":        # the loss has been computed: its statistics are at hand
        s["lse"], s["entropy"] = _row_statistics(s["logits"])
    if own:
        import paper_2406_03285_amd as rb
        if case["op"] in ("score", "grad"):
            s["scorer"] = rb.TokenScorer(case["vocab"], DTYPES[case["dtype"]], given=case["given"], top=case.get("top", 0))
            if case["op"] == "score":
                s["out"] = s["scorer"].outputs(case["rows"])
            else:                   # laid out like the logits
                s["out"] = torch.empty((case["rows"], case["vocab"] + case["pad"]), dtype=DTYPES[case["dtype"]], device="cuda")[:, :case["vocab"]]
        else:
            s["ortho"] = rb.Orthogonalizer(case["m"], case["n"], batch=case["batch"], dtype=DTYPES[case["dtype"]],
                                           out_dtype=DTYPES[case.get("weights", case["dtype"])], coefficients=[COEFFICIENTS] * STEPS, eps=EPS)
            s["out"] = torch.empty_like(s["update"]) if case["op"] == "ortho" else None
    return s


def _row_statistics(logits):
    lse, entropy = [], []
    for z in logits.split(512):
        p = torch.log_softmax(z.double(), 1)
        lse.append(torch.logsumexp(z.double(), 1).float())
        entropy.append(-(p.exp() * p.nan_to_num(neginf=0.0)).sum(1).float())
    return torch.cat(lse), torch.cat(entropy)


def run(state):
    case = state["case"]
    if not own:
        return {"score": _plain_score, "grad": _plain_grad, "ortho": _plain_ortho, "step": _plain_step}[case["op"]](state)
    if case["op"] == "score":
        o = state["scorer"].score(state["logits"], state["tokens"], out=state["out"])
        return {"logp": o.logp, "lse": o.lse, "entropy": o.entropy, "top_logp": o.top_logp, "top_ids": o.top_ids}
    if case["op"] == "grad":
        return {"grad_logits": state["scorer"].grad(state["logits"], state["tokens"], state["lse"], state["entropy"], state["grad_logp"],
                                                    state["grad_entropy"], out=state["out"])}
    if case["op"] == "ortho":
        return {"out": state["ortho"].orthogonalize(state["update"], out=state["out"])}
    state["ortho"].step(state["weight"], state["grad"], state["momentum"], lr=LR, beta=BETA, weight_decay=DECAY, scale=_scale(case))
    return {"weight": state["weight"], "momentum": state["momentum"]}


def _plain_score(state):
    case, tokens = state["case"], state["tokens"]
    z = state["logits"].float()
    m = z.amax(1, keepdim=True)
    d = z - m
    e = d.exp()
    s = e.sum(1)
    lse = m[:, 0] + s.log()
    entropy = s.log() - torch.where(e > 0, e * d, 0.0).sum(1) / s
    there = (tokens >= 0) & (tokens < case["vocab"])
    logp = torch.where(there, z.gather(1, tokens.clamp(0, case["vocab"] - 1)) - lse[:, None], 0.0)
    out = {"logp": logp, "lse": lse, "entropy": entropy, "top_logp": None, "top_ids": None}
    if case["top"]:
        # equal logits in the order of their indices: one whole number per logit that orders by both
        bits = (z + 0.0).view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        keys = (order << 32) + torch.arange(case["vocab"] - 1, -1, -1, device=z.device)
        ids = case["vocab"] - 1 - (keys.topk(case["top"], dim=1).values & 0xFFFFFFFF)
        out["top_ids"], out["top_logp"] = ids, z.gather(1, ids) - lse[:, None]
    return out


def _plain_grad(state):
    tokens, w, vocab = state["tokens"], state["grad_logp"], state["case"]["vocab"]
    logp = state["logits"].float() - state["lse"][:, None]
    p = logp.exp()
    there = (tokens >= 0) & (tokens < vocab)
    w = torch.where(there, w, 0.0)
    if state["grad_entropy"] is None:
        dz = -p * w.sum(1, keepdim=True)
    else:
        dz = -p * (w.sum(1, keepdim=True) + state["grad_entropy"][:, None] * (torch.where(p > 0, logp, 0.0) + state["entropy"][:, None]))
    dz.scatter_add_(1, tokens.clamp(0, vocab - 1), w)
    return {"grad_logits": dz.to(state["logits"].dtype)}


def _newton_schulz(x):
    tall = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2).contiguous() if tall else x
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    a, b, c = COEFFICIENTS
    for _ in range(STEPS):
        p = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.matmul(b * p + c * torch.matmul(p, p), x)
    return x.transpose(1, 2) if tall else x


def _plain_ortho(state):
    return {"out": _newton_schulz(state["update"].float()).to(state["update"].dtype).contiguous()}


def _plain_step(state):
    w, mom, g = state["weight"], state["momentum"], state["grad"].float()
    mom.copy_(BETA * mom + g)
    o = _newton_schulz(g + BETA * mom)
    w.copy_((1 - LR * DECAY) * w.float() - LR * _scale(state["case"]) * o)
    return {"weight": w, "momentum": mom}


def work(case):
    if case["op"] in ("score", "grad"):
        rows, vocab, given = case["rows"], case["vocab"], case["given"]
        size = rows * vocab * (4 if case["dtype"] == "f32" else 2)
        if case["op"] == "score":
            return {"bytes": size + rows * (12 * given + 8 + 12 * case["top"]), "flops": 6.0 * rows * vocab}
        return {"bytes": 2 * size + rows * (12 * given + 12), "flops": 7.0 * rows * vocab}
    short, long = sorted((case["m"], case["n"]))
    elems, size = case["batch"] * short * long, 4 if case["dtype"] == "f32" else 2
    # two of a step's three products are symmetric
    flops = case["batch"] * STEPS * (short * short * long + short ** 3 + 2 * short * short * long)
    if case["op"] == "ortho":
        return {"bytes": 2 * elems * size, "flops": float(flops)}
    return {"bytes": elems * (size + 8 + 2 * (4 if case["weights"] == "f32" else 2)), "flops": float(flops)}


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "score":
        return _exact_score(case, s)
    if case["op"] == "grad":
        return _exact_grad(case, s)
    if case["op"] == "ortho":
        return {"out": _exact_ortho(s["update"].double())}
    mom = BETA * s["momentum"].double() + s["grad"].double()
    o = _exact_ortho(s["grad"].double() + BETA * mom)
    return {"weight": (1 - LR * DECAY) * s["weight"].double() - LR * _scale(case) * o, "momentum": mom}


def _exact_score(case, s):
    parts = {"logp": [], "lse": [], "entropy": [], "top_logp": []}
    for z, t in zip(s["logits"].split(512), s["tokens"].split(512)):
        logp = torch.log_softmax(z.double(), 1)
        at = logp.gather(1, t.clamp(min=0))
        parts["logp"].append(torch.where(t >= 0, at, torch.zeros_like(at)))
        parts["lse"].append(torch.logsumexp(z.double(), 1))
        parts["entropy"].append(-(logp.exp() * logp.clamp(min=-1e300)).sum(1))
        parts["top_logp"].append(logp.topk(case["top"], 1).values if case["top"] else logp[:, :0])
    out = {k: torch.cat(v) for k, v in parts.items()}
    return {**out, "top_logp": out["top_logp"] if case["top"] else None, "top_ids": None}


def _exact_grad(case, s):
    """By differentiation of the definition."""
    rows = []
    for i in range(0, case["rows"], 256):
        z = s["logits"][i:i + 256].double().requires_grad_()
        t = s["tokens"][i:i + 256]
        logp = torch.log_softmax(z, 1)
        loss = (logp.gather(1, t.clamp(min=0)) * (s["grad_logp"][i:i + 256].double() * (t >= 0))).sum()
        if s["grad_entropy"] is not None:
            live = torch.isfinite(z)
            entropy = -(logp.exp() * logp.masked_fill(~live, 0.0)).sum(1)
            loss = loss + (entropy * s["grad_entropy"][i:i + 256].double()).sum()
        rows.append(torch.autograd.grad(loss, z)[0])
    return {"grad_logits": torch.cat(rows)}


def _exact_ortho(g):
    """A step multiplies by a polynomial of the Gram matrix, and those of all steps commute: only the Gram matrix is iterated."""
    tall = g.shape[1] > g.shape[2]
    g = g.transpose(1, 2).contiguous() if tall else g
    a, b, c = COEFFICIENTS
    outs = []
    for x in g:
        x = x / (torch.linalg.vector_norm(x) + EPS)
        eye = torch.eye(x.shape[0], dtype=x.dtype, device=x.device)
        gram, total = x @ x.t().contiguous(), eye
        for _ in range(STEPS):
            p = a * eye + b * gram + c * (gram @ gram)
            total = p @ total
            gram = p @ gram @ p
        outs.append(total @ x)
    o = torch.stack(outs)
    return o.transpose(1, 2).contiguous() if tall else o
