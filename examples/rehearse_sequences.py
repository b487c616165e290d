"""Training a small language model task by task with rehearsal: a buffer of token sequences of any length, packed behind the fresh ones.

Each task has a language of its own: what token follows which.  A row of the buffer is a sequence in a place of `PLACE` tokens with its length in front.  In
every iteration fresh and rehearsed sequences lie behind one another, each a document of its own, and the model's blocks are

    norm(x)                                   LayerNorm
    queries, keys, values                     a product
    attention                                 DocumentAttention: causal within a document, its first `PROMPT` tokens seen by all of it
    norm(residual + dropout(product))         LayerNorm with Drop: the sum is the next residual
    a layer in between, dropout               products, rb.dropout

with TokenScorer's likelihoods at the end and Orthogonalizer's steps for the matrices.

Run it: python examples/rehearse_sequences.py [--no-rehearsal] [--steps N]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2406_03285_amd as rb  # noqa: E402

VOCAB, TASKS, PLACE, PROMPT = 48, 3, 47, 4
WIDTH, HEADS, KV_HEADS, BLOCKS = 64, 4, 2, 2
FRESH, CANDIDATES, REHEARSED = 24, 8, 8
SLOTS, DROPOUT = 40, 0.1


class Model(torch.nn.Module):
    def __init__(self, device, dropout=DROPOUT):
        super().__init__()
        g = torch.Generator().manual_seed(1)
        dim = WIDTH // HEADS

        def matrix(m, n):
            return torch.nn.Parameter((torch.randn((m, n), generator=g) * n ** -0.5).to(device))
        self.tokens = matrix(VOCAB, WIDTH)
        self.blocks = torch.nn.ModuleList(torch.nn.ParameterDict({
            "qkv": matrix((HEADS + 2 * KV_HEADS) * dim, WIDTH), "back": matrix(WIDTH, HEADS * dim), "up": matrix(2 * WIDTH, WIDTH), "down": matrix(WIDTH, 2 * WIDTH),
            "before": torch.nn.Parameter(torch.ones(WIDTH, device=device)), "between": torch.nn.Parameter(torch.ones(WIDTH, device=device)),
            "bias": torch.nn.Parameter(torch.zeros(WIDTH, device=device))}) for _ in range(BLOCKS))
        self.dropout, self.dim = dropout, dim
        # one handle of each serves all blocks
        self.norm = rb.LayerNorm(WIDTH, torch.bfloat16, weight_dtype=torch.float32, device=device)
        self.attention = rb.DocumentAttention(HEADS, dim, KV_HEADS, max_tokens=(FRESH + REHEARSED) * PLACE, device=device)

    def forward(self, tokens, documents, step):
        """Logits [positions, VOCAB] of packed documents."""
        half = torch.bfloat16
        x = self.tokens[tokens].to(half)
        for i, b in enumerate(self.blocks):
            def drop(layer):           # every layer and step has a mask of its own
                return rb.Drop(self.dropout, 1000 * i + layer, step)
            y = self.norm(x, b["before"]).y
            heads = (y @ b["qkv"].to(half).t()).split([HEADS * self.dim, KV_HEADS * self.dim, KV_HEADS * self.dim], 1)
            q, k, v = (z.unflatten(1, (n, self.dim)) for z, n in zip(heads, (HEADS, KV_HEADS, KV_HEADS)))
            a = self.attention(q, k, v, documents).flatten(1)
            o = self.norm(a @ b["back"].to(half).t(), b["between"], b["bias"], residual=x, drop=drop(0))
            x = o.total + rb.dropout(torch.relu(o.y @ b["up"].to(half).t()) @ b["down"].to(half).t(), drop(1))
        return (x @ self.tokens.to(half).t()).float()


def sequences(task, step, count, device):
    """[count, 1 + PLACE]: lengths, and tokens behind them: each follows from the one before by the task's table, or one in five by chance."""
    g = torch.Generator().manual_seed(10 ** 6 * task + step)
    follows = torch.randperm(VOCAB, generator=torch.Generator().manual_seed(task))
    lengths = torch.randint(PLACE // 3, PLACE + 1, (count,), generator=g)
    t = torch.randint(0, VOCAB, (count, PLACE), generator=g)
    free = torch.rand((count, PLACE), generator=g) < 0.2
    for i in range(1, PLACE):
        t[:, i] = torch.where(free[:, i], t[:, i], follows[t[:, i - 1]])
    return torch.cat([lengths[:, None], t], 1).to(device)


def packed(rows):
    """(tokens, documents, the token that follows each position or -1) of rows of sequences, each in its place."""
    lengths, tokens = rows[:, 0], rows[:, 1:].reshape(-1)
    offsets = torch.arange(rows.shape[0] + 1, device=rows.device) * PLACE
    at = torch.arange(PLACE, device=rows.device)
    target = torch.where(at[None] + 1 < lengths[:, None], rows[:, 1:].roll(-1, 1), -1).clone()
    target[:, :PROMPT - 1] = -1                     # (the prompt sees itself)
    return tokens, rb.Documents(offsets, lengths.contiguous(), torch.full_like(lengths, PROMPT)), target.reshape(-1)


def train(rehearse=True, steps=40, device="cuda"):
    """Mean likelihoods of every task's sequences after the last one, and the losses on the way."""
    model = Model(device)
    scorer = rb.TokenScorer(VOCAB, torch.float32, device=device)
    matrices = [w for w in model.parameters() if w.dim() == 2]
    vectors = [w for w in model.parameters() if w.dim() == 1]
    ortho = [rb.Orthogonalizer(*w.shape, device=device) for w in matrices]
    momenta = [torch.zeros_like(w) for w in matrices]
    buffer = rb.RehearsalBuffer(TASKS, SLOTS, (1 + PLACE,), torch.float32, device=device)
    rehearsed = torch.zeros((REHEARSED, 1 + PLACE), device=device)
    labels = torch.full((REHEARSED,), -1, dtype=torch.int64, device=device)
    losses, t = [], 0
    for task in range(TASKS):
        for step in range(steps):
            fresh = sequences(task, step, FRESH, device)
            old = rehearsed.contiguous().view(torch.int32).long()
            there = (labels >= 0) & rehearse                       # (no representatives before the first update: documents of no tokens)
            rows = torch.cat([fresh, torch.where(there[:, None], old, 0)])
            tokens, documents, target = packed(rows)
            logp = scorer(model(tokens, documents, t), target[:, None]).logp
            loss = -logp.sum() / (target >= 0).sum()
            for w in model.parameters():
                w.grad = None
            loss.backward()
            for o, w, m in zip(ortho, matrices, momenta):
                o.step(w, w.grad, m, lr=0.02, weight_decay=0.01)
            with torch.no_grad():
                for w in vectors:
                    w -= 0.05 * w.grad
            losses.append(loss.detach())
            stored = fresh.to(torch.int32).view(torch.float32)     # the bits of whole numbers
            buffer.update_sample(stored, torch.full((FRESH,), task, device=device), CANDIDATES, REHEARSED, 7, t, rehearsed, labels)
            t += 1
    model.dropout = 0.0
    likelihoods = []
    with torch.no_grad():
        for task in range(TASKS):
            tokens, documents, target = packed(sequences(task, 10 ** 5, FRESH, device))
            logp = scorer.score(model(tokens, documents, 0), target[:, None]).logp
            likelihoods.append((logp.sum() / (target >= 0).sum()).item())
    return likelihoods, torch.stack(losses).cpu()


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--no-rehearsal", action="store_true")
    p.add_argument("--steps", type=int, default=60, help="iterations per task")
    a = p.parse_args()
    likelihoods, losses = train(not a.no_rehearsal, a.steps)
    print("loss of the first and the last ten iterations: %.3f %.3f" % (losses[:10].mean(), losses[-10:].mean()))
    print("mean log likelihood by task:", " ".join("%.3f" % v for v in likelihoods))


if __name__ == "__main__":
    main()
