"""Class-incremental training with rehearsal: a buffer of feature rows, each kept with what the model once answered for it.

Tasks come one after the other, each with classes of its own.  A row of the buffer holds a sample's features and, behind them, the
`ALTERNATIVES` best classes that the model named when the sample was new, with their log probabilities.  In every iteration

    logits = model(fresh and rehearsed samples)
    scorer(logits, ...)             log probabilities of the labels and of the stored alternatives, entropy, the new alternatives
    loss.backward()                 likelihood of the labels + distillation of what is rehearsed - a little entropy
    Orthogonalizer.step(...)        each weight matrix by its orthogonalised momentum
    buffer.update_sample(...)       the fresh samples (with their alternatives) go in, the next representatives come out

Run it: python examples/rehearse_classes.py [--no-rehearsal] [--steps N]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2406_03285_amd as rb  # noqa: E402

CLASSES, TASKS, FEATURES, HIDDEN = 40, 4, 256, 192
ALTERNATIVES = 8
FRESH, CANDIDATES, REHEARSED = 96, 24, 32
SLOTS = 30
DISTILL, ENTROPY = 0.5, 0.01


class Model(torch.nn.Module):
    def __init__(self, device):
        super().__init__()
        g = torch.Generator().manual_seed(1)
        self.hidden = torch.nn.Parameter((torch.randn((HIDDEN, FEATURES), generator=g) / FEATURES ** 0.5).to(device))
        self.classes = torch.nn.Parameter((torch.randn((CLASSES, HIDDEN), generator=g) / HIDDEN ** 0.5).to(device))

    def forward(self, x):
        return torch.relu(x @ self.hidden.t()) @ self.classes.t()


def batches(means, task, step, count):
    """Samples of the classes of one task: a class is a direction and noise around it."""
    g = torch.Generator(device=means.device).manual_seed(1000 * task + step)
    per = CLASSES // TASKS
    y = task * per + torch.randint(0, per, (count,), generator=g, device=means.device)
    return means[y] + torch.randn((count, FEATURES), generator=g, device=means.device), y


def pack(x, ids, logp):
    """Rows of the buffer: features, the alternatives' numbers (the bits of int32), their log probabilities."""
    return torch.cat([x, ids.to(torch.int32).view(torch.float32), logp], 1)


def unpack(rows):
    ids = rows[:, FEATURES:FEATURES + ALTERNATIVES].contiguous().view(torch.int32).long()
    return rows[:, :FEATURES], ids, rows[:, FEATURES + ALTERNATIVES:]


def train(rehearse=True, steps=60, device="cuda"):
    """Accuracy on every task after the last one, and the losses on the way."""
    g = torch.Generator().manual_seed(0)
    means = 0.35 * torch.randn((CLASSES, FEATURES), generator=g).to(device)
    model = Model(device)
    # one given token is the label, the others are stored alternatives (a fresh sample has none: -1 is left out)
    scorer = rb.TokenScorer(CLASSES, torch.float32, given=1 + ALTERNATIVES, top=ALTERNATIVES, device=device)
    weights = [model.hidden, model.classes]
    ortho = [rb.Orthogonalizer(*w.shape, device=device) for w in weights]
    momenta = [torch.zeros_like(w) for w in weights]
    buffer = rb.RehearsalBuffer(CLASSES, SLOTS, (FEATURES + 2 * ALTERNATIVES,), torch.float32, device=device)
    rehearsed = torch.zeros((REHEARSED, FEATURES + 2 * ALTERNATIVES), device=device)
    labels = torch.full((REHEARSED,), -1, dtype=torch.int64, device=device)
    losses, t = [], 0
    for task in range(TASKS):
        for step in range(steps):
            x, y = batches(means, task, step, FRESH)
            old_x, old_ids, old_logp = unpack(rehearsed)
            there = (labels >= 0)[:, None] & rehearse                # (no representatives before the first update)
            tokens = torch.full((FRESH + REHEARSED, 1 + ALTERNATIVES), -1, device=device)
            tokens[:FRESH, 0] = y
            tokens[FRESH:, 0] = torch.where(there[:, 0], labels, -1)
            tokens[FRESH:, 1:] = torch.where(there, old_ids, -1)
            old_p = torch.where(there, old_logp.exp(), 0.0)

            scores = scorer(model(torch.cat([x, old_x])), tokens)
            likelihood = -scores.logp[:, 0].sum() / (tokens[:, 0] >= 0).sum()
            distilled = -(old_p * scores.logp[FRESH:, 1:]).sum() / REHEARSED
            loss = likelihood + DISTILL * distilled - ENTROPY * scores.entropy[:FRESH].mean()
            for w in weights:
                w.grad = None
            loss.backward()
            for o, w, m in zip(ortho, weights, momenta):
                o.step(w, w.grad, m, lr=0.02, weight_decay=0.01)
            losses.append(loss.detach())

            rows = pack(x, scores.top_ids[:FRESH], scores.top_logp[:FRESH].detach())
            buffer.update_sample(rows, y, CANDIDATES, REHEARSED, 7, t, rehearsed, labels)
            t += 1
    accuracy = []
    with torch.no_grad():
        best = rb.TokenScorer(CLASSES, torch.float32, given=0, top=1, device=device)
        for task in range(TASKS):
            x, y = batches(means, task, 10 ** 6, 1000)
            accuracy.append((best.score(model(x)).top_ids[:, 0] == y).float().mean().item())
    return accuracy, torch.stack(losses).cpu()


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--no-rehearsal", action="store_true")
    p.add_argument("--steps", type=int, default=60, help="iterations per task")
    a = p.parse_args()
    accuracy, losses = train(not a.no_rehearsal, a.steps)
    print("loss of the first and the last ten iterations: %.3f %.3f" % (losses[:10].mean(), losses[-10:].mean()))
    print("accuracy by task:", " ".join("%.3f" % v for v in accuracy))


if __name__ == "__main__":
    main()
