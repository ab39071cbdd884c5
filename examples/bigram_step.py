"""A next-word model trained by n simulated workers on one GPU, every step
through this library:

  loss       xent_forward / xent_backward   the head's loss and gradients
  compress   ht_compress                    each worker's gradient, error feedback
  average    sparse_accumulate              the workers' payloads
  update     muon_apply                     momentum and orthogonalised step

    python examples/bigram_step.py [--steps 60] [--workers 4]

The model looks a word's vector up, multiplies it by one matrix and scores the
next word with the output head: three weight matrices in one flat fp32 vector,
whose views are the tensors that the calls take.  The data are pairs of words
drawn from a fixed random table, so that the loss has a known floor, the
table's entropy.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2108_00951_amd import binding as efs  # noqa: E402

VOCAB, WIDTH, CHOICES = 1000, 96, 4
IGNORE = -100


class Model:
    """Layers of a flat vector: (offset, rows, cols)."""

    def __init__(self, device):
        self.layers, at = [], 0
        for rows, cols in ((VOCAB, WIDTH), (WIDTH, WIDTH), (VOCAB, WIDTH)):
            self.layers.append((at, rows, cols))
            at += rows * cols
        self.size = at
        gen = torch.Generator(device=device).manual_seed(1)
        self.x = torch.randn(at, generator=gen, device=device).mul_(WIDTH ** -0.5)

    def views(self, flat):
        return [flat[at:at + rows * cols].view(rows, cols) for at, rows, cols in self.layers]


class Worker:
    """One worker's data stream, gradient, residual and payload."""

    def __init__(self, model, seed, tokens, device):
        self.gen = torch.Generator(device=device).manual_seed(100 + seed)
        self.g = torch.zeros(model.size, device=device)
        self.e = torch.zeros(model.size, device=device)
        room = model.size
        self.payload = (torch.empty(room, dtype=torch.int32, device=device), torch.empty(room, device=device),
                        efs.new_counter(device))
        self.loss = torch.empty(tokens, device=device)
        self.lse = torch.empty(tokens, device=device)
        self.dh = torch.empty(tokens, WIDTH, device=device)
        self.ws = efs.new_xent_workspace(tokens, VOCAB, WIDTH, torch.float32, device)

    def batch(self, table, tokens):
        """Words and the words after them; a tenth are padding."""
        word = torch.randint(0, VOCAB, (tokens,), generator=self.gen, device=table.device)
        pick = torch.randint(0, CHOICES, (tokens,), generator=self.gen, device=table.device)
        after = table[word, pick]
        pad = torch.rand(tokens, generator=self.gen, device=table.device) < 0.1
        return word, torch.where(pad, IGNORE, after)

    def step(self, model, table, tokens, lr, lam):
        """The gradient of this worker's batch, compressed.  Returns the mean loss."""
        embed, mix, head = model.views(model.x)
        d_embed, d_mix, d_head = model.views(self.g)
        word, after = self.batch(table, tokens)
        count = (after != IGNORE).sum().clamp_(min=1)
        v = embed[word]
        h = v @ mix
        efs.xent_forward(h, head, after, self.loss, self.lse, self.ws, ignore_index=IGNORE)
        weight = torch.ones(tokens, device=h.device).div_(count)
        # the head's gradient lands in the flat vector itself
        efs.xent_backward(h, head, after, self.lse, weight, self.dh, d_head, self.ws, ignore_index=IGNORE)
        torch.mm(v.t(), self.dh, out=d_mix)
        d_embed.zero_().index_add_(0, word, self.dh @ mix.t())
        efs.ht_compress(self.g, self.e, lr, lam, *self.payload)
        return self.loss.sum() / count


def train(steps, workers, tokens=512, device="cuda", lam=2e-4, gamma=0.05, report=None):
    """Trains; returns the mean loss of every step and the share of entries sent."""
    model = Model(device)
    gen = torch.Generator(device=device).manual_seed(2)
    table = torch.randint(0, VOCAB, (VOCAB, CHOICES), generator=gen, device=device)
    team = [Worker(model, s, tokens, device) for s in range(workers)]
    avg = torch.empty(model.size, device=device)
    m = torch.zeros(model.size, device=device)
    payloads = [w.payload for w in team]
    average = efs.prepare_sparse_accumulate(payloads, model.size, avg, efs.new_apply_workspace(payloads, model.size, device))
    update = efs.prepare_muon_apply(avg, model.x, m, model.layers, efs.new_muon_workspace([v[1:] for v in model.layers], device),
                                    beta=0.9, gamma=gamma, weight_decay=0.0)
    losses, sent = [], 0.0
    for t in range(steps):
        loss = sum(w.step(model, table, tokens, 1.0, lam) for w in team) / workers
        average()
        update()
        losses.append(float(loss))
        sent += sum(efs.counter_value(w.payload[2]) for w in team) / (workers * model.size)
        if report is not None:
            report(t, losses[-1])
    return losses, sent / max(steps, 1)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--workers", type=int, default=4)
    a = ap.parse_args()

    def report(t, loss):
        if t % 10 == 0:
            print("step %3d  loss %.4f" % (t, loss), flush=True)
    losses, density = train(a.steps, a.workers, report=report)
    print("loss %.4f -> %.4f (uniform guess %.4f, the data's own entropy about %.4f); %.2f %% of the gradient sent"
          % (losses[0], losses[-1], math.log(VOCAB), math.log(CHOICES), 100 * density))


if __name__ == "__main__":
    main()
