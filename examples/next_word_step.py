"""A next-word model trained by n simulated workers on one GPU, with no arithmetic
of the step outside this library but two products with one small matrix:

  lookup     embed_forward / embed_backward          the words' vectors, scaled
  norm       layernorm_forward / layernorm_backward  before the head
  loss       xent_forward / xent_backward            the head's loss; the head is the
                                                     lookup's table (shared weights)
  compress   ht_compress                             each worker's gradient, error feedback
  average    sparse_accumulate                       the workers' payloads
  update     muon_apply                              the matrix between lookup and norm
             adamw_apply                             table and norm, states in 8 bits

    python examples/next_word_step.py [--steps 60] [--workers 4]

The parameters are layers of one flat fp32 vector, whose views are the tensors
that the calls take.  The data are pairs of words drawn from a fixed random
table.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2108_00951_amd import binding as efs  # noqa: E402

VOCAB, WIDTH, CHOICES = 1000, 96, 4
SCALE = math.sqrt(WIDTH)
IGNORE = -100


class Model:
    """Layers of a flat vector: the table (also the head), the matrix, the norm's
    weight and bias."""

    def __init__(self, device):
        self.shapes = [(VOCAB, WIDTH), (WIDTH, WIDTH), (WIDTH,), (WIDTH,)]
        self.sizes = [math.prod(s) for s in self.shapes]
        self.size = sum(self.sizes)
        gen = torch.Generator(device=device).manual_seed(1)
        self.x = torch.zeros(self.size, device=device)
        table, mix, weight, _ = self.views(self.x)
        table.copy_(torch.randn(table.shape, generator=gen, device=device).mul_(1.0 / SCALE))
        mix.copy_(torch.randn(mix.shape, generator=gen, device=device).mul_(WIDTH ** -0.5))
        weight.fill_(1.0)

    def views(self, flat):
        return [part.view(shape) for part, shape in zip(flat.split(self.sizes), self.shapes)]


class Worker:
    """One worker's data stream, activations, gradient, residual and payload."""

    def __init__(self, model, seed, tokens, device):
        self.gen = torch.Generator(device=device).manual_seed(100 + seed)
        self.tokens = tokens
        self.g, self.e = (torch.zeros(model.size, device=device) for _ in range(2))
        self.payload = (torch.empty(model.size, dtype=torch.int32, device=device), torch.empty(model.size, device=device),
                        efs.new_counter(device))
        self.v, self.h, self.y, self.dy, self.dh = (torch.empty(tokens, WIDTH, device=device) for _ in range(5))
        self.loss, self.lse, self.mean, self.rstd = (torch.empty(tokens, device=device) for _ in range(4))
        self.lookup_ws = efs.new_embed_workspace(tokens, VOCAB, WIDTH, device)
        self.norm_ws = efs.new_layernorm_workspace(tokens, WIDTH, device)
        self.loss_ws = efs.new_xent_workspace(tokens, VOCAB, WIDTH, torch.float32, device)

    def batch(self, table):
        """Words and the words after them; a tenth are padding."""
        word = torch.randint(0, VOCAB, (self.tokens,), generator=self.gen, device=table.device)
        pick = torch.randint(0, CHOICES, (self.tokens,), generator=self.gen, device=table.device)
        pad = torch.rand(self.tokens, generator=self.gen, device=table.device) < 0.1
        return torch.where(pad, IGNORE, word), torch.where(pad, IGNORE, table[word, pick])

    def gradient(self, model, word, after):
        """The gradient of the mean loss over the batch into self.g.  Returns the mean loss."""
        table, mix, weight, bias = model.views(model.x)
        d_table, d_mix, d_weight, d_bias = model.views(self.g)
        count = (after != IGNORE).sum().clamp_(min=1)
        efs.embed_forward(table, word, self.v, scale=SCALE, ignore_index=IGNORE)
        torch.mm(self.v, mix, out=self.h)
        efs.layernorm_forward(self.h, weight, bias, self.y, self.mean, self.rstd)
        efs.xent_forward(self.y, table, after, self.loss, self.lse, self.loss_ws, ignore_index=IGNORE)
        share = torch.ones(self.tokens, device=word.device).div_(count)
        # the head's gradient writes the table's layer, the lookup's adds to it
        efs.xent_backward(self.y, table, after, self.lse, share, self.dy, d_table, self.loss_ws, ignore_index=IGNORE)
        efs.layernorm_backward(self.h, weight, self.mean, self.rstd, self.dy, self.dh, d_weight, d_bias, self.norm_ws)
        torch.mm(self.v.t(), self.dh, out=d_mix)
        torch.mm(self.dh, mix.t(), out=self.dy)   # of the lookup
        efs.embed_backward(self.dy, word, d_table, self.lookup_ws, scale=SCALE, ignore_index=IGNORE, accumulate=True)
        return self.loss.sum() / count


class Update:
    """The averaged gradient into the parameters: the matrix orthogonalised, the
    rest by AdamW, of which only the table decays."""

    def __init__(self, model, avg, lr, device):
        g, x = avg.split(model.sizes), model.x.split(model.sizes)
        rest = [0, 2, 3]
        m, v = efs.new_adamw_state([model.sizes[i] for i in rest], device)
        self.adamw = efs.prepare_adamw_apply([g[i] for i in rest], [x[i] for i in rest], m, v, lr=lr,
                                             weight_decay=[0.01, 0.0, 0.0])
        layer = (model.sizes[0], WIDTH, WIDTH)
        self.muon = efs.prepare_muon_apply(avg, model.x, torch.zeros_like(model.x), [layer],
                                           efs.new_muon_workspace([layer[1:]], device), beta=0.9, gamma=0.02)
        self.steps = 0

    def __call__(self):
        self.steps += 1
        self.muon()
        self.adamw(self.steps)


def train(steps, workers, tokens=512, device="cuda", lam=2e-3, lr=3e-3, report=None):
    """Trains; returns the mean loss of every step and the share of entries sent."""
    model = Model(device)
    gen = torch.Generator(device=device).manual_seed(2)
    pairs = torch.randint(0, VOCAB, (VOCAB, CHOICES), generator=gen, device=device)
    team = [Worker(model, s, tokens, device) for s in range(workers)]
    avg = torch.empty(model.size, device=device)
    payloads = [w.payload for w in team]
    average = efs.prepare_sparse_accumulate(payloads, model.size, avg, efs.new_apply_workspace(payloads, model.size, device))
    update = Update(model, avg, lr, device)
    losses, sent = [], 0.0
    for t in range(steps):
        loss = 0.0
        for w in team:
            loss = loss + w.gradient(model, *w.batch(pairs)) / workers
            efs.ht_compress(w.g, w.e, 1.0, lam, *w.payload)
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
