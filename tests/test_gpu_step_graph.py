"""The lookup, the layer norm, the head's loss and the AdamW step together, as a
step of a small model: its gradients against the whole model's in 64 bits, and
the step captured in a HIP graph and replayed, against the same step run
eagerly; other streams; other devices."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2108_00951_amd import binding as efs  # noqa: E402

DEV = "cuda"
IGNORE = -100


class Model:
    """table (tied to the head or not), norm, head: layers of flat fp32 vectors."""

    def __init__(self, vocab, width, tokens, bits, tied, dtype=torch.float32):
        self.vocab, self.width, self.tokens, self.tied, self.dtype = vocab, width, tokens, tied, dtype
        self.sizes = [vocab * width, width, width] + ([] if tied else [vocab * width])
        rng = np.random.default_rng(2)
        first = [rng.standard_normal(self.sizes[0]) * 0.1, 1 + 0.2 * rng.standard_normal(width), 0.1 * rng.standard_normal(width)]
        if not tied:
            first.append(rng.standard_normal(vocab * width) * 0.1)
        self.x = torch.from_numpy(np.concatenate(first).astype(np.float32)).to(DEV)
        self.g = torch.zeros_like(self.x)
        self.work = self.x.to(dtype) if dtype != torch.float32 else self.x   # what the model computes with
        self.m, self.v = efs.new_adamw_state(self.sizes, DEV) if bits == 8 else \
            tuple(list(torch.zeros_like(self.x).split(self.sizes)) for _ in range(2))
        self.step = torch.zeros((), dtype=torch.int64, device=DEV)
        self.factors = torch.ones(2, device=DEV)
        t = (tokens,)
        self.ids, self.target = (torch.zeros(t, dtype=torch.int64, device=DEV) for _ in range(2))
        self.weight = torch.zeros(t, device=DEV)
        self.loss, self.lse, self.mean, self.rstd = (torch.zeros(t, device=DEV) for _ in range(4))
        self.h, self.y, self.dy, self.dh = (torch.zeros(tokens, width, dtype=dtype, device=DEV) for _ in range(4))
        self.dhead = torch.zeros(vocab, width, dtype=dtype, device=DEV) if dtype != torch.float32 else None
        self.ews = efs.new_embed_workspace(tokens, vocab, width, DEV)
        self.nws = efs.new_layernorm_workspace(tokens, width, DEV)
        self.xws = efs.new_xent_workspace(tokens, vocab, width, dtype, DEV)
        self.ews.fill_(0xFF), self.nws.fill_(0xFF)

    def views(self, flat):
        parts = flat.split(self.sizes)
        table, head = parts[0].view(self.vocab, self.width), parts[0 if self.tied else 3].view(self.vocab, self.width)
        return table, parts[1], parts[2], head

    def gradients(self, stream=None):
        table, w, b, head = self.views(self.work)
        dtable, dw, db, dhead = self.views(self.g)
        s = {"stream": stream}
        efs.embed_forward(table, self.ids, self.h, scale=3.0, ignore_index=IGNORE, **s)
        efs.layernorm_forward(self.h, w, b, self.y, self.mean, self.rstd, **s)
        efs.xent_forward(self.y, head, self.target, self.loss, self.lse, self.xws, ignore_index=IGNORE, **s)
        efs.xent_backward(self.y, head, self.target, self.lse, self.weight, self.dy,
                          dhead if self.dhead is None else self.dhead, self.xws, ignore_index=IGNORE, **s)
        if self.dhead is not None:
            dhead.copy_(self.dhead)
        efs.layernorm_backward(self.h, w, self.mean, self.rstd, self.dy, self.dh, dw if self.dhead is None else None,
                               db if self.dhead is None else None, self.nws, **s)
        if self.dhead is not None:   # weights of the norm in 32 bits: their gradients too
            efs.layernorm_backward(self.h, self.views(self.x)[1], self.mean, self.rstd, self.dy, self.dh, dw, db, self.nws, **s)
        efs.embed_backward(self.dh, self.ids, dtable, self.ews, scale=3.0, ignore_index=IGNORE, accumulate=self.tied, **s)

    def update(self, stream=None):
        copy = list(self.work.split(self.sizes)) if self.dhead is not None else None
        efs.adamw_apply(self.g.split(self.sizes), self.x.split(self.sizes), self.m, self.v, self.step, lr=1e-2,
                        weight_decay=[0.1, 0.0, 0.0, 0.1][:len(self.sizes)], copy=copy, factors=self.factors, seed=3,
                        stream=stream)

    def batch(self, seed):
        rng = np.random.default_rng(seed)
        ids = rng.integers(0, self.vocab, self.tokens)
        ids[: self.tokens // 3] = self.vocab // 2   # a word that many tokens are
        ids[-3:] = IGNORE
        target = rng.integers(0, self.vocab, self.tokens)
        target[-5:] = IGNORE
        self.ids.copy_(torch.from_numpy(ids))
        self.target.copy_(torch.from_numpy(target))
        self.weight.fill_(1.0 / (self.tokens - 5))
        self.step += 1
        self.factors.copy_(torch.tensor([1.0 / (1 + seed), 0.9]))

    def state(self):
        return [self.x.clone(), self.g.clone(), self.work.clone(), self.loss.clone()] + [t.clone() for t in list(self.m) + list(self.v)]


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("vocab, width, tokens", [(50, 33, 40), (300, 130, 700), (200, 64, 5000)])
def test_gradients_of_the_whole_step(vocab, width, tokens, tied):
    model = Model(vocab, width, tokens, 32, tied)
    model.batch(1)
    model.gradients()
    x = model.x.double().cpu().requires_grad_()
    table, w, b, head = model.views(x)
    ids, target = model.ids.cpu(), model.target.cpu()
    there = ids != IGNORE
    h = torch.where(there[:, None], table[torch.where(there, ids, 0)] * 3.0, 0.0)
    c = h - h.mean(1, keepdim=True)
    y = c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5) * w + b
    loss = torch.nn.functional.cross_entropy(y @ head.t(), target, reduction="sum", ignore_index=IGNORE) / (tokens - 5)
    loss.backward()
    assert abs(float(model.loss.double().sum()) / (tokens - 5) - loss.item()) <= 1e-6 * loss.item()
    start = 0
    for n in model.sizes:
        got, want = model.g[start:start + n].double().cpu(), x.grad[start:start + n]
        # the loss's gradients are of 22 bits' products; sums of up to `tokens` terms follow
        assert float((got - want).norm() / want.norm()) <= 2.0 ** -16
        start += n


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("vocab, width, tokens, dtype", [(50, 33, 40, torch.float32), (300, 64, 5000, torch.float32),
                                                         (300, 128, 700, torch.bfloat16)])
def test_step_replays_in_a_graph(vocab, width, tokens, dtype, bits):
    eager, graphed = (Model(vocab, width, tokens, bits, False, dtype) for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):   # recorded only
        graphed.gradients()
        graphed.update()
    torch.cuda.synchronize()
    for t in range(4):
        eager.batch(t)
        eager.gradients()
        eager.update()
        graphed.batch(t)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k, (got, want) in enumerate(zip(graphed.state(), eager.state())):
            assert torch.equal(got, want), (t, k)


def test_two_graphs_with_workspaces_of_their_own():
    models = [Model(300, 64, 5000, 32, False) for _ in range(2)]
    graphs = [torch.cuda.CUDAGraph() for _ in models]
    torch.cuda.synchronize()
    for g, m in zip(graphs, models):
        with torch.cuda.graph(g):
            m.gradients()
    streams = [torch.cuda.Stream() for _ in models]
    for t in range(3):
        for m in models:
            m.batch(5 + t)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):   # at once
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        want = Model(300, 64, 5000, 32, False)
        want.batch(5 + t)
        want.gradients()
        for m in models:
            assert torch.equal(m.g, want.g)


@pytest.mark.parametrize("explicit", [False, True])
def test_calls_run_on_another_stream(explicit):
    want = Model(300, 64, 700, 8, False)
    want.batch(1)
    want.gradients()
    want.update()
    got = Model(300, 64, 700, 8, False)
    got.batch(1)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    if explicit:
        got.gradients(s)
        got.update(s)
    else:
        with torch.cuda.stream(s):
            got.gradients()
            got.update()
    s.synchronize()
    for a, b in zip(got.state(), want.state()):
        assert torch.equal(a, b)


def test_tensors_of_another_device_are_refused(monkeypatch):
    m = Model(50, 32, 20, 32, False)
    m.batch(0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    table, w, b, _ = m.views(m.x)
    for call in (lambda: efs.embed_forward(table, m.ids, m.h), lambda: efs.embed_backward(m.h, m.ids, table, m.ews),
                 lambda: efs.layernorm_forward(m.h, w, b, m.y),
                 lambda: efs.layernorm_backward(m.h, w, m.mean, m.rstd, m.dy, m.dh, None, None, m.nws), m.update):
        with pytest.raises(ValueError, match="current device"):
            call()


@pytest.mark.parametrize("wrapped", [2 ** 64, -2 ** 64])
def test_whole_numbers_past_64_bits_are_refused(wrapped):
    """An ignored word 2^64 on would be the word itself, and so would a step."""
    m = Model(50, 32, 20, 32, False)
    m.batch(0)
    table = m.views(m.x)[0]
    before = m.x.clone()
    loss, lse = torch.empty(20, device=DEV), torch.empty(20, device=DEV)
    ws = efs.new_xent_workspace(20, 50, 32, torch.float32, DEV)
    for call in (lambda: efs.embed_forward(table, m.ids, m.h, ignore_index=3 + wrapped),
                 lambda: efs.embed_backward(m.h, m.ids, table, m.ews, ignore_index=3 + wrapped),
                 lambda: efs.xent_forward(m.h, table, m.target, loss, lse, ws, ignore_index=3 + wrapped),
                 lambda: efs.xent_backward(m.h, table, m.target, lse, m.weight, m.dh, torch.empty_like(table), ws,
                                           ignore_index=3 + wrapped),
                 lambda: efs.adamw_apply([m.g], [m.x], [torch.zeros_like(m.g)], [torch.zeros_like(m.g)], 3 + wrapped, lr=1.0)):
        with pytest.raises(ValueError, match="64 bits"):
            call()
    assert torch.equal(m.x, before)
