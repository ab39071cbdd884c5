"""The example of a step with lookup, norm, loss and both updates runs, and its
gradients are those of the model."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from examples import next_word_step as example  # noqa: E402


def test_it_runs():
    losses, density = example.train(8, 2, tokens=300)
    assert len(losses) == 8 and all(math.isfinite(v) for v in losses)
    assert 0.0 < density < 1.0


def test_its_gradients():
    model = example.Model("cuda")
    worker = example.Worker(model, 0, 200, "cuda")
    pairs = torch.arange(example.VOCAB * example.CHOICES, device="cuda").view(-1, example.CHOICES) % example.VOCAB
    word, after = worker.batch(pairs)
    loss = worker.gradient(model, word, after)
    x = model.x.double().cpu().requires_grad_()
    table, mix, weight, bias = model.views(x)
    word, after = word.cpu(), after.cpu()
    there = word != example.IGNORE
    v = torch.where(there[:, None], table[torch.where(there, word, 0)] * example.SCALE, 0.0)
    h = v @ mix
    c = h - h.mean(1, keepdim=True)
    y = c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5) * weight + bias
    want = torch.nn.functional.cross_entropy(y @ table.t(), after, ignore_index=example.IGNORE)
    want.backward()
    assert abs(float(loss) - want.item()) <= 1e-5 * want.item()
    # products of fp32 and of 22 bits, sums of up to 1,000 terms
    for got, ref in zip(model.views(worker.g), model.views(x.grad)):
        assert float((got.cpu().double() - ref).norm() / ref.norm()) <= 2.0 ** -15
