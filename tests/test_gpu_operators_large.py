"""The cross entropy at sizes whose offsets pass 32 bits, and prepared updates."""
import gc
import weakref

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2108_00951_amd import binding as efs  # noqa: E402

DEV = "cuda"


def say(*a):
    print(*a, flush=True)


def _reference(h, w, target, dloss, rows):
    """In 64 bits on the device, some words at a time: lse, loss, dh, and dw at `rows`."""
    hd, t = h.double(), h.shape[0]
    parts, at = [], torch.empty(t, dtype=torch.float64, device=DEV)
    step = 1 << 16
    for v in range(0, w.shape[0], step):
        l = hd @ w[v:v + step].double().t()
        parts.append(torch.logsumexp(l, 1))
        here = (target >= v) & (target < v + step)
        at[here] = l[here, target[here] - v]
    lse = torch.logsumexp(torch.stack(parts), 0)
    dh = torch.zeros_like(hd)
    for v in range(0, w.shape[0], step):
        part = w[v:v + step].double()
        p = torch.exp(hd @ part.t() - lse[:, None])
        here = (target >= v) & (target < v + step)
        p[here, target[here] - v] -= 1.0
        dh += (p * dloss.double()[:, None]) @ part
    p = torch.exp(hd @ w[rows].double().t() - lse[:, None])
    p -= (target[:, None] == rows[None, :]).double()
    return lse, lse - at, dh, (p * dloss.double()[:, None]).t() @ hd


@pytest.mark.parametrize("tokens, vocab, hidden", [(5, 600_011, 4096), (90, 540_007, 4097)])
def test_offsets_past_32_bits(tokens, vocab, hidden):
    assert vocab * hidden > 2 ** 31
    say("xent", tokens, vocab, hidden)
    gen = torch.Generator(device=DEV).manual_seed(tokens)
    w = torch.empty((vocab, hidden), dtype=torch.bfloat16, device=DEV).normal_(0.0, 0.02, generator=gen)
    h = torch.randn((tokens, hidden), generator=gen, device=DEV).to(torch.bfloat16)
    target = torch.randint(0, vocab, (tokens,), generator=gen, device=DEV)
    target[-1] = vocab - 1
    dloss = torch.rand(tokens, generator=gen, device=DEV) + 0.5
    ws = efs.new_xent_workspace(tokens, vocab, hidden, w.dtype, DEV)
    loss, lse = torch.empty(tokens, device=DEV), torch.empty(tokens, device=DEV)
    dh, dw = torch.empty_like(h), torch.full_like(w, 7.0)
    efs.xent_forward(h, w, target, loss, lse, ws)
    efs.xent_backward(h, w, target, lse, dloss, dh, dw, ws)
    torch.cuda.synchronize()
    say("reference")
    rows = torch.cat([target, torch.tensor([0, 1, vocab // 2, vocab - 2, vocab - 1], device=DEV)])
    rlse, rloss, rdh, rdw = _reference(h, w, target, dloss, rows)
    # sums of 4096 terms of 2^-7 in 32 bits, and log's rounding
    assert torch.all((lse - rlse).abs() <= 1e-5 * rlse.abs())
    assert torch.all((loss - rloss).abs() <= 1e-5 * rlse.abs())
    # g to 11 bits and the results to 8: elementwise a few of the largest's 2^-8
    for got, want in ((dh, rdh), (dw[rows], rdw)):
        assert float((got.double() - want).norm() / want.norm()) <= 2.0 ** -8
    assert torch.isfinite(dw).all()


def test_prepared_update_keeps_its_tensors():
    layers = [(0, 100, 70)]
    t = {k: torch.randn(7000, device=DEV) for k in ("avg", "x", "m")}
    t["ws"] = efs.new_muon_workspace([(100, 70)], DEV)
    want = t["x"].clone()
    efs.muon_apply(t["avg"], want, t["m"].clone(), layers, t["ws"], 0.9, 0.1)
    x = t["x"]
    call = efs.prepare_muon_apply(t["avg"], t["x"], t["m"], layers, t["ws"], 0.9, 0.1)
    alive = [weakref.ref(v) for k, v in t.items() if k != "x"]
    layers.clear()
    del t
    gc.collect()
    call()
    assert torch.equal(x, want)
    assert all(r() is not None for r in alive)
    del call
    gc.collect()
    assert all(r() is None for r in alive)


def test_tensors_of_more_rows_than_32_bits_count_are_refused():
    """Their low 32 bits would pass for a size."""
    many = torch.empty((2 ** 32 + 8, 1), dtype=torch.bfloat16, device=DEV)
    ws = efs.new_muon_workspace([(8, 1)], DEV)
    with pytest.raises(ValueError, match="32 bits"):
        efs.muon_orthogonalize(many, many, ws)
    with pytest.raises(ValueError, match="32 bits"):
        efs.muon_orthogonalize(many.t(), many.t(), ws)
    with pytest.raises(ValueError, match="32 bits"):
        efs.muon_orthogonalize(torch.ones((8, 1), device=DEV), torch.ones((8, 1), device=DEV), ws, steps=2 ** 32 + 5)
    h = torch.ones((2, 1), dtype=torch.bfloat16, device=DEV)
    target, f = torch.zeros(2, dtype=torch.int64, device=DEV), torch.empty(2, device=DEV)
    ws = efs.new_xent_workspace(2, 8, 1, h.dtype, DEV)
    with pytest.raises(ValueError, match="32 bits"):
        efs.xent_forward(h, many, target, f, torch.empty_like(f), ws)
    flat = torch.zeros(40, device=DEV)
    with pytest.raises(ValueError, match="32 bits"):
        efs.muon_apply(flat, flat.clone(), flat.clone(), [(0, 2 ** 32 + 4, 5)], ws, 0.9, 0.1)
