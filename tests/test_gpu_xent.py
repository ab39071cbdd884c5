"""Cross entropy and its gradients (xent_forward, xent_backward) against their
formulas in 64 bits, within elementwise limits (tests/_dense.py)."""
import numpy as np
import pytest

from tests import _dense

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2108_00951_amd import binding as efs  # noqa: E402

DEV = "cuda"
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
# tokens, vocab, hidden: one of each, around the steps (32, 64), the tiles
# (128, 256) and the pack's 64, odd ones, many words for few tokens
SIZES = [(1, 1, 1), (1, 2, 64), (1, 1000, 64), (2, 33, 31), (3, 4097, 65), (16, 257, 128), (17, 5003, 33),
         (31, 129, 96), (32, 2048, 64), (33, 300, 100), (64, 1023, 200), (65, 64, 64), (127, 130, 63),
         (129, 255, 257), (300, 777, 130), (513, 1500, 70)]


def say(*a):
    print(*a, flush=True)


def inputs(tokens, vocab, hidden, dtype, seed=0, ignored=0.2, scale=1.0):
    rng = np.random.default_rng([seed, tokens, vocab, hidden])
    h = torch.from_numpy(rng.standard_normal((tokens, hidden)).astype(np.float32) * np.float32(scale)).to(DTYPES[dtype])
    w = torch.from_numpy(rng.standard_normal((vocab, hidden)).astype(np.float32) *
                         np.float32(2.0 / np.sqrt(hidden) / scale)).to(DTYPES[dtype])
    target = rng.integers(0, vocab, tokens)
    target[rng.random(tokens) < ignored] = -100
    dloss = rng.standard_normal(tokens).astype(np.float32)
    return h, w, torch.from_numpy(target), torch.from_numpy(dloss)


def call(h, w, target, dloss, stream=None, **kw):
    """All four results, every buffer full of other values before."""
    t, v = h.shape[0], w.shape[0]
    ws = efs.new_xent_workspace(t, v, h.shape[1], h.dtype, DEV)
    ws.fill_(0xFF)
    out = {k: torch.full((t,), 9.0, device=DEV) for k in ("loss", "lse")}
    out["dh"], out["dw"] = (torch.full(x.shape, 9.0, dtype=x.dtype, device=DEV) for x in (h, w))
    if stream is not None:
        torch.cuda.synchronize()
    efs.xent_forward(h, w, target, out["loss"], out["lse"], ws, stream=stream, **kw)
    out["status"] = ws[:4].clone() if stream is None else None
    efs.xent_backward(h, w, target, out["lse"], dloss, out["dh"], out["dw"], ws, stream=stream, **kw)
    if stream is not None:
        torch.cuda.synchronize()
    return out


def check(got, h, w, target, dloss, dtype, what=""):
    want, limits = _dense.xent(h.float().cpu().numpy(), w.float().cpu().numpy(), target.cpu().numpy(),
                               dloss.cpu().numpy())
    for k in ("lse", "loss", "dh", "dw"):
        g = got[k].float().cpu().numpy()
        # bf16 affects the gradients only; 2^-126: results below that are not normal
        limit = limits[dtype if k in ("dh", "dw") else "fp32"][k] + 2.0 ** -126
        off = np.abs(g - want[k])
        assert np.all(off <= limit), "%s %s: %g times the limit" % (what, k, float(np.max(off / limit)))
    return want


@pytest.mark.parametrize("tokens, vocab, hidden", SIZES)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_sizes(tokens, vocab, hidden, dtype):
    say("xent", tokens, vocab, hidden, dtype)
    h, w, target, dloss = inputs(tokens, vocab, hidden, dtype)
    got = call(*(x.to(DEV) for x in (h, w, target, dloss)))
    check(got, h, w, target, dloss, dtype)
    assert not got["status"].any()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_large_tiles_and_several_pieces(dtype, monkeypatch):
    """Enough tiles for the larger kind; more words than a piece holds."""
    tokens, vocab, hidden = (2100, 20011, 64) if dtype == "fp32" else (4200, 20011, 64)
    say("xent", tokens, vocab, hidden, dtype)
    h, w, target, dloss = inputs(tokens, vocab, hidden, dtype)
    # two copies of g for the whole vocabulary would not fit
    assert efs.xent_workspace_bytes(tokens, vocab, hidden, h.dtype) < 2 * tokens * vocab * (4 if dtype == "fp32" else 2)
    got = call(*(x.to(DEV) for x in (h, w, target, dloss)))
    check(got, h, w, target, dloss, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("pad, shift", [(0, 1), (3, 0), (8, 0), (64, 2)])
def test_strides_and_alignment(dtype, pad, shift):
    """Rows further apart than they are long, off any alignment: the same bits
    as contiguous tensors, and nothing between the rows is written."""
    h, w, target, dloss = (x.to(DEV) for x in inputs(70, 300, 128, dtype))
    want = call(h, w, target, dloss)

    def view(x, fill=5.0):
        rows, cols = x.shape
        buf = torch.full((rows * (cols + pad) + shift,), fill, dtype=x.dtype, device=DEV)
        v = buf[shift:].view(rows, cols + pad)
        return v[:, :cols], v[:, cols:]
    (hv, _), (wv, _), (dh, gap_h), (dw, gap_w) = view(h), view(w), view(h), view(w)
    hv.copy_(h)
    wv.copy_(w)
    ws = efs.new_xent_workspace(70, 300, 128, h.dtype, DEV)
    loss, lse = torch.empty(70, device=DEV), torch.empty(70, device=DEV)
    efs.xent_forward(hv, wv, target, loss, lse, ws)
    efs.xent_backward(hv, wv, target, lse, dloss, dh, dw, ws)
    for k, v in (("loss", loss), ("lse", lse), ("dh", dh), ("dw", dw)):
        assert torch.equal(v, want[k]), k
    assert torch.all(gap_h == 5.0) and torch.all(gap_w == 5.0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("tokens, hidden", [(5, 128), (20, 65), (50, 200), (100, 129)])
@pytest.mark.parametrize("pad, shift", [(0, 1), (8, 0), (5, 3)])
def test_strides_and_alignment_of_few_tokens(dtype, tokens, hidden, pad, shift):
    """The path that reads the head where it is, aligned to whole steps or not."""
    h, w, target, dloss = inputs(tokens, 700, hidden, dtype)

    def view(x):
        rows, cols = x.shape
        buf = torch.full((rows * (cols + pad) + shift,), float("nan"), dtype=x.dtype, device=DEV)
        return buf[shift:].view(rows, cols + pad)[:, :cols]
    hv, wv, dh, dw = view(h), view(w), view(h), view(w)
    hv.copy_(h)
    wv.copy_(w)
    target, dloss = target.to(DEV), dloss.to(DEV)
    ws = efs.new_xent_workspace(tokens, 700, hidden, h.dtype, DEV)
    got = {"loss": torch.empty(tokens, device=DEV), "lse": torch.empty(tokens, device=DEV), "dh": dh, "dw": dw}
    efs.xent_forward(hv, wv, target, got["loss"], got["lse"], ws)
    efs.xent_backward(hv, wv, target, got["lse"], dloss, dh, dw, ws)
    check(got, h, w, target, dloss, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -3.3e38])
@pytest.mark.parametrize("hidden", [64, 70])
def test_ignored_tokens_hold_anything(dtype, bad, hidden):
    h, w, target, dloss = inputs(40, 500, hidden, dtype)
    target[::3] = -100
    clean = h.clone()
    clean[::3] = 0.0
    h[::3] = bad
    dloss[::3] = bad
    got = call(*(x.to(DEV) for x in (h, w, target, dloss)))
    check(got, clean, w, target, torch.where(target == -100, torch.zeros(()), dloss), dtype)
    for k in ("loss", "lse", "dh"):
        assert torch.all(got[k][::3] == 0.0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_every_token_ignored(dtype):
    h, w, target, dloss = (x.to(DEV) for x in inputs(20, 300, 64, dtype))
    got = call(torch.full_like(h, float("nan")), w, torch.full_like(target, -100), dloss)
    for k in ("loss", "lse", "dh", "dw"):
        assert torch.all(got[k] == 0.0), k


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_targets_outside_the_vocabulary_are_reported(dtype):
    h, w, target, dloss = inputs(40, 500, 64, dtype)
    target[3], target[17], target[30] = 500, -1, 2 ** 40
    got = call(*(x.to(DEV) for x in (h, w, target, dloss)))
    check(got, h, w, target, dloss, dtype)
    assert int(got["status"].cpu().numpy().view("<u4")[0]) == efs.XENT_BAD_TARGET
    # another ignore_index: -100 is then bad as well, 500 is not
    target[:] = 7
    target[5] = 500
    ws = efs.new_xent_workspace(40, 500, 64, h.dtype, DEV)
    loss, lse = torch.empty(40, device=DEV), torch.empty(40, device=DEV)
    efs.xent_forward(h.to(DEV), w.to(DEV), target.to(DEV), loss, lse, ws, ignore_index=500)
    assert efs.xent_status(ws) == 0 and float(loss[5]) == 0.0 and float(loss[6]) > 0.0
    efs.xent_forward(h.to(DEV), w.to(DEV), target.to(DEV), loss, lse, ws)
    assert efs.xent_status(ws) == efs.XENT_BAD_TARGET


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_special_values_stay_with_their_token(dtype):
    h, w, target, dloss = (x.to(DEV) for x in inputs(40, 500, 64, dtype, ignored=0.0))
    want = call(h, w, target, dloss)
    h[11, 5] = float("inf")
    h[12, 6] = float("nan")
    got = call(h, w, target, dloss)
    for k in ("loss", "lse", "dh"):
        rest = torch.ones(40, dtype=torch.bool, device=DEV)
        rest[11:13] = False
        assert torch.equal(got[k][rest], want[k][rest]), k
        assert torch.all(torch.isnan(got[k][12])), k
        assert not torch.isfinite(got[k][11]).any(), k
    assert torch.isnan(got["dw"]).all()


@pytest.mark.parametrize("scale", [1e-15, 1e-6, 1e6, 1e15])
def test_tensors_of_any_magnitude(scale):
    """The split form is scaled to each tensor."""
    h, w, target, dloss = inputs(50, 400, 96, "fp32", scale=scale)
    got = call(*(x.to(DEV) for x in (h, w, target, dloss)))
    check(got, h, w, target, dloss, "fp32")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_logits_far_apart(dtype):
    """Probabilities of exactly one and zero: maxima in the first and the last
    tile, logits thousands apart."""
    h, w, target, dloss = inputs(60, 1000, 64, dtype, ignored=0.0)
    w[0] *= 200.0
    w[999] *= 300.0
    got = call(*(x.to(DEV) for x in (h, w, target, dloss)))
    check(got, h, w, target, dloss, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_no_tokens(dtype):
    w = torch.ones((30, 20), dtype=DTYPES[dtype], device=DEV)
    h = torch.empty((0, 20), dtype=DTYPES[dtype], device=DEV)
    none = torch.empty(0, device=DEV)
    got = call(h, w, torch.empty(0, dtype=torch.int64, device=DEV), none)
    assert torch.all(got["dw"] == 0.0)


def test_gradients_against_differences():
    """Along random directions, central differences of the 64-bit loss: their
    own error is the third derivative's, 1e-8 of the loss at this step."""
    h, w, target, dloss = inputs(30, 200, 40, "fp32", ignored=0.1)
    got = call(*(x.to(DEV) for x in (h, w, target, dloss)))
    hn, wn, tn, dn = (x.numpy().astype(np.float64) if x.is_floating_point() else x.numpy() for x in (h, w, target, dloss))
    rng = np.random.default_rng(1)
    step = 1e-4

    def total(a, b):
        return float((_dense.xent(a, b, tn, dn)[0]["loss"] * dn).sum())
    for _ in range(5):
        dh, dw = rng.standard_normal(hn.shape), rng.standard_normal(wn.shape)
        slope = (total(hn + step * dh, wn + step * dw) - total(hn - step * dh, wn - step * dw)) / (2 * step)
        mine = float((got["dh"].double().cpu().numpy() * dh).sum() + (got["dw"].double().cpu().numpy() * dw).sum())
        size = np.linalg.norm(got["dh"].cpu().numpy()) * np.linalg.norm(dh) + \
            np.linalg.norm(got["dw"].cpu().numpy()) * np.linalg.norm(dw)
        assert abs(mine - slope) <= 1e-5 * size


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_the_same_every_time_and_on_a_side_stream(dtype):
    args = [x.to(DEV) for x in inputs(200, 3000, 130, dtype)]
    want = call(*args)
    for stream in (None, torch.cuda.Stream()):
        got = call(*args, stream=stream)
        for k in ("loss", "lse", "dh", "dw"):
            assert torch.equal(got[k], want[k]), k


@pytest.mark.parametrize("tokens", [1, 150])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_in_a_graph(dtype, tokens):
    h, w, target, dloss = (x.to(DEV) for x in inputs(tokens, 1000, 70, dtype, ignored=0.0))
    ws = efs.new_xent_workspace(tokens, 1000, 70, h.dtype, DEV)
    out = [torch.empty(tokens, device=DEV), torch.empty(tokens, device=DEV), torch.empty_like(h), torch.empty_like(w)]

    def step():
        efs.xent_forward(h, w, target, out[0], out[1], ws)
        efs.xent_backward(h, w, target, out[1], dloss, out[2], out[3], ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):   # new inputs and eager work between the replays
        h.add_(0.01 * k)
        step()
        want = [x.clone() for x in out]
        for x in out:
            x.fill_(3.0)
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(out, want):
            assert torch.equal(x, y)


def test_binding_refuses_what_the_kernels_do_not_take():
    h, w, target, dloss = (x.to(DEV) for x in inputs(5, 20, 8, "fp32"))
    ws = efs.new_xent_workspace(5, 20, 8, h.dtype, DEV)
    f = torch.empty(5, device=DEV)
    for bad in ((h.double(), w.double(), target), (h, w.to(torch.bfloat16), target), (h, w, target.int()),
                (torch.empty(8, 5, device=DEV).t(), w, target)):
        with pytest.raises(TypeError):
            efs.xent_forward(*bad, f, f, ws)
    with pytest.raises(ValueError):
        efs.xent_forward(h, w[:, :7], target, f, f, ws)
    with pytest.raises(ValueError):
        efs.xent_forward(h, w, target[:4], f, f, ws)
    with pytest.raises(efs.EfsError):
        efs.xent_forward(h, w, target, f, f, ws[:64])
    with pytest.raises(efs.EfsError):   # dh must not be h
        efs.xent_backward(h, w, target, f, dloss, h, torch.empty_like(w), ws)
    with pytest.raises(ValueError):
        efs.xent_backward(h, w, target, f, dloss, torch.empty_like(w), torch.empty_like(w), ws)


@pytest.mark.parametrize("tokens", [9, 150])
def test_gradients_beside_their_tensors(tokens):
    """dh and dw in other columns of the rows that hold h and w."""
    h, w, target, dloss = (x.to(DEV) for x in inputs(tokens, 700, 70, "fp32"))
    want = call(h, w, target, dloss)
    both_h, both_w = torch.cat((h, h), 1), torch.cat((w, w), 1)
    ws = efs.new_xent_workspace(tokens, 700, 70, h.dtype, DEV)
    efs.xent_backward(both_h[:, :70], both_w[:, :70], target, want["lse"], dloss, both_h[:, 70:], both_w[:, 70:], ws)
    for k, both, x in (("dh", both_h, h), ("dw", both_w, w)):
        assert torch.equal(both[:, 70:], want[k]), k
        assert torch.equal(both[:, :70], x), k


@pytest.mark.parametrize("hidden, pad, shift", [(511, 0, 0), (512, 0, 0), (513, 2, 1), (1024, 0, 0), (1027, 0, 3), (2500, 4, 0),
                                                (4095, 1, 0), (4096, 0, 1), (4097, 0, 0)])
@pytest.mark.parametrize("tokens", [1, 2, 3, 4])
def test_one_to_four_tokens_of_long_rows(tokens, hidden, pad, shift):
    """Rows that a workgroup holds whole, of any length and alignment, and just
    shorter and longer ones; a vocabulary of 331 is no multiple of anything."""
    h, w, target, dloss = inputs(tokens, 331, hidden, "fp32", ignored=0.3)
    buf = torch.zeros(331 * (hidden + pad) + shift, device=DEV)
    rows = buf[shift:].view(331, hidden + pad)[:, :hidden]
    rows.copy_(w)
    got = call(h.to(DEV), rows, target.to(DEV), dloss.to(DEV))
    check(got, h, w, target, dloss, "fp32")


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_an_ignored_token_of_a_long_row_holds_anything(bad):
    h, w, target, dloss = (x.to(DEV) for x in inputs(3, 90, 700, "fp32", ignored=0.0))
    target[1] = -100
    want = call(h, w, target, dloss)
    h[1], dloss[1] = bad, bad
    got = call(h, w, target, dloss)
    for k in ("loss", "lse", "dh", "dw"):
        assert torch.equal(got[k], want[k]), k


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("tokens, vocab, hidden", [(40, 2000, 256), (65, 500, 64), (150, 2000, 256), (700, 8000, 64)])
@pytest.mark.parametrize("gap, spread", [(30.0, 1.0), (40.0, 1.0), (0.0, 6.0)])
def test_words_that_no_token_finds_likely(dtype, tokens, vocab, hidden, gap, spread):
    """Targets' logits far above the others', or logits of a standard deviation
    of 12: the rows of dw of words with tiny probabilities alone are as near,
    each for itself, as those of the targets."""
    say("xent", tokens, vocab, hidden, dtype, gap, spread)
    h, w, target, dloss = inputs(tokens, vocab, hidden, dtype, seed=3)
    counts = target >= 0
    h = h.float() * spread
    h[counts] += w[target[counts]].float() * (gap / 4.0)   # |w|^2 is about 4
    h = h.to(DTYPES[dtype])
    got = call(*(x.to(DEV) for x in (h, w, target, dloss)))
    check(got, h, w, target, dloss, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_no_tokens_have_no_bad_target(dtype):
    w = torch.ones((30, 20), dtype=DTYPES[dtype], device=DEV)
    h = torch.empty((0, 20), dtype=DTYPES[dtype], device=DEV)
    none, target = torch.empty(0, device=DEV), torch.empty(0, dtype=torch.int64, device=DEV)
    ws = efs.new_xent_workspace(0, 30, 20, h.dtype, DEV)
    ws.fill_(0xFF)
    efs.xent_forward(h, w, target, none, none, ws)
    assert efs.xent_status(ws) == 0
    ws.fill_(0xFF)
    efs.xent_backward(h, w, target, none, none, h, torch.empty_like(w), ws)
    assert efs.xent_status(ws) == 0


def test_a_token_between_the_rows_of_a_gradient():
    h, w, target, dloss = (x.to(DEV) for x in inputs(1, 300, 64, "fp32", ignored=0.0))
    want = call(h, w, target, dloss)
    both = torch.full((300, 192), 5.0, device=DEV)
    both[7, 64:128], both[9, 128:] = h[0], 9.0
    ws = efs.new_xent_workspace(1, 300, 64, h.dtype, DEV)
    efs.xent_backward(both[7:8, 64:128], w, target, want["lse"], dloss, both[9:10, 128:], both[:, :64], ws)
    assert torch.equal(both[:, :64], want["dw"]) and torch.equal(both[9:10, 128:], want["dh"])
    assert torch.equal(both[7, 64:128], h[0]) and torch.all(both[10:, 64:] == 5.0)
    with pytest.raises(efs.EfsError, match="must not overlap"):
        efs.xent_backward(both[7:8, 63:127], w, target, want["lse"], dloss, both[9:10, 128:], both[:, :64], ws)


# Above 128 tokens everything is laid out first, in both directions and types.
PACKED = 150


@pytest.mark.parametrize("scale", [1e-15, 1e-6, 1e6, 1e15])
def test_tensors_of_any_magnitude_laid_out(scale):
    """The split form is scaled to each tensor."""
    h, w, target, dloss = inputs(PACKED, 400, 96, "fp32", scale=scale)
    got = call(*(x.to(DEV) for x in (h, w, target, dloss)))
    check(got, h, w, target, dloss, "fp32")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("tokens", [40, PACKED])
def test_tokens_and_weights_of_many_magnitudes(dtype, tokens):
    """Within one call: rows of h from 2^-10 to 1, weights from 2^-10 to 1."""
    h, w, target, dloss = inputs(tokens, 400, 96, dtype)
    rng = np.random.default_rng(2)
    h = (h.float() * torch.from_numpy(2.0 ** rng.integers(-10, 1, (tokens, 1))).float()).to(DTYPES[dtype])
    dloss = dloss * torch.from_numpy(2.0 ** rng.integers(-10, 1, tokens)).float()
    got = call(*(x.to(DEV) for x in (h, w, target, dloss)))
    check(got, h, w, target, dloss, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -3.3e38])
@pytest.mark.parametrize("hidden", [64, 70])
def test_ignored_tokens_hold_anything_laid_out(dtype, bad, hidden):
    h, w, target, dloss = inputs(PACKED, 500, hidden, dtype)
    target[::3] = -100
    clean = h.clone()
    clean[::3] = 0.0
    h[::3] = bad
    dloss[::3] = bad
    got = call(*(x.to(DEV) for x in (h, w, target, dloss)))
    check(got, clean, w, target, torch.where(target == -100, torch.zeros(()), dloss), dtype)
    for k in ("loss", "lse", "dh"):
        assert torch.all(got[k][::3] == 0.0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_every_token_ignored_laid_out(dtype):
    h, w, target, dloss = (x.to(DEV) for x in inputs(PACKED, 300, 64, dtype))
    got = call(torch.full_like(h, float("nan")), w, torch.full_like(target, -100), torch.full_like(dloss, float("inf")))
    for k in ("loss", "lse", "dh", "dw"):
        assert torch.all(got[k] == 0.0), k
    assert not got["status"].any()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_targets_outside_the_vocabulary_are_reported_laid_out(dtype):
    h, w, target, dloss = inputs(PACKED, 500, 64, dtype)
    target[3], target[17], target[130] = 500, -1, 2 ** 40
    dev = [x.to(DEV) for x in (h, w, target, dloss)]
    got = call(*dev)
    check(got, h, w, target, dloss, dtype)
    assert int(got["status"].cpu().numpy().view("<u4")[0]) == efs.XENT_BAD_TARGET
    ws = efs.new_xent_workspace(PACKED, 500, 64, h.dtype, DEV)
    ws.fill_(0xFF)
    efs.xent_backward(*dev[:3], got["lse"], dev[3], torch.empty_like(dev[0]), torch.empty_like(dev[1]), ws)
    assert efs.xent_status(ws) == efs.XENT_BAD_TARGET
    # another ignore_index: -100 is then bad as well, 500 is not
    target[:] = 7
    target[5] = 500
    loss, lse = torch.empty(PACKED, device=DEV), torch.empty(PACKED, device=DEV)
    efs.xent_forward(dev[0], dev[1], target.to(DEV), loss, lse, ws, ignore_index=500)
    assert efs.xent_status(ws) == 0 and float(loss[5]) == 0.0 and float(loss[6]) > 0.0
    efs.xent_forward(dev[0], dev[1], target.to(DEV), loss, lse, ws)
    assert efs.xent_status(ws) == efs.XENT_BAD_TARGET


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_special_values_stay_with_their_token_laid_out(dtype):
    h, w, target, dloss = (x.to(DEV) for x in inputs(PACKED, 500, 64, dtype, ignored=0.0))
    want = call(h, w, target, dloss)
    h[11, 5] = float("inf")
    h[112, 6] = float("nan")
    got = call(h, w, target, dloss)
    rest = torch.ones(PACKED, dtype=torch.bool, device=DEV)
    rest[11] = rest[112] = False
    for k in ("loss", "lse", "dh"):
        assert torch.equal(got[k][rest], want[k][rest]), k
        assert torch.all(torch.isnan(got[k][112])), k
        assert not torch.isfinite(got[k][11]).any(), k
    assert torch.isnan(got["dw"]).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_logits_far_apart_laid_out(dtype):
    """Probabilities of exactly one and zero: maxima in the first and the last
    tile, logits thousands apart."""
    h, w, target, dloss = inputs(PACKED, 1000, 64, dtype, ignored=0.0)
    w[0] *= 200.0
    w[999] *= 300.0
    got = call(*(x.to(DEV) for x in (h, w, target, dloss)))
    check(got, h, w, target, dloss, dtype)


def test_gradients_against_differences_laid_out():
    """As above, with more tokens."""
    h, w, target, dloss = inputs(PACKED, 200, 40, "fp32", ignored=0.1)
    got = call(*(x.to(DEV) for x in (h, w, target, dloss)))
    hn, wn, tn, dn = (x.numpy().astype(np.float64) if x.is_floating_point() else x.numpy() for x in (h, w, target, dloss))
    rng = np.random.default_rng(1)
    step = 1e-4

    def total(a, b):
        return float((_dense.xent(a, b, tn, dn)[0]["loss"] * dn).sum())
    for _ in range(5):
        dh, dw = rng.standard_normal(hn.shape), rng.standard_normal(wn.shape)
        slope = (total(hn + step * dh, wn + step * dw) - total(hn - step * dh, wn - step * dw)) / (2 * step)
        mine = float((got["dh"].double().cpu().numpy() * dh).sum() + (got["dw"].double().cpu().numpy() * dw).sum())
        size = np.linalg.norm(got["dh"].cpu().numpy()) * np.linalg.norm(dh) + \
            np.linalg.norm(got["dw"].cpu().numpy()) * np.linalg.norm(dw)
        assert abs(mine - slope) <= 1e-5 * size


# By the rule for tiles on 256 compute units: dh of 256 x 256; the logits and g of
# 256 x 256, dh of 128 x 128; dw of 256 x 256; dw of 128 x 128; the logits and g of
# 128 x 128; dh of 128 x 128.
@pytest.mark.parametrize("tokens, vocab, hidden", [(3999, 301, 4001), (4001, 3990, 70), (150, 4001, 3999),
                                                   (150, 2800, 2900), (2040, 2040, 130), (1500, 260, 2000)])
@pytest.mark.parametrize("gap", [0.0, 30.0])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_every_product_with_every_tile(dtype, gap, tokens, vocab, hidden):
    say("xent", tokens, vocab, hidden, dtype, gap)
    h, w, target, dloss = inputs(tokens, vocab, hidden, dtype, seed=5)
    if gap:   # the targets' logits above the others'; |w|^2 is about 4
        counts = target >= 0
        h = h.float()
        h[counts] += w[target[counts]].float() * (gap / 4.0)
        h = h.to(DTYPES[dtype])
    got = call(*(x.to(DEV) for x in (h, w, target, dloss)))
    check(got, h, w, target, dloss, dtype)
