"""Layer norm and its gradients against plain 64-bit forms."""
import numpy as np
import pytest

from tests import _step

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2108_00951_amd import binding as efs  # noqa: E402

DEV = "cuda"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
SHAPES = [(1, 1), (3, 2), (1, 64), (5, 63), (4, 255), (70, 256), (2, 257), (700, 650), (9, 1024), (5, 1025), (33, 2048),
          (3, 2049), (6, 4096), (2, 4099), (3, 8192), (2, 8200), (3, 16384), (2, 16385), (20, 20000)]


def say(*a):
    print(*a, flush=True)


def rows(rng, shape, kind="gauss"):
    x = rng.standard_normal(shape)
    if kind == "columns":   # a mean in every column, and columns of large values
        x = x + 3.0 * rng.standard_normal(shape[1])
        x[:, :: max(1, shape[1] // 3)] *= 50.0
    elif kind == "offset":
        x = x + 1000.0
    return x.astype(np.float32)


class Call:
    """Inputs on the device and what the two calls make of them."""

    def __init__(self, x, w, b, dy, dtype="fp32", weight_dtype="fp32", eps=1e-5):
        t, f = TYPES[dtype], TYPES[weight_dtype]
        self.dtype, self.weight_dtype, self.eps = dtype, weight_dtype, eps
        self.x, self.dy = (torch.from_numpy(v).to(t).to(DEV) for v in (x, dy))
        self.w, self.b = (None if v is None else torch.from_numpy(v).to(f).to(DEV) for v in (w, b))
        self.run()

    def run(self):
        n, k = self.x.shape
        self.y, self.dx = (torch.full((n, k), 7.0, dtype=self.x.dtype, device=DEV) for _ in range(2))
        self.mean, self.rstd = (torch.full((n,), 7.0, device=DEV) for _ in range(2))
        self.dweight, self.dbias = (torch.full((k,), 7.0, dtype=TYPES[self.weight_dtype], device=DEV) for _ in range(2))
        ws = efs.new_layernorm_workspace(n, k, DEV)
        ws.fill_(0xFF)
        efs.layernorm_forward(self.x, self.w, self.b, self.y, self.mean, self.rstd, eps=self.eps)
        efs.layernorm_backward(self.x, self.w, self.mean, self.rstd, self.dy, self.dx, self.dweight, self.dbias, ws)
        self.out = {k: getattr(self, k) for k in ("y", "mean", "rstd", "dx", "dweight", "dbias")}

    def check(self):
        host = [None if v is None else v.float().cpu().numpy() for v in (self.x, self.w, self.b, self.dy)]
        want = _step.norm(*host, eps=self.eps, dtype=self.dtype, weight_dtype=self.weight_dtype)
        for name, got in self.out.items():
            _step.within(got.float().cpu().numpy(), want[name], name)


def make(n, k, dtype="fp32", weight_dtype="fp32", kind="gauss", affine=True, seed=0, **kw):
    rng = np.random.default_rng(seed + n * 7919 + k)
    w, b = (1.0 + 0.3 * rng.standard_normal(k)).astype(np.float32), rng.standard_normal(k).astype(np.float32)
    return Call(rows(rng, (n, k), kind), w if affine else None, b if affine else None, rows(rng, (n, k)), dtype,
                weight_dtype, **kw)


@pytest.mark.parametrize("n, k", SHAPES)
@pytest.mark.parametrize("dtype, weight_dtype", [("fp32", "fp32"), ("bf16", "fp32"), ("bf16", "bf16"), ("fp32", "bf16")])
def test_norm(n, k, dtype, weight_dtype):
    say("norm", n, k, dtype, weight_dtype)
    make(n, k, dtype, weight_dtype).check()


@pytest.mark.parametrize("kind", ["columns", "offset"])
@pytest.mark.parametrize("n, k", [(50, 300), (7, 3000), (3, 17000)])
def test_norm_of_rows_with_a_mean(n, k, kind):
    make(n, k, kind=kind).check()


@pytest.mark.parametrize("k", [40, 3000, 17000])
def test_without_weights(k):
    make(11, k, affine=False).check()
    c = make(11, k)
    c.b = None
    c.run()
    y = torch.empty_like(c.y)
    efs.layernorm_forward(c.x, c.w, torch.zeros_like(c.w), y)
    assert torch.equal(y, c.y)


@pytest.mark.parametrize("n, k", [(5000, 100), (3000, 1500), (1100, 5000), (600, 16400)])
def test_more_rows_than_workgroups(n, k):
    make(n, k, "bf16").check()


@pytest.mark.parametrize("k", [100, 3000, 17000])
def test_one_of_the_weights_gradients_or_none(k):
    c = make(37, k)
    ws = efs.new_layernorm_workspace(37, k, DEV)
    for dw, db in ((True, False), (False, True), (False, False)):
        dx = torch.empty_like(c.dx)
        got = [torch.empty_like(c.w) if want else None for want in (dw, db)]
        efs.layernorm_backward(c.x, c.w, c.mean, c.rstd, c.dy, dx, *got, ws)
        assert torch.equal(dx, c.dx)
        for g, want in zip(got, (c.dweight, c.dbias)):
            assert g is None or torch.equal(g, want)


@pytest.mark.parametrize("k", [100, 3000, 17000])
def test_in_place(k):
    c = make(37, k, "bf16")
    ws = efs.new_layernorm_workspace(37, k, DEV)
    x = c.x.clone()
    efs.layernorm_forward(x, c.w, c.b, x, eps=c.eps)
    assert torch.equal(x, c.y)
    dy = c.dy.clone()
    efs.layernorm_backward(c.x, c.w, c.mean, c.rstd, dy, dy, None, None, ws)
    assert torch.equal(dy, c.dx)
    x = c.x.clone()
    dw, db = torch.empty_like(c.w), torch.empty_like(c.w)
    efs.layernorm_backward(x, c.w, c.mean, c.rstd, c.dy, x, dw, db, ws)
    assert torch.equal(x, c.dx)
    # (the sums over the rows may be in another order)
    c.out = {"dweight": dw, "dbias": db}
    c.check()


@pytest.mark.parametrize("rows", [1, 2, 31, 33, 1024, 1025])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_weights_gradients_of_few_rows(rows, dtype):
    """By columns of all rows, up to 1,024 of them; in place and with more, by rows."""
    for k in (7, 8, 65, 1000):
        c = make(rows, k, dtype, kind="columns")
        c.check()
        dx, dw, db = c.dy.clone(), torch.empty_like(c.w), torch.empty_like(c.w)
        efs.layernorm_backward(c.x, c.w, c.mean, c.rstd, dx, dx, dw, db, efs.new_layernorm_workspace(rows, k, DEV))
        assert torch.equal(dx, c.dx)
        c.out = {"dweight": dw, "dbias": db}
        c.check()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("k", [77, 2501, 16999])
def test_strided_rows_leave_what_lies_between(k, dtype):
    c = make(13, k, dtype)

    def wide(v=None):
        t = torch.full((13, k + 9), 5.0, dtype=c.x.dtype, device=DEV)
        if v is not None:
            t[:, 1:k + 1] = v
        return t, t[:, 1:k + 1]
    (_, x), (_, dy), (wy, y), (wdx, dx) = wide(c.x), wide(c.dy), wide(), wide()
    dw, db = torch.empty_like(c.w), torch.empty_like(c.w)
    efs.layernorm_forward(x, c.w, c.b, y, eps=c.eps)
    efs.layernorm_backward(x, c.w, c.mean, c.rstd, dy, dx, dw, db, efs.new_layernorm_workspace(13, k, DEV))
    for got, want in ((y, c.y), (dx, c.dx), (dw, c.dweight), (db, c.dbias)):
        assert torch.equal(got, want)
    for w in (wy, wdx):
        assert torch.all(w[:, :1] == 5.0) and torch.all(w[:, k + 1:] == 5.0)


@pytest.mark.parametrize("k", [60, 3000, 17000])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_special_values_stay_in_their_row(k, bad):
    c = make(9, k)
    c.x[4, k // 2] = bad
    good = {name: v.clone() for name, v in c.out.items()}
    c.run()
    others = [0, 1, 2, 3, 5, 6, 7, 8]
    for name in ("y", "dx", "mean", "rstd"):
        assert torch.equal(c.out[name][others], good[name][others]), name
    assert torch.isnan(c.y[4]).any() and torch.isnan(c.dx[4]).any()


def test_constant_rows():
    for k in (64, 3000, 17000):
        x = np.full((3, k), 0.1, np.float32)
        x[1] = 0.0
        x[2] = -1e6
        c = Call(x, None, np.linspace(-1, 1, k).astype(np.float32), np.ones((3, k), np.float32))
        # what is left of x - mean is a rounding of the mean's, times 1 / sqrt(eps)
        slack = 2.0 ** -22 * np.abs(x[:, :1]) * 1e-5 ** -0.5
        assert np.all(np.abs(c.y.cpu().numpy() - np.linspace(-1, 1, k).astype(np.float32)) <= slack + 2.0 ** -22)
        y = torch.empty(3, k, device=DEV)
        efs.layernorm_forward(torch.zeros(3, k, device=DEV), None, None, y, eps=0.0)
        assert torch.all(torch.isnan(y))


def test_no_rows():
    w = torch.ones(50, device=DEV)
    x, none = torch.empty(0, 50, device=DEV), torch.empty(0, device=DEV)
    dw, db = torch.full_like(w, 3.0), torch.full_like(w, 3.0)
    efs.layernorm_forward(x, w, w, x.clone())
    efs.layernorm_backward(x, w, none, none, x, x.clone(), dw, db, efs.new_layernorm_workspace(0, 50, DEV))
    assert torch.all(dw == 0.0) and torch.all(db == 0.0)


def test_the_same_bits_each_time():
    for n, k in ((3000, 200), (500, 4000), (300, 17000)):
        c = make(n, k)
        first = {name: v.clone() for name, v in c.out.items()}
        c.run()
        for name, v in first.items():
            assert torch.equal(c.out[name], v), name


@pytest.mark.parametrize("k", [24, 1500])
def test_gradients_against_differences(k):
    c = make(6, k, eps=1e-3)
    weight = c.dy.double()

    def loss(x, w, b):
        y = torch.empty_like(c.y)
        efs.layernorm_forward(x, w, b, y, eps=c.eps)
        return float((y.double() * weight).sum())
    step = 2.0 ** -6
    for name, at in (("x", (2, 3)), ("x", (5, k - 1)), ("w", (1,)), ("b", (k // 2,))):
        grad = {"x": c.dx, "w": c.dweight, "b": c.dbias}[name][at]
        args = {"x": c.x, "w": c.w, "b": c.b}
        sides = []
        for s in (step, -step):
            moved = args[name].clone()
            moved[at] += s
            sides.append(loss(**dict(args, **{name: moved})))
        # each y is off by 2^-22 of up to 8; the third derivative adds its step^2 / 6
        slack = 2.0 ** -19 * float(weight.abs().sum()) / step + step ** 2 * 10.0
        assert abs((sides[0] - sides[1]) / (2 * step) - float(grad)) <= slack, name


@pytest.mark.parametrize("n, k", [(700, 650), (1, 1024), (768, 64), (769, 64), (40, 3000), (1025, 650), (300, 4096)])
@pytest.mark.parametrize("mean", [0.0, 7.5, 8.5, 1000.0, 10000.0, 131072.0])
def test_weights_gradient_of_rows_with_a_mean_between_two_values(n, k, mean):
    """Rows whose mean lies 0.45 of a step behind an fp32 value, so that what is stored
    is off by that in all of them, with gradients of one sign, which add it up (from
    1,000 on: smaller means lie anywhere).

    Limit, u = 2^-24: x - mean is rounded once.  No value passes more than 16 additions
    of its thread, 6 of its wave and 16 of the waves, so that what the mean's rounding
    left is off by 40 u of the mean magnitude of x - mean, rstd by 24 u, and h with its
    three roundings by 66 u |h| + 41 u mean|h|; the sums over the rows pass at most 128
    additions."""
    rng = np.random.default_rng(n + k)
    ulp = float(np.spacing(np.float32(max(mean, 1.0))))
    q = np.rint(rng.standard_normal((n, k)) / ulp)
    q -= np.rint(q.mean(1, keepdims=True))
    more = np.rint(0.45 * k) - q.sum(1, keepdims=True)
    q += np.sign(more) * (np.arange(k) < np.abs(more))
    exact = mean + ulp * q
    x = exact.astype(np.float32)
    assert mean < 1000.0 or np.array_equal(x, exact)
    exact = x.astype(np.float64)
    dy = (0.5 + rng.random((n, k))).astype(np.float32)
    c = Call(x, None, None, dy)
    d = exact - exact.mean(1, keepdims=True)
    h = d / np.sqrt((d * d).mean(1, keepdims=True) + float(np.float32(1e-5)))
    size = np.abs(h).mean(1, keepdims=True)
    limit = _step.EPS32 * (dy * (66 * np.abs(h) + 41 * size) + 128 * dy * np.abs(h)).sum(0)
    want = (dy.astype(np.float64) * h).sum(0)
    _step.within(c.dweight.cpu().numpy(), (want, limit), "dweight")
    left = exact.mean(1) - c.mean.double().cpu().numpy()
    uncorrected = (dy * left[:, None] / np.sqrt((d * d).mean(1, keepdims=True) + 1e-5)).sum(0)
    # an uncorrected sum fails
    assert mean < 2000.0 or np.all(np.abs(uncorrected) > 2 * limit)
    for into in ("x", "dy"):   # in place: by rows, whatever their number
        x, dy = c.x.clone(), c.dy.clone()
        dw, db = torch.empty_like(c.dweight), torch.empty_like(c.dbias)
        efs.layernorm_backward(x, None, c.mean, c.rstd, dy, x if into == "x" else dy, dw, db,
                               efs.new_layernorm_workspace(n, k, DEV))
        _step.within(dw.cpu().numpy(), (want, limit), "dweight in place of " + into)
