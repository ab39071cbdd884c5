"""Plain 64-bit forms of the orthogonalised update and of the cross entropy,
and how far 32-bit arithmetic may be from them."""
import numpy as np

COEFFS = (3.4445, -4.7750, 2.0315)
SLACK = 2.0 ** -20


def newton_schulz(u, steps=5, coeffs=COEFFS, eps=1e-7, dtype=np.float64):
    """One matrix; the products in `dtype`."""
    a, b, c = (dtype(np.float32(v)) for v in coeffs)
    x = u.astype(dtype)
    if x.shape[0] > x.shape[1]:
        x = x.T
    x = x / (np.sqrt((x * x).sum(dtype=np.float64)).astype(dtype) + dtype(np.float32(eps)))
    for _ in range(steps):
        g = x @ x.T
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.T if u.shape[0] > u.shape[1] else x


def relative(got, want):
    """2-norm of the difference over that of `want`."""
    d = np.linalg.norm(np.asarray(got, np.float64) - want)
    n = np.linalg.norm(want)
    return d / n if n else d


def ortho_limit(u, **kw):
    """What an orthogonalisation in 32 bits may be off by: three times what
    plain binary32 products are on this input (they are as good as the
    operands' 22 to 24 bits; the steps multiply what is lost by up to 3.4 each,
    on the directions of small singular values), and 2^-20."""
    return 3.0 * relative(newton_schulz(u, dtype=np.float32, **kw), newton_schulz(u, **kw)) + SLACK


def matrix(rng, kind, rows, cols):
    g = rng.standard_normal((rows, cols))
    if kind == "lowrank":
        r = max(1, min(rows, cols) // 8)
        g = rng.standard_normal((rows, r)) @ rng.standard_normal((r, cols)) / np.sqrt(r) + 0.02 * g
    elif kind == "tiny":
        g *= 1e-12
    elif kind == "huge":
        g *= 1e15
    elif kind == "one":   # a single entry
        g = np.zeros((rows, cols))
        g[rows // 2, cols // 3] = -3.0
    return g.astype(np.float32)


def xent(h, w, target, dloss, ignore=-100):
    """loss, lse, dh, dw in 64 bits, and elementwise limits on what fp32 sums
    (limits["fp32"]) or bf16 tensors (["bf16"]) may be off by.

    A logit is a sum whose terms have 22 bits at least, and its own sum's
    roundings: 2^-20 of the sum of the terms' magnitudes.  exp() turns that
    into a relative error of p, twice it with lse's.  Each product's sum again
    loses 2^-20 of its terms; bf16 rounds g and the result by 2^-8."""
    h, w, dloss = (np.asarray(v, np.float64) for v in (h, w, dloss))
    counts = (target != ignore) & (target >= 0) & (target < w.shape[0])
    h = np.where(counts[:, None], h, 0.0)
    at = np.where(counts, target, 0)
    rows = np.arange(len(target))
    l = h @ w.T
    top = l.max(1, keepdims=True, initial=-np.inf)
    lse = (top + np.log(np.exp(l - top).sum(1, keepdims=True)))[:, 0]
    loss = np.where(counts, lse - l[rows, at], 0.0)
    off = 2.0 ** -20 * (np.abs(h) @ np.abs(w).T).max(1, initial=0.0)
    p = np.exp(l - lse[:, None])
    weight = np.where(counts, dloss, 0.0)
    g = p * weight[:, None]
    g[rows, at] -= weight
    dh, dw = g @ w, g.T @ h
    out = {"loss": loss, "lse": np.where(counts, lse, 0.0), "dh": dh, "dw": dw}
    limits = {}
    for name, eps in (("fp32", 0.0), ("bf16", 2.0 ** -8)):
        dg = (2.0 ** -20 + eps) * np.abs(g) + 2 * off[:, None] * p * np.abs(weight)[:, None]
        # p - 1 at the target: rounded at the size of one
        dg[rows, at] += 2.0 ** -22 * np.abs(weight)
        limits[name] = {
            "lse": off + 2.0 ** -21 * (1.0 + np.abs(lse)), "loss": 2 * off + 2.0 ** -20 * (1.0 + np.abs(lse)),
            "dh": dg @ np.abs(w) + eps * np.abs(dh) + 2.0 ** -20 * (np.abs(g) @ np.abs(w)),
            "dw": dg.T @ np.abs(h) + eps * np.abs(dw) + 2.0 ** -20 * (np.abs(g).T @ np.abs(h)),
        }
    return out, limits
