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
