"""Plain 64-bit forms of the lookup, the layer norm and the AdamW step, and how
far 32-bit arithmetic may be from them.

A rounding is off by at most HALF[t] relative to the value.  A sum of n terms in
32 bits, in any order, is off by at most n * 2^-24 of the sum of their magnitudes
(every addition rounds a partial sum that is no larger than that)."""
import numpy as np

EPS32 = 2.0 ** -24
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}


def embed_gradient(dout, ids, vocab, scale, ignore=-100, before=None, to="fp32"):
    """dtable in 64 bits and its limit: the sum of n rows (n - 1 additions), the
    product, the addition to what was there, the rounding of the result."""
    dout = np.asarray(dout, np.float64)
    out, size = np.zeros((vocab, dout.shape[1])), np.zeros((vocab, dout.shape[1]))
    n = np.zeros((vocab, 1))
    for t, v in enumerate(ids):
        if v != ignore and 0 <= v < vocab:
            out[v] += dout[t]
            size[v] += np.abs(dout[t])
            n[v] += 1
    out, size = out * scale, size * abs(scale)
    limit = (n + 1) * EPS32 * size
    if before is not None:
        out = out + before
        limit = limit + EPS32 * (np.abs(before) + size)
    return out, limit * 1.01 + 1.01 * HALF[to] * np.abs(out)


def norm(x, w, b, dy=None, eps=1e-5, dtype="fp32", weight_dtype="fp32"):
    """y, mean, rstd and, with dy, dx, dweight, dbias; {name: (value, limit)}.

    Each is a few operations on values whose size is known: with u the rounding
    2^-24 and k = width, the mean is off by k u of the mean magnitude, as is the
    rest that is taken off after it; what is left of that is u |mean| k u, so that
    x - mean is off by 2 u |x - mean| + 2 u (|mean| u k + spread u k).  The sums
    for rstd are of squares, k u relative.  Each limit below takes 4 (k + 8) u of
    the magnitudes that its terms have."""
    x = np.asarray(x, np.float64)
    rows, k = x.shape
    w = np.ones(k) if w is None else np.asarray(w, np.float64)
    b = np.zeros(k) if b is None else np.asarray(b, np.float64)
    eps = float(np.float32(eps))
    u = 4.0 * (k + 8) * EPS32
    mean = x.mean(1, keepdims=True)
    c = x - mean
    rstd = 1.0 / np.sqrt((c * c).mean(1, keepdims=True) + eps)
    h = c * rstd
    big = np.abs(x).mean(1, keepdims=True)
    # x - mean: its own rounding, and what the mean's rounding leaves
    off = (np.abs(c) * EPS32 * 4 + big * EPS32 * u + np.abs(c).mean(1, keepdims=True) * u) * rstd
    # the rounding of x - m before the rest is taken off is u of it, also where that is large
    hl = off + np.abs(h) * u
    out = {"y": (h * w + b, hl * np.abs(w) + 4 * EPS32 * np.abs(b) + HALF[dtype] * np.abs(h * w + b)),
           "mean": (mean[:, 0], (u * big)[:, 0]), "rstd": (rstd[:, 0], (u * rstd)[:, 0])}
    if dy is not None:
        dy = np.asarray(dy, np.float64)
        g = dy * w
        sg, sgh = g.mean(1, keepdims=True), (g * h).mean(1, keepdims=True)
        dx = rstd * (g - sg - h * sgh)
        ag, agh = np.abs(g).mean(1, keepdims=True), (np.abs(g) * (np.abs(h) + hl / u)).mean(1, keepdims=True)
        lim = rstd * (u * (np.abs(g) + ag + np.abs(h) * agh) + hl * agh) + u * np.abs(dx)
        out["dx"] = (dx, lim + HALF[dtype] * np.abs(dx))
        r = 2.0 * (rows + 8) * EPS32
        dw, db = (dy * h).sum(0), dy.sum(0)
        out["dweight"] = (dw, r * np.abs(dy * h).sum(0) + (np.abs(dy) * hl).sum(0) + HALF[weight_dtype] * np.abs(dw))
        out["dbias"] = (db, r * np.abs(dy).sum(0) + HALF[weight_dtype] * np.abs(db))
    return {name: (v, 1.01 * limit + 1e-300) for name, (v, limit) in out.items()}


def within(got, pair, what):
    want, limit = pair
    got = np.asarray(got, np.float64)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    off = np.abs(got - want) - limit
    at = np.unravel_index(np.argmax(np.where(np.isnan(off), np.inf, off)), off.shape) if off.size else None
    assert off.size == 0 or np.all(off <= 0), (what, at, got[at], want[at], limit[at])


class Adamw:
    """The step bit by bit: every operation a separately rounded one of 32 bits,
    the rates from 64."""

    def __init__(self, lr, beta1=0.9, beta2=0.999, eps=1e-8, seed=0, bits=32):
        self.lr, self.b1, self.b2, self.eps = (np.float32(v) for v in (lr, beta1, beta2, eps))
        self.seed, self.bits = seed, bits

    @staticmethod
    def power(b, t):
        p, b = 1.0, float(b)
        while t:
            if t & 1:
                p *= b
            b *= b
            t >>= 1
        return p

    def step(self, t, ordinal, g, x, m, v, decay, lr_factor=1.0, gain=None, start=0):
        """New x, m, v (as the state holds them) of the elements from `start` on
        (a multiple of 256)."""
        with np.errstate(all="ignore"):
            lr = float(self.lr) * float(np.float32(lr_factor))
            alpha = np.float32(lr / (1.0 - self.power(self.b1, t)))
            root = np.float32(1.0 / np.sqrt(1.0 - self.power(self.b2, t)))
            keep = np.float32(1.0 - lr * float(np.float32(decay)))
            g = g.astype(np.float32)
            if gain is not None:
                g = g * np.float32(gain)
            m = self.b1 * m + np.float32(1.0 - float(self.b1)) * g
            v = self.b2 * v + (np.float32(1.0 - float(self.b2)) * g) * g
            x = x * keep - alpha * (m / (np.sqrt(v) * root + self.eps))
            if self.bits == 8:
                dm, dr = dither(g.size, ordinal, t, self.seed, start)
                m = np.copysign(in_8_bits(np.abs(m), 3, 0, dm), m)
                r = in_8_bits(np.sqrt(v), 4, 1, dr)
                v = r * r
        return x, m, v


def dither(n, ordinal, step, seed, start=0):
    """Random numbers below 1 in steps of 2^-16 for m and for r."""
    mask = np.uint64(0xFFFFFFFF)

    def mixed(z):
        z = z ^ (z >> np.uint64(16))
        z = (z * np.uint64(0x6A09E667)) & mask
        z = z ^ (z >> np.uint64(15))
        z = (z * np.uint64(0xBB67AE85)) & mask
        return z ^ (z >> np.uint64(16))
    key = mixed(np.uint64((seed + ordinal * 0x3C6EF373 + step * 0xA54FF53B) & 0xFFFFFFFF))
    z = mixed(((np.arange(start, start + n, dtype=np.uint64) * np.uint64(0x9E3779B1)) & mask) ^ key)
    return (z & np.uint64(0xFFFF)).astype(np.float64) / 65536, (z >> np.uint64(16)).astype(np.float64) / 65536


def in_8_bits(y, mantissa, least, up):
    """The values that y >= 0 (fp32) becomes in a state of 8 bits."""
    out = np.empty(y.size, np.float32)
    up = np.broadcast_to(up, y.shape)
    for at in range(0, y.size, 256):
        part = y[at:at + 256].astype(np.float64)
        ok = np.isfinite(part)
        top = part[ok].max(initial=0.0)
        e = max(int(np.frexp(top)[1]) - 1 if top > 0 else -95, -95)
        z = np.where(ok, part, 0.0) * 2.0 ** (7 - e)
        q = 2.0 ** (np.maximum(np.where(z > 0, np.frexp(np.where(z > 0, z, 1.0))[1] - 1, -6), -6) - mantissa)
        # fp32 all the same: the quotient is exact, the sum rounds where it has more than 24 bits
        n = np.floor(((z / q).astype(np.float32) + up[at:at + 256].astype(np.float32)).astype(np.float64))
        n = np.where((z > 0) & (n < least), least, n)
        out[at:at + 256] = np.where(ok, n * q * 2.0 ** (e - 7), np.nan)
    return out
