"""The rest of a language model's training step, as cases that can be timed:
the lookup of the words' vectors at its start, the norm before its head, and
the update of the parameters that are no matrices or are not to be
orthogonalised.

  look     words' vectors looked up and scaled (embed_forward).
  spread   its gradient: every word's row is the sum of its tokens' rows, into a
           row of the flat gradient vector (embed_backward); `tied` adds to the
           output head's gradient instead of writing the whole table.
  norm     layer norm of a few rows, as a sampler takes it (layernorm_forward).
  normed   layer norm and its gradients, those of weight and bias among them
           (layernorm_forward, layernorm_backward).
  adamw    an AdamW step over many tensors at once, views of flat vectors
           (adamw_apply), its states in 32 bits or in 8 (read by
           adamw_read_state).
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda"
IGNORE = -100
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
NORM_EPS = 1e-5
LR, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
BLOCK = 256   # elements of an 8-bit state that share a scale


def _look(name, tokens, vocab, width, dtype, scale=1.0):
    return {"name": name, "kind": "look", "tokens": tokens, "vocab": vocab, "width": width, "dtype": dtype,
            "table": dtype, "scale": scale}


def _spread(name, tokens, vocab, width, dtype, table, tied=False):
    return {"name": name, "kind": "spread", "tokens": tokens, "vocab": vocab, "width": width, "dtype": dtype,
            "table": table, "scale": math.sqrt(width), "tied": tied}


def _norm(name, kind, rows, width, dtype, weight, pad=0):
    return {"name": name, "kind": kind, "rows": rows, "width": width, "dtype": dtype, "weight": weight, "pad": pad}


def _adamw(name, tensors, grad, bits, copy=False):
    return {"name": name, "kind": "adamw", "tensors": tensors, "grad": grad, "bits": bits, "copy": copy}


def listed():
    return [
        # one token's vector, as a sampler looks it up
        _look("look_1x33278", 1, 33278, 1024, "bf16"),
        # a large batch of sequences
        _look("look_32768x131072", 32768, 131072, 4096, "bf16", 64.0),
        # fine-tuning on a handful of tokens, the head's gradient already in the row
        _spread("spread_64x33278_tied", 64, 33278, 1024, "fp32", "fp32", tied=True),
        # a step of an LSTM-sized model (35 steps of 20 sequences): the whole table's gradient
        _spread("spread_700x33278", 700, 33278, 650, "fp32", "fp32"),
        # a training batch, 16-bit gradients into the flat fp32 vector
        _spread("spread_16384x131072", 16384, 131072, 2048, "bf16", "fp32"),
        # one token's norm
        _norm("norm_1x1024", "norm", 1, 1024, "bf16", "fp32"),
        # rows of an odd number of values, further apart than they are long
        _norm("normed_700x650_view", "normed", 700, 650, "fp32", "fp32", 13),
        # ordinary and large training batch
        _norm("normed_16384x4096", "normed", 16384, 4096, "bf16", "fp32"),
        # norms and biases of a model: many short tensors, no work but their number
        _adamw("adamw_97_vectors", "48*1024,24*4096,24*333,1*33278", "fp32", 32),
        # the tensors of a ResNet-50-sized network: 161, from 64 elements to 2.4 million
        _adamw("adamw_37m_161", "53*64,40*600,12*4099,16*65536,16*262144,8*589824,8*1048576,8*2359296", "fp32", 32),
        # an LSTM-sized model, no tensor a multiple of a block
        _adamw("adamw8_10m_lstm", "4*1690000,1*3250000,8*2603", "fp32", 8),
        # wide blocks: 16-bit gradients, 8-bit states, the working copy of the weights written too
        _adamw("adamw8_134m_wide", "4*16777216,1*67108864,16*4096", "bf16", 8, copy=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes over their logarithm, half of the rows even
    multiples of 64 long as most models' are, half as they fall."""
    kind = rng.choice(["look", "spread", "norm", "normed", "adamw", "adamw"])
    if kind == "adamw":
        groups, left = [], _log_uniform(rng, 1000, 100_000_000)
        for _ in range(rng.randint(1, 6)):
            size = _log_uniform(rng, 1, max(2, left))
            n = max(1, min(_log_uniform(rng, 1, 120), left // size))
            if rng.random() < 0.5:
                size = max(64, size // 64 * 64)
            groups.append("%d*%d" % (n, size))
            left -= n * size
            if left < 2:
                break
        c = _adamw("", ",".join(groups), rng.choice(["fp32", "bf16"]), rng.choice([32, 8]), rng.random() < 0.5)
    else:
        width = _log_uniform(rng, 16, 4096 if kind in ("look", "spread") else 16384)
        if rng.random() < 0.5:
            width = max(64, width // 64 * 64)
        dtype, other = rng.choice(["fp32", "bf16"]), rng.choice(["fp32", "bf16"])
        if kind in ("look", "spread"):
            tokens, vocab = _log_uniform(rng, 1, 32768), _log_uniform(rng, 1000, 131072)
            tokens = min(tokens, int((6.7e7 if kind == "spread" or dtype == "bf16" else 3.3e7) / width))
            vocab = max(1000, min(vocab, int(2.0e8 / width)))
            c = _look("", tokens, vocab, width, dtype, rng.choice([1.0, 0.37])) if kind == "look" else \
                _spread("", tokens, vocab, width, dtype, other, rng.random() < 0.3)
        else:
            rows = min(_log_uniform(rng, 1, 16384), max(1, int((6.7e7 if dtype == "bf16" else 3.3e7) / width)))
            c = _norm("", kind, rows, width, dtype, other, rng.choice([0, 0, rng.randint(1, 64)]))
    del c["name"]
    return c


def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(seed)


def _words(case, gen):
    """Words fall off as one over their rank, in a shuffled order; a twentieth
    of the tokens are padding where there are many."""
    t, v = case["tokens"], case["vocab"]
    u = torch.rand(t, generator=gen, device=DEVICE, dtype=torch.float64)
    rank = torch.exp(u * math.log(v)).to(torch.int64).clamp_(1, v) - 1
    ids = torch.randperm(v, generator=gen, device=DEVICE)[rank]
    if t > 16:
        ids = torch.where(torch.rand(t, generator=gen, device=DEVICE) < 0.05, IGNORE, ids)
    return ids


def _lookup(case, seed):
    gen = _generator(seed * 8 + 1)
    ids = _words(case, gen)
    if case["kind"] == "look":
        table = torch.randn((case["vocab"], case["width"]), generator=gen, device=DEVICE).mul_(0.02)
        return {"ids": ids, "table": table.to(DTYPES[case["table"]])}
    dout = torch.randn((case["tokens"], case["width"]), generator=gen, device=DEVICE).mul_(1e-3)
    s = {"ids": ids, "dout": dout.to(DTYPES[case["dtype"]])}
    if case["tied"]:   # what the head's gradient left there
        s["dtable"] = torch.randn((case["vocab"], case["width"]), generator=gen, device=DEVICE).mul_(1e-3)
        s["dtable"] = s["dtable"].to(DTYPES[case["table"]])
    return s


def _rows(case, seed):
    """Hidden states with a mean of their own in every column and a few columns
    of large values, and a gradient of their size."""
    gen = _generator(seed * 8 + 2)
    r, w, dtype, wide = case["rows"], case["width"], DTYPES[case["dtype"]], DTYPES[case["weight"]]
    x = torch.randn((r, w), generator=gen, device=DEVICE)
    x.add_(torch.randn(w, generator=gen, device=DEVICE), alpha=0.5)
    x.mul_(torch.where(torch.rand(w, generator=gen, device=DEVICE) < 0.01, 12.0, 1.0))
    s = {"x": _padded(x.to(dtype), case["pad"])}
    s["weight"] = (1.0 + 0.2 * torch.randn(w, generator=gen, device=DEVICE)).to(wide)
    s["bias"] = (0.1 * torch.randn(w, generator=gen, device=DEVICE)).to(wide)
    if case["kind"] == "normed":
        s["dy"] = _padded(torch.randn((r, w), generator=gen, device=DEVICE).mul_(1e-2).to(dtype), case["pad"])
    return s


def _padded(x, pad):
    if pad == 0:
        return x
    wide = torch.zeros((x.shape[0], x.shape[1] + pad), dtype=x.dtype, device=DEVICE)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def _sizes(case):
    out = []
    for part in case["tensors"].split(","):
        n, size = part.split("*")
        out += [int(size)] * int(n)
    return out


def _decays(sizes):
    """Short tensors are norms and biases, which do not decay."""
    return [DECAY if n > 5000 else 0.0 for n in sizes]


def _log2(y):
    """The exponent of the power of two at or below y >= 0 (-127 where that is
    below 2^-126)."""
    return y.view(torch.int32).div(1 << 23, rounding_mode="floor").sub_(127)


def _power(e):
    return (e + 127).mul_(1 << 23).view(torch.float32)


def _in_8_bits(y, mantissa, low, dither):
    """The values that blocks of BLOCK elements y >= 0 stand for in 8 bits: the
    block's largest lies in [2^7, 2^8) of its scale, a power of two; a value
    takes `mantissa` bits below its leading one, from 2^-6 down those of 2^-6;
    what is below them is rounded up by the share `dither` of a step, and a value
    above 0 is `low` steps at least."""
    n = y.numel()
    full = torch.zeros(-(-n // BLOCK) * BLOCK, device=DEVICE)
    full[:n] = y
    rows = full.view(-1, BLOCK)
    e = _log2(rows.amax(1)).clamp_(min=-95)
    up = _power(7 - e)[:, None].expand(-1, BLOCK).reshape(-1)[:n]
    y = y * up
    q = _power(_log2(y).clamp_(min=-6) - mantissa)
    steps = torch.floor(y / q + dither)
    return torch.where(y > 0, steps.clamp_(min=low), steps) * q / up


def _dither(n, tensor, step, seed=0):
    """Two random numbers below 1 for every element, 16 bits each, from the
    element, its tensor and the step."""
    def mixed(z):
        z = z ^ (z >> 16)
        z = (z * 0x6A09E667) & 0xFFFFFFFF
        z = z ^ (z >> 15)
        z = (z * 0xBB67AE85) & 0xFFFFFFFF
        return z ^ (z >> 16)
    key = mixed((seed + tensor * 0x3C6EF373 + step * 0xA54FF53B) & 0xFFFFFFFF)
    z = mixed(((torch.arange(n, device=DEVICE) * 0x9E3779B1) & 0xFFFFFFFF) ^ key)
    return (z & 0xFFFF).float() / 65536, (z >> 16).float() / 65536


def _model(case, seed):
    """Flat vectors g, x, m, v after some steps, tensor after tensor."""
    gen = _generator(seed * 8 + 3)
    sizes = _sizes(case)
    d = sum(sizes)
    # every tensor's gradients have a size of their own, and every element's within it
    size = torch.repeat_interleave(torch.exp(torch.randn(len(sizes), generator=gen, device=DEVICE) * 1.5 - 7.0),
                                   torch.tensor(sizes, device=DEVICE), output_size=d)
    size.mul_(torch.exp(torch.randn(d, generator=gen, device=DEVICE)))
    g = torch.randn(d, generator=gen, device=DEVICE).mul_(size)
    m = torch.randn(d, generator=gen, device=DEVICE).mul_(size).mul_(0.3)
    v = size.mul_(torch.rand(d, generator=gen, device=DEVICE).add_(0.5)).square_()
    x = torch.randn(d, generator=gen, device=DEVICE).mul_(0.02)
    if case["bits"] == 8:   # states that 8 bits hold (again, where the first rounding moved a block's scale)
        for _ in range(2):
            at = 0
            for n in sizes:
                part = m[at:at + n]
                part.copy_(torch.sign(part) * _in_8_bits(part.abs(), 3, 0, 0.5))
                part = v[at:at + n]
                part.copy_(_in_8_bits(part.sqrt(), 4, 1, 0.5).square_())
                at += n
    return {"g": g.to(DTYPES[case["grad"]]), "x": x, "m": m, "v": v}


def prepare(case, seed):
    kind = case["kind"]
    if kind in ("look", "spread"):
        s = _lookup(case, seed)
        s["scale"], s["tied"], s["shape"] = case["scale"], case.get("tied", False), (case["vocab"], case["width"])
        s["to"] = DTYPES[case["table"]]
    elif kind in ("norm", "normed"):
        s = _rows(case, seed)
    else:
        s = _model(case, seed)
        s["sizes"], s["bits"], s["step"] = _sizes(case), case["bits"], 1000 + seed % 1000
        if case["copy"]:
            s["copy"] = s["x"].to(torch.bfloat16)
    s["kind"] = kind
    if own:   # workspaces, output buffers, prepared calls: what a program keeps from step to step
        from paper_2108_00951_amd import binding as efs
        s["efs"] = efs
        if kind == "look":
            s["out"] = torch.empty((case["tokens"], case["width"]), dtype=s["table"].dtype, device=DEVICE)
        elif kind == "spread":
            s["ws"] = efs.new_embed_workspace(case["tokens"], case["vocab"], case["width"], DEVICE)
            if not case["tied"]:
                s["dtable"] = torch.empty(s["shape"], dtype=s["to"], device=DEVICE)
        elif kind in ("norm", "normed"):
            s["y"] = torch.empty((case["rows"], case["width"]), dtype=s["x"].dtype, device=DEVICE)
            if kind == "normed":
                s["mean"], s["rstd"] = (torch.empty(case["rows"], device=DEVICE) for _ in range(2))
                s["dx"] = torch.empty_like(s["y"])
                s["dweight"], s["dbias"] = torch.empty_like(s["weight"]), torch.empty_like(s["bias"])
                s["ws"] = efs.new_layernorm_workspace(case["rows"], case["width"], DEVICE)
        else:
            _prepare_adamw(s, efs)
    return s


def _prepare_adamw(s, efs):
    sizes = s["sizes"]
    split = {k: list(torch.split(s[k], sizes)) for k in ("g", "x", "m", "v", "copy") if k in s}
    if s["bits"] == 8:
        split["m8"], split["v8"] = efs.new_adamw_state(sizes, DEVICE)
        efs.adamw_write_state(split["m"], split["v"], split["m8"], split["v8"])
        s["read"] = efs.prepare_adamw_read_state(split["m8"], split["v8"], split["m"], split["v"])
    m, v = (split["m8"], split["v8"]) if s["bits"] == 8 else (split["m"], split["v"])
    s["update"] = efs.prepare_adamw_apply(split["g"], split["x"], m, v, lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS,
                                          weight_decay=_decays(sizes), copy=split.get("copy"))


def _plain_adamw(s):
    """Every operation a separately rounded one of 32 bits."""
    def r(c):
        return float(np.float32(c))
    lr, b1, b2 = (float(np.float32(c)) for c in (LR, BETA1, BETA2))
    s["step"] += 1
    t, g, x = s["step"], s["g"].float(), s["x"]
    alpha = r(lr / (1.0 - b1 ** t))
    root = r(1.0 / math.sqrt(1.0 - b2 ** t))
    m = s["m"].mul_(b1).add_(g * r(1.0 - b1))
    v = s["v"].mul_(b2).add_((g * r(1.0 - b2)).mul_(g))
    den = v.sqrt().mul_(root).add_(r(EPS))
    at = 0
    for decay in _decays(s["sizes"]):   # the decay is a tensor's own
        n = s["sizes"][at]
        at += 1
        if decay:
            start = sum(s["sizes"][:at - 1])
            x[start:start + n].mul_(r(1.0 - lr * float(np.float32(decay))))
    x.sub_((m / den).mul_(alpha))
    if s["bits"] == 8:
        start = 0
        for i, n in enumerate(s["sizes"]):
            dm, dv = _dither(n, i, t)
            part = m[start:start + n]
            part.copy_(torch.sign(part) * _in_8_bits(part.abs(), 3, 0, dm))
            part = v[start:start + n]
            part.copy_(_in_8_bits(part.sqrt(), 4, 1, dv).square_())
            start += n
    out = {"x": x, "m": m, "v": v}
    if "copy" in s:
        out["copy"] = s["copy"].copy_(x)
    return out


def _plain_norm(s):
    x, w, b = s["x"].float(), s["weight"].float(), s["bias"].float()
    mean = x.mean(1, keepdim=True)
    c = x - mean
    rstd = c.square().mean(1, keepdim=True).add_(NORM_EPS).sqrt_().reciprocal_()
    xhat = c * rstd
    out = {"y": (xhat * w + b).to(s["x"].dtype)}
    if s["kind"] == "normed":
        dy = s["dy"].float()
        g = dy * w
        dx = (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True)) * rstd
        out.update(mean=mean[:, 0], rstd=rstd[:, 0], dx=dx.to(s["x"].dtype),
                   dweight=(dy * xhat).sum(0).to(s["weight"].dtype), dbias=dy.sum(0).to(s["bias"].dtype))
    return out


def _plain_lookup(s):
    kept = s["ids"] != IGNORE
    at = torch.where(kept, s["ids"], 0)
    if s["kind"] == "look":
        rows = s["table"][at].float() * s["scale"]
        return torch.where(kept[:, None], rows, 0.0).to(s["table"].dtype)
    rows = torch.where(kept[:, None], s["dout"].float(), 0.0)
    sums = torch.zeros(s["shape"], device=DEVICE).index_add_(0, at, rows).mul_(s["scale"])
    if s["tied"]:
        return s["dtable"].copy_(s["dtable"].float() + sums)
    return sums.to(s["to"])


def run(s):
    kind = s["kind"]
    if not own:
        if kind in ("look", "spread"):
            return _plain_lookup(s)
        return _plain_adamw(s) if kind == "adamw" else _plain_norm(s)
    efs = s["efs"]
    if kind == "look":
        efs.embed_forward(s["table"], s["ids"], s["out"], scale=s["scale"], ignore_index=IGNORE)
        return s["out"]
    if kind == "spread":
        efs.embed_backward(s["dout"], s["ids"], s["dtable"], s["ws"], scale=s["scale"], ignore_index=IGNORE,
                           accumulate=s["tied"])
        return s["dtable"]
    if kind == "norm":
        efs.layernorm_forward(s["x"], s["weight"], s["bias"], s["y"], eps=NORM_EPS)
        return {"y": s["y"]}
    if kind == "normed":
        efs.layernorm_forward(s["x"], s["weight"], s["bias"], s["y"], s["mean"], s["rstd"], eps=NORM_EPS)
        efs.layernorm_backward(s["x"], s["weight"], s["mean"], s["rstd"], s["dy"], s["dx"], s["dweight"], s["dbias"],
                               s["ws"])
        return {k: s[k] for k in ("y", "mean", "rstd", "dx", "dweight", "dbias")}
    s["step"] += 1
    s["update"](s["step"])
    if s["bits"] == 8:
        s["read"]()
    out = {k: s[k] for k in ("x", "m", "v")}
    if "copy" in s:
        out["copy"] = s["copy"]
    return out


def _distinct(case):
    """How many words that many tokens are expected to be."""
    k = np.arange(1, case["vocab"] + 1, dtype=np.float64)
    p = np.log1p(1.0 / k) / math.log(case["vocab"])
    return float(-np.expm1(case["tokens"] * np.log1p(-np.minimum(p, 0.999))).sum())


def work(case):
    kind = case["kind"]
    if kind == "adamw":
        d = sum(_sizes(case))
        each = 8 + (4 if case["grad"] == "fp32" else 2) + (16 if case["bits"] == 32 else 4 + 8) + (2 if case["copy"] else 0)
        return {"bytes": each * d, "flops": 15 * d}
    e = 4 if case["dtype"] == "fp32" else 2
    if kind in ("look", "spread"):
        f, t, w = 4 if case["table"] == "fp32" else 2, case["tokens"], case["width"]
        if kind == "look":
            table = _distinct(case) * f
        else:
            table = 2 * _distinct(case) * f if case["tied"] else case["vocab"] * f
        return {"bytes": int(8 * t + t * w * e + table * w), "flops": t * w}
    r, w, f = case["rows"], case["width"], 4 if case["weight"] == "fp32" else 2
    if kind == "norm":
        return {"bytes": 2 * r * w * e + 2 * w * f, "flops": 8 * r * w}
    return {"bytes": 4 * r * w * e + 4 * w * f + 8 * r, "flops": 22 * r * w}


def exact(case, seed):
    kind = case["kind"]
    if kind in ("look", "spread"):
        s = _lookup(case, seed)
        kept = (s["ids"] != IGNORE).nonzero()[:, 0]
        words = s["ids"][kept]
        if kind == "look":
            out = torch.zeros((case["tokens"], case["width"]), dtype=torch.float64, device=DEVICE)
            out[kept] = s["table"][words].double() * float(np.float32(case["scale"]))
            return out
        out = torch.zeros((case["vocab"], case["width"]), dtype=torch.float64, device=DEVICE)
        out.index_put_((words,), s["dout"][kept].double() * float(np.float32(case["scale"])), accumulate=True)
        return out + s["dtable"].double() if case["tied"] else out
    if kind in ("norm", "normed"):
        return _exact_norm(case, _rows(case, seed))
    s = _model(case, seed)
    g, x, m, v = (s[k].double() for k in ("g", "x", "m", "v"))
    lr, b1, b2, eps = (float(np.float32(c)) for c in (LR, BETA1, BETA2, EPS))
    t = 1000 + seed % 1000 + 1
    sizes = _sizes(case)
    decay = torch.repeat_interleave(torch.tensor([float(np.float32(c)) for c in _decays(sizes)], dtype=torch.float64,
                                                 device=DEVICE), torch.tensor(sizes, device=DEVICE), output_size=x.numel())
    m = b1 * m + (1.0 - b1) * g
    v = b2 * v + (1.0 - b2) * g * g
    x = x - lr * decay * x - lr * (m / (1.0 - b1 ** t)) / (torch.sqrt(v / (1.0 - b2 ** t)) + eps)
    # where 8 bits hold the states, a value next to a border has no one answer
    out = {"x": x, "m": m if case["bits"] == 32 else None, "v": v if case["bits"] == 32 else None}
    if case["copy"]:
        out["copy"] = x
    return out


def _exact_norm(case, s):
    x, w, b = s["x"].double(), s["weight"].double(), s["bias"].double()
    n = case["width"]
    out = {"y": torch.empty((case["rows"], n), dtype=torch.float64, device=DEVICE)}
    train = case["kind"] == "normed"
    if train:
        for k in ("mean", "rstd"):
            out[k] = torch.empty(case["rows"], dtype=torch.float64, device=DEVICE)
        out["dx"] = torch.empty_like(out["y"])
        out["dweight"], out["dbias"] = torch.zeros_like(w), torch.zeros_like(b)
    for lo in range(0, case["rows"], 2048):   # some rows at a time
        part = slice(lo, min(lo + 2048, case["rows"]))
        var, mean = torch.var_mean(x[part], dim=1, correction=0)
        rstd = (var + NORM_EPS) ** -0.5
        unit = (x[part] - mean[:, None]) / torch.sqrt(var + NORM_EPS)[:, None]
        out["y"][part] = unit * w + b
        if train:
            dy = s["dy"][part].double()
            g = dy * w
            along = (g * unit).sum(1, keepdim=True) / n
            out["dx"][part] = rstd[:, None] * (g - unit * along - g.sum(1, keepdim=True) / n)
            out["mean"][part], out["rstd"][part] = mean, rstd
            out["dweight"] += (unit * dy).sum(0)
            out["dbias"] += dy.sum(0)
    return out
