"""Training with 8-bit activations, as timed cases: what a program does between two gradient exchanges.

All operators share one format ("q8"): int8 codes, a row per token (of an activation) or per output channel (of a
weight), rows a multiple of 16 bytes apart, and one float32 scale per row, a power of two.  Kinds of case:

  checkpoint    an activation is stored in 8 bits and restored
  norm          RMS norm with the residual's addition and an output in 8 bits
  norm_grad     its backward pass; the normalised rows are kept as they are or as an 8-bit checkpoint
  matmul        product of 8-bit activations and 8-bit weights, with the scales of each token and channel
  grad_input    its gradient for the activations, from the 8-bit weights
  grad_weight   its gradient for the weights, from the 8-bit activations (the checkpoint), into the gradient bucket

Activations have a few channels that are an order of magnitude wider than the others, gradients are small, tokens
that were padded have rows of zeros.
"""
from __future__ import annotations

import math

import torch

own = False

F32, BF16 = "float32", "bfloat16"
EPS = 1e-5


def _nsml():
    import paper_2506_16235_b200 as nsml

    return nsml


def listed():
    return [
        # one token's row of a small decoder is kept: launches are all there is
        dict(name="checkpoint_token", kind="checkpoint", rows=1, cols=768, dtype=BF16),
        # the widest activation of the 1.3B decoder (ffn 8192) for 16 sequences of 1024 tokens
        dict(name="checkpoint_16384x8192", kind="checkpoint", rows=16_384, cols=8192, dtype=BF16),
        # a ragged batch in float32, no residual (the first norm of a model), odd width
        dict(name="norm_ragged", kind="norm", rows=301, cols=1027, dtype=F32, residual=False),
        # the norms inside the 1.3B decoder, 8 sequences of 2048 tokens
        dict(name="norm_16384x2048", kind="norm", rows=16_384, cols=2048, dtype=BF16, residual=True),
        dict(name="norm_grad_ragged", kind="norm_grad", rows=301, cols=1027, dtype=F32, packed=False, extra=False),
        # its backward pass with the residual stream kept in 8 bits and a gradient that arrives past the block
        dict(name="norm_grad_16384x2048", kind="norm_grad", rows=16_384, cols=2048, dtype=BF16, packed=True, extra=True),
        # one token through the decoder's first ffn matrix: the weights have to be read, nothing else
        dict(name="matmul_token", kind="matmul", m=1, n=8192, k=2048, out=BF16),
        # the same matrix for a batch of 8192 tokens
        dict(name="matmul_8192", kind="matmul", m=8192, n=8192, k=2048, out=BF16),
        # gradients of a ragged batch through a layer of odd sizes
        dict(name="grad_input_ragged", kind="grad_input", m=301, n=1003, k=771, out=F32),
        dict(name="grad_input_8192", kind="grad_input", m=8192, n=8192, k=2048, out=BF16),
        # a weight of GPT-2 small's width from one sequence: a small matrix, a long sum
        dict(name="grad_weight_768", kind="grad_weight", m=1025, n=768, k=768, out=F32),
        dict(name="grad_weight_8192", kind="grad_weight", m=8192, n=8192, k=2048, out=BF16),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: tokens from one to a long batch, widths from small to the largest, odd ones among them."""
    kind = rng.choice(("checkpoint", "norm", "norm_grad", "matmul", "matmul", "grad_input", "grad_weight"))
    dtype = rng.choice((F32, BF16, BF16))
    if kind in ("checkpoint", "norm", "norm_grad"):
        case = dict(kind=kind, rows=_log_int(rng, 1, 32_768), cols=_log_int(rng, 64, 16_384), dtype=dtype)
        if kind == "norm":
            case.update(residual=rng.random() < 0.7)
        elif kind == "norm_grad":
            case.update(packed=rng.random() < 0.5, extra=rng.random() < 0.5)
        while work(case)["bytes"] > 0.6e9:
            case["rows"] = case["rows"] // 2 + 1
        return case
    case = dict(kind=kind, m=_log_int(rng, 1, 32_768), n=_log_int(rng, 64, 16_384), k=_log_int(rng, 64, 16_384), out=dtype)
    while work(case)["flops"] > 2.7e11:
        size = max(("m", "n", "k"), key=lambda s: case[s])
        case[size] = case[size] // 2 + 1
    return case


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _generator(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1_000_003 + salt * 7919 + 4321) % (1 << 62))
    return g


def _dtype(name):
    return torch.float32 if name == F32 else torch.bfloat16


def _activation(rows, cols, seed, salt):
    """Gaussian, about one channel in a hundred ten times as wide; one row in fifty is padding (zeros), if there are several."""
    gen = _generator(seed, salt)
    x = torch.randn(rows, cols, generator=gen, device="cuda")
    x.mul_(torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.01, 10.0, 1.0))
    if rows > 1:
        x.masked_fill_(torch.rand(rows, 1, generator=gen, device="cuda") < 0.02, 0.0)
    return x


def _gradient(rows, cols, seed, salt):
    """Small, and a token's size differs from the next one's by up to an order of magnitude."""
    gen = _generator(seed, salt)
    g = torch.randn(rows, cols, generator=gen, device="cuda")
    return g.mul_(1e-3 * 10.0 ** (torch.rand(rows, 1, generator=gen, device="cuda") - 0.5))


def _padded_rows(x):
    """x with its rows a multiple of 16 bytes apart, as the products' gradients have to be."""
    rows, cols = x.shape
    out = torch.zeros(rows, (cols + 7) // 8 * 8, dtype=x.dtype, device=x.device)[:, :cols]
    return out.copy_(x)


def _scale_of(amax):
    """The smallest power of two whose 127 steps reach amax (between 2^-126 and 2^121), 0 for 0."""
    m, e = torch.frexp(amax)
    e = torch.where(m <= 127.0 / 128.0, e - 7, e - 6).clamp(-126, 121)
    return torch.where(amax == 0, torch.zeros_like(amax), torch.ldexp(torch.ones_like(amax), e))


def _quantise(y):
    """Codes (as numbers of y's type) and scales of the rows of y."""
    scale = _scale_of(y.abs().amax(dim=1))
    inverse = torch.where(scale == 0, torch.zeros_like(scale), 1.0 / scale)
    return torch.round(y * inverse[:, None]).clamp(-127, 127), scale


def _q8(x):
    """x in the q8 format: int8 codes (rows a multiple of 16 bytes apart) and float32 scales."""
    rows, cols = x.shape
    codes = torch.zeros(rows, (cols + 15) // 16 * 16, dtype=torch.int8, device=x.device)[:, :cols]
    values, scales = _quantise(x)
    codes.copy_(values)
    return codes, scales


def _weight(rows, cols, seed, salt):
    gen = _generator(seed, salt)
    return torch.randn(rows, cols, generator=gen, device="cuda").mul_(cols ** -0.5)


def prepare(case, seed):
    kind, s = case["kind"], dict(case)
    if kind in ("checkpoint", "norm", "norm_grad"):
        rows, cols, dtype = case["rows"], case["cols"], _dtype(case["dtype"])
        padded = (cols + 15) // 16 * 16
        s["x"] = _activation(rows, cols, seed, 1).to(dtype)
        s["weight"] = (1.0 + 0.1 * torch.randn(cols, generator=_generator(seed, 2), device="cuda")).to(dtype)
        # what the program keeps for the results
        s["codes"] = torch.empty(rows, padded, dtype=torch.int8, device="cuda")[:, :cols]
        s["scales"], s["rstd"] = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        s["into"] = torch.empty(rows, cols, dtype=dtype, device="cuda")
        s["values"] = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda") if kind == "norm" else None
        if kind == "norm":
            s["residual"] = _activation(rows, cols, seed, 3).to(dtype) if case["residual"] else None
        if kind == "norm_grad":
            x = s["x"].float()
            s["rstd"] = torch.rsqrt(x.double().square().mean(dim=1) + EPS).float()
            s["dy"] = _gradient(rows, cols, seed, 4).to(dtype)
            s["dh"] = _gradient(rows, cols, seed, 5).to(dtype) if case["extra"] else None
            s["dweight"] = torch.empty(cols, device="cuda")
            s["workspace"] = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
            if case["packed"]:
                s["codes"], s["scales"] = _q8(x)
                s["x"] = None
        return s
    m, n, k, out = case["m"], case["n"], case["k"], _dtype(case["out"])
    s["workspace"] = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    if kind in ("matmul", "grad_weight"):
        s["a"], s["a_scales"] = _q8(_activation(m, k, seed, 1))
    if kind in ("matmul", "grad_input"):
        s["b"], s["b_scales"] = _q8(_weight(n, k, seed, 2))
    if kind != "matmul":
        s["dy"] = _padded_rows(_gradient(m, n, seed, 4).to(torch.bfloat16))
    shape = {"matmul": (m, n), "grad_input": (m, k), "grad_weight": (n, k)}[kind]
    s["into"] = torch.empty(shape, dtype=out, device="cuda")
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    nsml, kind = _nsml(), s["kind"]
    if kind == "checkpoint":
        nsml.nsml_q8_pack(s["x"], codes=s["codes"], scales=s["scales"])
        return {"values": nsml.nsml_q8_unpack(s["codes"], s["scales"], out=s["into"]), "scales": s["scales"]}
    if kind == "norm":
        _, _, rstd, h = nsml.nsml_q8_rms_norm(s["x"], s["weight"], EPS, residual=s["residual"], codes=s["codes"],
                                              scales=s["scales"], rstd=s["rstd"],
                                              h=s["into"] if s["residual"] is not None else None)
        values = nsml.nsml_q8_unpack(s["codes"], s["scales"], out=s["values"])
        return {"values": values, "scales": s["scales"], "rstd": rstd, "h": h}
    if kind == "norm_grad":
        kept = dict(h=s["x"]) if s["x"] is not None else dict(codes=s["codes"], scales=s["scales"])
        dx, dw = nsml.nsml_q8_rms_norm_backward(s["dy"], s["weight"], s["rstd"], dh=s["dh"], dx=s["into"],
                                                dweight=s["dweight"], workspace=s["workspace"], **kept)
        return {"dx": dx, "dweight": dw}
    if kind == "matmul":
        return nsml.nsml_q8_matmul(s["a"], s["a_scales"], s["b"], s["b_scales"], out=s["into"], workspace=s["workspace"])
    if kind == "grad_input":
        return nsml.nsml_q8_matmul_grad_input(s["dy"], s["b"], s["b_scales"], dx=s["into"], workspace=s["workspace"])
    return nsml.nsml_q8_matmul_grad_weight(s["dy"], s["a"], s["a_scales"], dw=s["into"], workspace=s["workspace"])


def _run_plain(s):
    kind = s["kind"]
    if kind == "checkpoint":
        codes, scales = _quantise(s["x"].float())
        return {"values": (codes * scales[:, None]).to(s["x"].dtype), "scales": scales}
    if kind == "norm":
        x = s["x"]
        h = x if s["residual"] is None else (x.float() + s["residual"].float()).to(x.dtype)
        hf = h.float()
        # the codes are next to borders: the sum of squares is in 64 bits
        rstd = (1.0 / torch.sqrt(hf.double().square().mean(dim=1) + EPS)).float()
        codes, scales = _quantise(hf * rstd[:, None] * s["weight"].float())
        return {"values": (codes * scales[:, None]).to(torch.bfloat16), "scales": scales, "rstd": rstd, "h": h}
    if kind == "norm_grad":
        h = s["x"].float() if s["x"] is not None else s["codes"].float() * s["scales"][:, None]
        normed, dy, rstd = h * s["rstd"][:, None], s["dy"].float(), s["rstd"][:, None]
        g = dy * s["weight"].float()
        dx = rstd * (g - normed * (g * normed).mean(dim=1, keepdim=True))
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        return {"dx": dx.to(s["dy"].dtype), "dweight": (dy * normed).sum(dim=0)}
    dtype = s["into"].dtype
    if kind == "matmul":
        y = torch.matmul(s["a"].float(), s["b"].float().T)
        return (y * s["a_scales"][:, None] * s["b_scales"]).to(dtype)
    if kind == "grad_input":
        return torch.matmul(s["dy"].float(), s["b"].float() * s["b_scales"][:, None]).to(dtype)
    return torch.matmul(s["dy"].float().T, s["a"].float() * s["a_scales"][:, None]).to(dtype)


# ---------------------------------------------------------------------------
# what a pass cannot do without, and its results in 64 bits
# ---------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind in ("checkpoint", "norm", "norm_grad"):
        rows, cols, e = case["rows"], case["cols"], 4 if case["dtype"] == F32 else 2
        size = rows * cols
        if kind == "checkpoint":  # read, written in 8 bits, read in 8 bits, written
            return {"bytes": size * (e + 1 + 1 + e) + 8 * rows, "flops": 4 * size}
        if kind == "norm":
            return {"bytes": size * ((3 * e if case["residual"] else e) + 1) + 8 * rows + e * cols, "flops": 8 * size}
        kept = 1 if case["packed"] else e
        return {"bytes": size * (e + kept + e + (e if case["extra"] else 0)) + 8 * rows + (e + 4) * cols, "flops": 10 * size}
    m, n, k, e = case["m"], case["n"], case["k"], 4 if case["out"] == F32 else 2
    bytes_of = {"matmul": m * k + n * k + m * n * e + 4 * (m + n), "grad_input": 2 * m * n + n * k + m * k * e + 4 * n,
                "grad_weight": 2 * m * n + m * k + n * k * e + 4 * m}
    return {"bytes": bytes_of[kind], "flops": 2.0 * m * n * k}


def exact(case, seed):
    """The operators' definitions in 64 bits.  What is rounded by definition (the sum that the residual stream keeps, the
    codes) is rounded once, from 64 bits."""
    s, kind = prepare(case, seed), case["kind"]
    if kind in ("checkpoint", "norm"):
        if kind == "checkpoint":
            y = s["x"].double()
        else:
            h = s["x"].double() + (0.0 if s["residual"] is None else s["residual"].double())
            kept = h.to(s["x"].dtype).double()
            rstd = (kept.square().sum(dim=1) / case["cols"] + EPS).rsqrt()
            y = kept * rstd.unsqueeze(1) * s["weight"].double()
        top = y.abs().max(dim=1).values
        step = torch.exp2(torch.ceil(torch.log2(top / 127.0)).clamp(-126, 121))
        step = torch.where(top / 127.0 > step, step * 2.0, step)  # (a logarithm next to a whole number)
        step = torch.where(top / 127.0 <= step / 2.0, step / 2.0, step).clamp(min=2.0 ** -126)
        step = torch.where(top > 0, step, torch.zeros_like(step))
        code = torch.where(top.unsqueeze(1) > 0, y / step.unsqueeze(1), torch.zeros_like(y)).round().clamp(-127, 127)
        out = {"values": code * step.unsqueeze(1), "scales": step}
        return out if kind == "checkpoint" else {**out, "rstd": rstd, "h": h}
    if kind == "norm_grad":
        h = s["x"].double() if s["x"] is not None else s["codes"].double() * s["scales"].double().unsqueeze(1)
        rstd, dy, w = s["rstd"].double().unsqueeze(1), s["dy"].double(), s["weight"].double()
        along = (dy * w * h).sum(dim=1, keepdim=True) / case["cols"]
        dx = rstd * dy * w - rstd ** 3 * along * h
        return {"dx": dx if s["dh"] is None else dx + s["dh"].double(), "dweight": (dy * h * rstd).sum(dim=0)}
    if kind == "matmul":
        return (s["a"].double() * s["a_scales"].double().unsqueeze(1)) @ (s["b"].double() * s["b_scales"].double().unsqueeze(1)).T
    if kind == "grad_input":
        return s["dy"].double() @ (s["b"].double() * s["b_scales"].double().unsqueeze(1))
    return s["dy"].double().T @ (s["a"].double() * s["a_scales"].double().unsqueeze(1))
