"""Measured cases of what lies inside a worker's gradient, between the loss and deco_ef_compress: layer norm with its
gradient, 8-bit checkpoints of activations, and the backward pass that reads them (layer norm's gradient and a linear
layer's weight gradient, written where the compressed exchange takes it from).

`own` chooses the side: False computes each operator in its plain form (elementary torch operations in 32 bits,
rounded once at the end), True makes the calls a user makes of paper_2507_17346_b200.binding.

A checkpoint in 8 bits holds, for every 32 consecutive entries of a row (the last block of a row may be shorter), one
exponent byte b and 32 signed bytes q; entry j stands for q_j 2^(b - 127).  The exponent is the smallest one for which
the block's largest magnitude still rounds to at most 127, and at least 1; q = entry / 2^(b - 127) rounded to even.

Operators and what a pass returns
  norm       x [rows, cols] (+ residual) -> y, mean, rstd (and the residual sum; and the values of its checkpoint)
  norm_grad  x or its checkpoint, mean, rstd, weight, dy (+ the gradient that bypasses the norm) -> dx, dweight, dbias
  pack       x -> the values of its checkpoint, through memory
  wgrad      dy [tokens, out], checkpoint of the input [tokens, in] -> dw, db
"""
import math

import torch

own = False

EPS = 1e-5
BLOCK = 32


def listed():
    return [
        # one token of a stream being decoded, width of GPT-2 small: latency
        {"name": "norm 1x768 bf16", "op": "norm", "rows": 1, "cols": 768, "dtype": "bf16", "add": True, "keep8": False},
        # a training step's norm behind a residual sum: 8 sequences of 1024 tokens, GPT-2 small
        {"name": "norm 8192x768 bf16 residual", "op": "norm", "rows": 8192, "cols": 768, "dtype": "bf16", "add": True, "keep8": False},
        # a ragged batch, an odd width, f32, with the input kept in 8 bits
        {"name": "norm 1999x1001 f32 keep8", "op": "norm", "rows": 1999, "cols": 1001, "dtype": "f32", "add": False, "keep8": True},
        # the 1.1 B decoder's width, 16 sequences of 2048 tokens, residual sum kept in 8 bits
        {"name": "norm 32768x2048 bf16 residual keep8", "op": "norm", "rows": 32768, "cols": 2048, "dtype": "bf16", "add": True, "keep8": True},
        # the gradients of the same: GPT-2 small from saved inputs
        {"name": "norm_grad 8192x768 bf16 residual", "op": "norm_grad", "rows": 8192, "cols": 768, "dtype": "bf16", "add": True, "saved": "x"},
        # the ragged f32 batch
        {"name": "norm_grad 1999x1001 f32", "op": "norm_grad", "rows": 1999, "cols": 1001, "dtype": "f32", "add": False, "saved": "x"},
        # the decoder from checkpoints in 8 bits
        {"name": "norm_grad 32768x2048 bf16 residual from 8 bits", "op": "norm_grad", "rows": 32768, "cols": 2048, "dtype": "bf16", "add": True, "saved": "8"},
        # a linear layer's input put away and taken back: the decoder's hidden layer; and a ragged f32 one
        {"name": "pack 8192x5632 bf16", "op": "pack", "rows": 8192, "cols": 5632, "dtype": "bf16"},
        {"name": "pack 333x1001 f32", "op": "pack", "rows": 333, "cols": 1001, "dtype": "f32"},
        # weight gradients: one short sequence through an odd layer, f32 gradients
        {"name": "wgrad 100x333x129 f32", "op": "wgrad", "rows": 100, "out": 333, "cols": 129, "dtype": "f32", "grad": "f32", "transposed": False},
        # GPT-2 small's attention input, kept [in][out] as that model keeps it
        {"name": "wgrad 8192x2304x768 bf16 transposed", "op": "wgrad", "rows": 8192, "out": 2304, "cols": 768, "dtype": "bf16", "grad": "f32", "transposed": True},
        # the decoder's first hidden product, bf16 gradients
        {"name": "wgrad 8192x5632x2048 bf16", "op": "wgrad", "rows": 8192, "out": 5632, "cols": 2048, "dtype": "bf16", "grad": "bf16", "transposed": False},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """Widths of models are round more often than not."""
    n = _log_int(rng, lo, hi)
    return n if n < 64 or rng.random() < 0.4 else n // 64 * 64


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "pack", "wgrad"])
    dtype = rng.choice(["f32", "bf16"])
    if op == "wgrad":
        # (three factors, together at most the largest listed product; f32 at a third of it)
        out, cols = _width(rng, 16, 8192), _width(rng, 16, 8192)
        room = 8192 * 5632 * 2048 // (out * cols) // (1 if dtype == "bf16" else 3)
        return {"op": op, "rows": _log_int(rng, 16, max(16, min(32768, room))), "out": out, "cols": cols, "dtype": dtype,
                "grad": rng.choice(["f32", "bf16"]), "transposed": rng.random() < 0.5}
    cols = _width(rng, 32, 8192)
    entries = 64_000_000 if dtype == "bf16" else 32_000_000
    if op == "pack":
        entries = entries * 2 // 3
    case = {"op": op, "rows": _log_int(rng, 1, min(32768, entries // cols)), "cols": cols, "dtype": dtype}
    if op == "norm":
        case.update(add=rng.random() < 0.5, keep8=rng.random() < 0.5)
    elif op == "norm_grad":
        case.update(add=rng.random() < 0.5, saved=rng.choice(["x", "8"]))
    return case


def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _blocks(cols):
    return (cols + BLOCK - 1) // BLOCK


def _power(e):
    """2^e in 32 bits from its bits, e in [-126, 127] (a power by way of logarithms need not be exact)."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _checkpoint(x):
    """-> (codes [rows, 32 blocks] int8, exponent bytes [rows, blocks] uint8) of x [rows, cols]."""
    rows, cols = x.shape
    n = _blocks(cols)
    v = torch.zeros(rows, n * BLOCK, device=x.device)
    v[:, :cols] = x
    v = v.view(rows, n, BLOCK)
    frac, e = torch.frexp(v.abs().amax(2))               # largest magnitude = frac 2^e, frac in [1/2, 1)
    b = (e + (frac >= 127.5 / 128).int() + (127 - 7)).clamp_min_(1)
    q = (v * _power(127 - b)[:, :, None]).round_().to(torch.int8)
    return q.view(rows, n * BLOCK), b.to(torch.uint8)


def _values(codes, exps, cols):
    rows, n = exps.shape
    v = codes.view(rows, n, BLOCK).float() * _power(exps.int() - 127)[:, :, None]
    return v.view(rows, n * BLOCK)[:, :cols]


def _activations(rows, cols, dt, g):
    """A residual stream: rows of different sizes, a few wide channels, a common offset per channel."""
    x = torch.randn(rows, cols, generator=g, device="cuda")
    x *= torch.exp(0.5 * torch.randn(rows, 1, generator=g, device="cuda"))
    x += 0.3 * torch.randn(1, cols, generator=g, device="cuda")
    x[:, ::97] *= 12.0
    return x.to(dt)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    op, rows, cols, dt = case["op"], case["rows"], case["cols"], _dtype(case["dtype"])
    s = {"case": case, "x": _activations(rows, cols, dt, g)}
    new = lambda *shape, **kw: torch.empty(*shape, device="cuda", **kw)  # noqa: E731
    if op == "wgrad":
        s["codes"], s["exps"] = _checkpoint(s.pop("x").float())
        dy = torch.randn(rows, case["out"], generator=g, device="cuda")
        # most tokens' gradients are small, a few are not
        dy *= 1e-3 * torch.exp(torch.randn(rows, 1, generator=g, device="cuda"))
        s["dy"] = dy.to(dt)
        shape = (cols, case["out"]) if case["transposed"] else (case["out"], cols)
        s["dw"], s["db"] = new(shape, dtype=_dtype(case["grad"])), new(case["out"], dtype=_dtype(case["grad"]))
        return s
    if op == "pack":
        s["codes"], s["exps"] = new(rows, _blocks(cols) * BLOCK, dtype=torch.int8), new(rows, _blocks(cols), dtype=torch.uint8)
        s["y"] = torch.empty_like(s["x"])
        return s
    s["weight"] = 1.0 + 0.2 * torch.randn(cols, generator=g, device="cuda")
    s["add"] = _activations(rows, cols, dt, g) if case["add"] else None
    if op == "norm":
        s["bias"] = 0.1 * torch.randn(cols, generator=g, device="cuda")
        s["y"], s["mean"], s["rstd"] = torch.empty_like(s["x"]), new(rows), new(rows)
        s["total"] = torch.empty_like(s["x"]) if case["add"] else None
        if case["keep8"]:
            s["codes"], s["exps"] = new(rows, _blocks(cols) * BLOCK, dtype=torch.int8), new(rows, _blocks(cols), dtype=torch.uint8)
            s["kept"] = torch.empty_like(s["x"])
        return s
    x = s["x"].float()                                   # what the forward pass saved
    s["mean"] = x.mean(1)
    s["rstd"] = 1.0 / ((x - s["mean"][:, None]).square().mean(1) + EPS).sqrt()
    if case["saved"] == "8":
        s["codes"], s["exps"] = _checkpoint(x)
        del s["x"]
    del x
    dy = torch.randn(rows, cols, generator=g, device="cuda")
    dy *= 1e-3 * torch.exp(torch.randn(rows, 1, generator=g, device="cuda"))
    s["dy"] = dy.to(dt)
    if case["add"]:
        s["add"] = (1e-3 * torch.randn(rows, cols, generator=g, device="cuda")).to(dt)
    s["dx"], s["dweight"], s["dbias"] = torch.empty_like(s["dy"]), new(cols), new(cols)
    return s


def _plain_norm(s):
    c = s["case"]
    x = s["x"].float()
    out = {}
    if c["add"]:
        out["total"] = (x + s["add"].float()).to(s["x"].dtype)
        x = out["total"].float()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = 1.0 / (d.square().mean(1, keepdim=True) + EPS).sqrt()
    out["y"] = (d * rstd * s["weight"] + s["bias"]).to(s["x"].dtype)
    out["mean"], out["rstd"] = mean.squeeze(1), rstd.squeeze(1)
    if c["keep8"]:
        out["kept"] = _values(*_checkpoint(x), c["cols"]).to(s["x"].dtype)
    return out


def _plain_norm_grad(s):
    c = s["case"]
    x = s["x"].float() if c["saved"] == "x" else _values(s["codes"], s["exps"], c["cols"])
    xhat = (x - s["mean"][:, None]) * s["rstd"][:, None]
    dy = s["dy"].float()
    g = dy * s["weight"]
    dx = (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True)) * s["rstd"][:, None]
    if c["add"]:
        dx += s["add"].float()
    return {"dx": dx.to(s["dy"].dtype), "dweight": (dy * xhat).sum(0), "dbias": dy.sum(0)}


def _plain_wgrad(s):
    c = s["case"]
    x = _values(s["codes"], s["exps"], c["cols"])
    dy = s["dy"].float()
    dw = x.t() @ dy if c["transposed"] else dy.t() @ x
    return {"dw": dw.to(s["dw"].dtype), "db": dy.sum(0).to(s["db"].dtype)}


def run(s):
    c = s["case"]
    op = c["op"]
    if not own:
        if op == "pack":
            return {"y": _values(*_checkpoint(s["x"].float()), c["cols"]).to(s["x"].dtype)}
        return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "wgrad": _plain_wgrad}[op](s)
    from paper_2507_17346_b200 import binding as B
    if op == "norm":
        kept = (s["codes"], s["exps"]) if c["keep8"] else None
        B.deco_layernorm(s["x"], s["weight"], s["bias"], s["y"], mean=s["mean"], rstd=s["rstd"], eps=EPS,
                         add=s["add"], total=s["total"], packed=kept)
        out = {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
        if c["add"]:
            out["total"] = s["total"]
        if c["keep8"]:
            B.deco_unpack8(kept, s["kept"])
            out["kept"] = s["kept"]
        return out
    if op == "norm_grad":
        B.deco_layernorm_grad(s["x"] if c["saved"] == "x" else (s["codes"], s["exps"]), s["mean"], s["rstd"],
                              s["weight"], s["dy"], s["dx"], dweight=s["dweight"], dbias=s["dbias"], add=s["add"])
        return {"dx": s["dx"], "dweight": s["dweight"], "dbias": s["dbias"]}
    if op == "pack":
        B.deco_pack8(s["x"], (s["codes"], s["exps"]))
        B.deco_unpack8((s["codes"], s["exps"]), s["y"])
        return {"y": s["y"]}
    B.deco_weight_grad8(s["dy"], (s["codes"], s["exps"]), s["dw"], db=s["db"], transposed=c["transposed"])
    return {"dw": s["dw"], "db": s["db"]}


def work(case):
    rows, cols, op = case["rows"], case["cols"], case["op"]
    n, size = rows * cols, 4 if case["dtype"] == "f32" else 2
    packed = rows * _blocks(cols) * (BLOCK + 1)
    if op == "pack":                                     # x in, checkpoint out and in, its values out
        return {"bytes": 2 * n * size + 2 * packed, "flops": 4 * n}
    if op == "norm":
        nbytes = 2 * n * size + 8 * rows + 8 * cols
        nbytes += 2 * n * size if case["add"] else 0
        nbytes += 2 * packed + n * size if case["keep8"] else 0
        return {"bytes": nbytes, "flops": 8 * n}
    if op == "norm_grad":
        nbytes = (n * size if case["saved"] == "x" else packed) + 2 * n * size + 8 * rows + 12 * cols
        return {"bytes": nbytes + (n * size if case["add"] else 0), "flops": 12 * n}
    out, gsize = case["out"], 4 if case["grad"] == "f32" else 2
    return {"bytes": rows * out * size + packed + (cols + 1) * out * gsize, "flops": 2 * n * out}


def _exact_step(e):
    """2^e in 64 bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_checkpoint(x):
    """Values of the checkpoint of x (64 bits, finite), from the definition."""
    rows, cols = x.shape
    out = torch.zeros_like(x)
    for lo in range(0, cols, BLOCK):
        part = x[:, lo:lo + BLOCK]
        top = part.abs().max(1, keepdim=True).values
        step = _exact_step(torch.frexp(top / 127.5).exponent.clamp_min(-126))    # the smallest 2^e above top / 127.5
        out[:, lo:lo + BLOCK] = torch.round(part / step) * step
    return out


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    op, cols = case["op"], case["cols"]
    if op == "pack":
        return {"y": _exact_checkpoint(s["x"].double())}
    if op == "norm":
        x = s["x"].double()
        out = {}
        if case["add"]:                                  # the norm and the checkpoint are those of the stored sum
            out["total"] = x + s["add"].double()
            x = out["total"].to(s["x"].dtype).double()
        var, mean = torch.var_mean(x, dim=1, correction=0)
        out["mean"], out["rstd"] = mean, torch.rsqrt(var + EPS)
        out["y"] = torch.addcmul(s["bias"].double(), (x - mean[:, None]) * out["rstd"][:, None], s["weight"].double())
        if case["keep8"]:
            out["kept"] = _exact_checkpoint(x)
        return out
    if op != "wgrad" and case["saved"] == "x":
        x = s["x"].double()
    else:
        step = _exact_step(s["exps"].long() - 127)
        x = (s["codes"].double() * step.repeat_interleave(BLOCK, 1))[:, :cols]
    dy = s["dy"].double()
    if op == "wgrad":
        dw = torch.einsum("ti,to->io" if case["transposed"] else "ti,to->oi", x, dy)
        return {"dw": dw, "db": dy.sum(0)}
    rstd = s["rstd"].double()[:, None]
    xhat = (x - s["mean"].double()[:, None]) * rstd
    dxhat = dy * s["weight"].double()
    # (dxhat - its mean - xhat <dxhat, xhat> / cols) rstd
    dx = rstd * (dxhat - dxhat.sum(1, keepdim=True) / cols - xhat * (dxhat * xhat).sum(1, keepdim=True) / cols)
    if case["add"]:
        dx = dx + s["add"].double()
    return {"dx": dx, "dweight": (dy * xhat).sum(0), "dbias": dy.sum(0)}
