"""Measured cases of the training-step operators either side of the compressed exchange: log probabilities of given
tokens with their gradient (the worker's end, before deco_ef_compress) and orthogonalised updates (the server's end,
in place of the plain update).

`own` chooses the side: False computes each operator in its plain form (elementary torch operations in 32 bits,
rounded once at the end), True makes the calls a user makes of paper_2507_17346_b200.binding.

Operators and what a pass returns
  logprobs   logits [rows, vocab], targets [rows] -> logprob, entropy, lse [rows] f32, and with top > 0 the `top`
             largest logits' indices (ties to the lower index) and log probabilities [rows, top]
  grad       the same inputs, the saved lse and entropy and the gradients of logprob (and of entropy and of the top
             log probabilities where the case has them) -> gradient of the logits, in the logits' type
  orth       flat vector of matrices -> Newton-Schulz orthogonalised matrices, bf16, and with momentum the updated
             momentum buffer, f32
"""
import math

import torch

own = False

STEPS = 5
COEF = (3.4445, -4.7750, 2.0315)
EPS = 1e-7
MU = 0.95

RESNET18 = "64x147,64x576*4,128x576,128x1152*3,128x64,256x1152,256x2304*3,256x128,512x2304,512x4608*3,512x256,1000x512"
DECODER_BLOCK = "2048x2048*%d,256x2048*%d,5632x2048*%d,2048x5632*%d"


def listed():
    return [
        # one sampled token of a stream being decoded: latency of a single row, as an inference server reports it
        {"name": "logprobs 1x32000 bf16 top20", "op": "logprobs", "rows": 1, "vocab": 32000, "dtype": "bf16", "top": 20, "scale": 1.0, "mask": 0.0},
        # a decode batch at temperature 0.8 with a constrained vocabulary (half of the tokens forbidden)
        {"name": "logprobs 64x50257 f32 top5", "op": "logprobs", "rows": 64, "vocab": 50257, "dtype": "f32", "top": 5, "scale": 1.25, "mask": 0.5},
        # evaluation: log probabilities of a ragged batch of prompts with the most likely alternatives
        {"name": "logprobs 1999x50257 bf16 top8", "op": "logprobs", "rows": 1999, "vocab": 50257, "dtype": "bf16", "top": 8, "scale": 1.0, "mask": 0.0},
        # a training step's loss: 8 sequences of 1024 tokens over the GPT-2 vocabulary
        {"name": "logprobs 8192x50257 bf16", "op": "logprobs", "rows": 8192, "vocab": 50257, "dtype": "bf16", "top": 0, "scale": 1.0, "mask": 0.0},
        # its gradient
        {"name": "grad 8192x50257 bf16", "op": "grad", "rows": 8192, "vocab": 50257, "dtype": "bf16", "top": 0, "scale": 1.0, "mask": 0.0, "entropy": False},
        # a policy-gradient step with an entropy bonus and a term on the alternatives, f32 logits
        {"name": "grad 513x32000 f32 entropy top4", "op": "grad", "rows": 513, "vocab": 32000, "dtype": "f32", "top": 4, "scale": 1.25, "mask": 0.1, "entropy": True},
        # the gradient of one short answer
        {"name": "grad 7x50257 bf16 entropy", "op": "grad", "rows": 7, "vocab": 50257, "dtype": "bf16", "top": 0, "scale": 1.0, "mask": 0.0, "entropy": True},
        # the update of one small tensor (the first convolution of ResNet-18 as a matrix): latency
        {"name": "orth 64x147 f32", "op": "orth", "shapes": "64x147", "dtype": "f32", "momentum": False, "input": "student"},
        # every matrix of ResNet-18, odd and small sizes, momentum fed by a sparse aggregate
        {"name": "orth resnet18 f32 momentum", "op": "orth", "shapes": RESNET18, "dtype": "f32", "momentum": True, "input": "sparse"},
        # the attention matrices of GPT-2 small (12 layers), bf16 gradients with outlier rows
        {"name": "orth gpt2 attention bf16", "op": "orth", "shapes": "2304x768*12,768x768*12", "dtype": "bf16", "momentum": False, "input": "outlier"},
        # one block of the 1.1 B decoder, bf16
        {"name": "orth decoder block bf16", "op": "orth", "shapes": DECODER_BLOCK % (2, 2, 2, 1), "dtype": "bf16", "momentum": False, "input": "lowrank"},
        # four blocks of it with momentum: the bulk of a server update
        {"name": "orth 4 decoder blocks f32 momentum", "op": "orth", "shapes": DECODER_BLOCK % (8, 8, 8, 4), "dtype": "f32", "momentum": True, "input": "lowrank"},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["logprobs", "grad", "orth"])
    dtype = rng.choice(["f32", "bf16"])
    if op == "orth":
        parts = []
        for _ in range(rng.randint(1, 4)):
            rows, cols = _log_int(rng, 8, 4096), _log_int(rng, 8, 4096)
            parts.append("%dx%d*%d" % (rows, cols, rng.randint(1, 4)))
        return {"op": op, "shapes": ",".join(parts), "dtype": dtype, "momentum": rng.random() < 0.5,
                "input": rng.choice(["student", "sparse", "outlier", "lowrank"])}
    vocab = _log_int(rng, 1000, 200000)
    rows = _log_int(rng, 1, max(1, min(8192, 8192 * 25000 // vocab)))
    # alternatives are asked for where answers are given: not for the largest batches
    top = rng.choice([0, 1, 5, 20]) if rows * vocab < 60_000_000 else 0
    case = {"op": op, "rows": rows, "vocab": vocab, "dtype": dtype, "top": top,
            "scale": rng.choice([1.0, 1.25, 0.5]), "mask": rng.choice([0.0, 0.0, 0.3])}
    if op == "grad":
        case["entropy"] = rng.random() < 0.5
    return case


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _matrices(case):
    """[(offset, rows, cols)] of a case's flat vector, matrices back to back, and its length."""
    out, at = [], 0
    for part in case["shapes"].split(","):
        size, _, count = part.partition("*")
        rows, cols = (int(v) for v in size.split("x"))
        for _ in range(int(count or 1)):
            out.append((at, rows, cols))
            at += rows * cols
    return out, at


class _Handle:
    """Keeps a library handle as long as the state that uses it."""

    def __init__(self, d, matrices, mu):
        from paper_2507_17346_b200 import binding
        self.binding = binding
        self.value = binding.deco_orth_init(d, matrices, momentum=mu)

    def __del__(self):
        self.binding.deco_orth_destroy(self.value)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    dt = _dtype(case)
    if case["op"] == "orth":
        mats, d = _matrices(case)
        x = torch.randn(d, generator=g, device="cuda")
        if case["input"] == "student":                   # heavy tails: a normal over a chi of three degrees
            chi = sum(torch.randn(d, generator=g, device="cuda").square_() for _ in range(3))
            x /= (chi / 3.0).sqrt_()
        elif case["input"] == "sparse":                  # what the server receives: 8 % of the entries, the largest
            x = torch.where(x.abs() > 1.75, x, torch.zeros_like(x))
        else:
            for at, rows, cols in mats:
                w = x[at:at + rows * cols].view(rows, cols)
                if case["input"] == "outlier":           # one row in a hundred fifty times as large
                    w[::100] *= 50.0
                else:                                    # a few tokens' outer products over a floor of noise
                    u = torch.randn(rows, 32, generator=g, device="cuda")
                    v = torch.randn(32, cols, generator=g, device="cuda")
                    w.mul_(0.3).add_(u @ (v / torch.arange(1, 33, device="cuda")[:, None]))
        x *= 0.01
        state = {"case": case, "x": x.to(dt), "mats": mats, "d": d, "mu": MU if case["momentum"] else 0.0}
        state["m"] = 0.1 * torch.randn(d, generator=g, device="cuda") if case["momentum"] else None
        state["out"] = torch.zeros(d, dtype=torch.bfloat16, device="cuda")
        if own:
            state["handle"] = _Handle(d, mats, state["mu"])
        return state
    rows, vocab, top = case["rows"], case["vocab"], case["top"]
    logits = torch.randn(rows, vocab, generator=g, device="cuda", dtype=dt).mul_(2.5)
    target = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    likely = logits.argmax(dim=1)                        # a trained model finds many tokens likely
    hit = torch.rand(rows, generator=g, device="cuda") < 0.6
    target = torch.where(hit, likely, target)
    logits[torch.arange(rows, device="cuda")[hit], target[hit]] += 6.0
    if case["mask"]:                                     # forbidden tokens; the target is allowed
        keep = logits.gather(1, target[:, None])
        logits.masked_fill_(torch.rand(rows, vocab, generator=g, device="cuda") < case["mask"], -math.inf)
        logits.scatter_(1, target[:, None], keep)
    ignored = torch.rand(rows, generator=g, device="cuda") < 0.02
    target = torch.where(ignored & (torch.arange(rows, device="cuda") > 0), torch.full_like(target, -100), target)
    state = {"case": case, "logits": logits, "target": target}
    if case["op"] == "logprobs":
        for name in ("logprob", "entropy", "lse"):
            state[name] = torch.empty(rows, device="cuda")
        state["top_idx"] = torch.empty(rows, top, dtype=torch.int32, device="cuda")
        state["top_logprob"] = torch.empty(rows, top, device="cuda")
    else:                                                # what the forward pass saved
        with torch.no_grad():
            x = logits.float() * case["scale"]
            state["lse"] = torch.logsumexp(x, 1)
            x -= state["lse"][:, None]
            state["entropy"] = -(x.exp() * x.clamp_min(-1e30)).sum(1)
            del x
        state["top_idx"] = logits.float().topk(top, dim=1).indices.int().contiguous() if top else None
        state["g"] = torch.randn(rows, generator=g, device="cuda") / rows
        state["g_entropy"] = torch.full((rows,), 0.01 / rows, device="cuda") if case["entropy"] else None
        state["g_top"] = torch.randn(rows, top, generator=g, device="cuda") / rows if top else None
        state["dx"] = torch.empty_like(logits)
    return state


def _plain_logprobs(s):
    c = s["case"]
    raw = s["logits"].float()
    x = raw * c["scale"]
    m = x.amax(1, keepdim=True)
    x -= m
    p = x.exp()
    z = p.sum(1, keepdim=True)
    logz = z.log()
    entropy = (logz - (p * x.clamp_min(-1e30)).sum(1, keepdim=True) / z).squeeze(1)
    x -= logz
    t = s["target"]
    logprob = torch.where(t >= 0, x.gather(1, t.clamp_min(0)[:, None]).squeeze(1), torch.zeros_like(entropy))
    out = {"logprob": logprob, "entropy": entropy, "lse": (m + logz).squeeze(1)}
    if c["top"]:
        at = raw.sort(dim=1, descending=True, stable=True).indices[:, :c["top"]]
        out["top_idx"] = at.int()
        out["top_logprob"] = x.gather(1, at)
    return out


def _plain_grad(s):
    c = s["case"]
    lp = s["logits"].float() * c["scale"] - s["lse"][:, None]
    p = lp.exp()
    g = torch.where(s["target"] >= 0, s["g"], torch.zeros_like(s["g"]))
    total = g if s["g_top"] is None else g + s["g_top"].sum(1)
    dx = p * -total[:, None]
    if s["g_entropy"] is not None:
        dx -= p * (lp.clamp_min(-1e30) + s["entropy"][:, None]) * s["g_entropy"][:, None]
    dx.scatter_add_(1, s["target"].clamp_min(0)[:, None], g[:, None])
    if s["g_top"] is not None:
        dx.scatter_add_(1, s["top_idx"].long(), s["g_top"])
    return (dx * c["scale"]).to(s["logits"].dtype)


def _plain_orth(s):
    x = s["x"].float()
    if s["m"] is not None:
        s["m"].mul_(s["mu"]).add_(x)
        x = s["m"]
    shapes = {}
    for at, rows, cols in s["mats"]:
        shapes.setdefault((rows, cols), []).append(at)
    for (rows, cols), ats in shapes.items():
        y = torch.stack([x[at:at + rows * cols].view(rows, cols) for at in ats])
        y = y / (y.square().sum((1, 2), keepdim=True).sqrt() + EPS)
        y = y.transpose(1, 2) if rows > cols else y
        for _ in range(STEPS):
            a = y @ y.transpose(1, 2)
            y = COEF[0] * y + (COEF[1] * a + COEF[2] * (a @ a)) @ y
        y = (y.transpose(1, 2) if rows > cols else y).to(torch.bfloat16)
        for at, w in zip(ats, y):
            s["out"][at:at + rows * cols].view(rows, cols).copy_(w)
    return {"out": s["out"]} if s["m"] is None else {"out": s["out"], "momentum": s["m"]}


def run(s):
    op = s["case"]["op"]
    if not own:
        return {"logprobs": _plain_logprobs, "grad": _plain_grad, "orth": _plain_orth}[op](s)
    from paper_2507_17346_b200 import binding as B
    c = s["case"]
    if op == "orth":
        B.deco_orth_run(s["handle"].value, s["x"], s["out"], momentum=s["m"])
        return {"out": s["out"]} if s["m"] is None else {"out": s["out"], "momentum": s["m"]}
    if op == "grad":
        B.deco_token_logprobs_grad(s["logits"], s["target"], s["lse"], s["dx"], g_logprob=s["g"], entropy=s["entropy"],
                                   g_entropy=s["g_entropy"], top_idx=s["top_idx"], g_top=s["g_top"], scale=c["scale"])
        return s["dx"]
    top = c["top"]
    B.deco_token_logprobs(s["logits"], s["target"], s["logprob"], entropy=s["entropy"], lse=s["lse"], scale=c["scale"],
                          top_idx=s["top_idx"] if top else None, top_logprob=s["top_logprob"] if top else None)
    out = {"logprob": s["logprob"], "entropy": s["entropy"], "lse": s["lse"]}
    if top:
        out["top_idx"], out["top_logprob"] = s["top_idx"], s["top_logprob"]
    return out


def work(case):
    if case["op"] == "orth":
        # the two symmetric products of a step need one triangle each
        size = 4 if case["dtype"] == "f32" else 2
        nbytes = flops = 0
        for _, rows, cols in _matrices(case)[0]:
            m, n = min(rows, cols), max(rows, cols)
            nbytes += m * n * (size + 2 + (8 if case["momentum"] else 0))
            flops += STEPS * (3 * m * m * n + m * m * m)
        return {"bytes": nbytes, "flops": flops}
    rows, vocab, top = case["rows"], case["vocab"], case["top"]
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "logprobs":
        return {"bytes": rows * vocab * size + rows * (8 + 12 + 8 * top), "flops": 6 * rows * vocab}
    return {"bytes": 2 * rows * vocab * size + rows * (8 + 16 + 8 * top), "flops": 6 * rows * vocab}


def exact(case, seed):
    global own
    was, own = own, False                                # inputs alone: no handle
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "orth":
        x = s["x"].double()
        if case["momentum"]:
            x = x + s["m"].double() * MU
        out = torch.zeros(s["d"], dtype=torch.float64, device="cuda")
        for at, rows, cols in s["mats"]:
            w = x[at:at + rows * cols].view(rows, cols)
            w = w / (w.pow(2).sum().sqrt() + EPS)
            for _ in range(STEPS):
                if rows <= cols:
                    gram = torch.mm(w, w.t())
                    w = torch.mm(COEF[0] * torch.eye(rows, dtype=w.dtype, device=w.device)
                                 + torch.mm(gram, COEF[1] * torch.eye(rows, dtype=w.dtype, device=w.device) + COEF[2] * gram), w)
                else:
                    gram = torch.mm(w.t(), w)
                    w = torch.mm(w, COEF[0] * torch.eye(cols, dtype=w.dtype, device=w.device)
                                 + torch.mm(gram, COEF[1] * torch.eye(cols, dtype=w.dtype, device=w.device) + COEF[2] * gram))
            out[at:at + rows * cols] = w.reshape(-1)
        return {"out": out, "momentum": x} if case["momentum"] else {"out": out}
    outs, step = [], max(1, 60_000_000 // case["vocab"])
    for lo in range(0, case["rows"], step):              # in blocks of rows: 64-bit copies are large
        z = s["logits"][lo:lo + step].double() * case["scale"]
        t = s["target"][lo:lo + step]
        lse = torch.logsumexp(z, 1)
        lp = z - lse[:, None]
        p = torch.softmax(z, 1)
        entropy = torch.special.entr(p).sum(1)
        if case["op"] == "logprobs":
            logprob = torch.where(t < 0, 0.0, lp[torch.arange(len(t), device="cuda"), t.clamp_min(0)])
            part = {"logprob": logprob, "entropy": entropy, "lse": lse}
            if case["top"]:
                at = s["logits"][lo:lo + step].double().sort(dim=1, descending=True, stable=True).indices[:, :case["top"]]
                part["top_logprob"] = torch.take_along_dim(lp, at, 1)
            outs.append(part)
            continue
        # d logprob_t / d z = onehot(t) - p;  d entropy / d z = -p (lp + entropy);  z = scale * logits
        one = torch.zeros_like(z)
        one[torch.arange(len(t), device="cuda"), t.clamp_min(0)] = torch.where(t < 0, 0.0, s["g"][lo:lo + step].double())
        if s["g_top"] is not None:
            one.scatter_add_(1, s["top_idx"][lo:lo + step].long(), s["g_top"][lo:lo + step].double())
        dz = one - p * one.sum(1, keepdim=True)
        if s["g_entropy"] is not None:
            dz -= s["g_entropy"][lo:lo + step, None].double() * torch.where(p > 0, p * (lp + entropy[:, None]), 0.0)
        outs.append(dz * case["scale"])
    if case["op"] == "grad":
        return torch.cat(outs)
    whole = {k: torch.cat([o[k] for o in outs]) for k in outs[0]}
    if case["top"]:
        whole["top_idx"] = None
    return whole
