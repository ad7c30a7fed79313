"""Norm, checkpoints in 8 bits and the gradients that read them together, as the example's model uses them.

The gradient of the whole is compared with the formulas in 64 bits, from the checkpoints' own values.  Every product
of torch's is fp32, 2^-24 a term over up to 512 terms in blocks, and gradients pass through three of them: 1e-5 of the largest
entry of each part bounds that (64 eps a product would be 4e-6)."""
import pytest
import torch

from paper_2507_17346_b200 import binding as B
from paper_2507_17346_b200 import example_lm

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2507_17346_b200 import build
    build.build()
    B.load()
    torch.cuda.set_device(0)


def values(packed, cols):
    codes, exps = packed
    step = ((exps.long() - 127 + 1023) << 52).view(torch.float64)
    return (codes.double() * step.repeat_interleave(32, 1))[:, :cols]


@pytest.mark.parametrize("vocab,width,hidden,rows", [(64, 32, 64, 100), (101, 45, 70, 333), (512, 128, 256, 1024)])
def test_gradient_of_the_model(vocab, width, hidden, rows):
    model = example_lm.NormModel(vocab, width, hidden)
    chain = example_lm.Chain(vocab)
    tokens, targets = chain.sample(rows)
    flat = torch.full((model.d,), 9.0, device="cuda")
    logprob = model.gradient(tokens, targets, flat)
    h, logits, (x8, mean, rstd, y8, h8) = model.forward(tokens)
    embed, hid, head = (t.double() for t in model.views(model.params))
    weight = model.norm_views(model.params)[0].double()
    x, y, hv = values(x8, width), values(y8, width), values(h8, hidden)
    # the checkpoints stand for what was computed, to half a step
    assert (x - embed[tokens]).abs().max() <= embed[tokens].abs().max() * 2.0 ** -7
    assert (hv - h.double()).abs().max() <= h.double().abs().max() * 2.0 ** -7
    lp = torch.log_softmax(logits.double(), 1)
    assert (lp[torch.arange(rows, device="cuda"), targets] - logprob).abs().max() < 1e-5
    dl = lp.exp()
    dl[torch.arange(rows, device="cuda"), targets] -= 1
    dl /= rows
    dh = (dl @ head) * (hv > 0)
    dy = dh @ hid.t()
    xhat = (x - mean.double()[:, None]) * rstd.double()[:, None]
    g = dy * weight
    dx = rstd.double()[:, None] * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    d_embed = torch.zeros_like(embed).index_add_(0, tokens, dx)
    want = [d_embed, y.t() @ dh, dl.t() @ hv, (dy * xhat).sum(0), dy.sum(0)]
    got = model.views(flat) + list(model.norm_views(flat))
    for a, b in zip(got, want):
        assert a.shape == b.shape
        assert (a.double() - b).abs().max() <= 1e-5 * b.abs().max() + 1e-9


def test_the_example_runs():
    losses, model, chain = example_lm.train(steps=3, workers=2, vocab=64, width=32, hidden=64, batch=128, norm8=True)
    assert len(losses) == 3 and all(v == v and v < 100 for v in losses)
    assert torch.isfinite(model.params).all()
    weight, bias = model.norm_views(model.params)
    assert (weight != 1).any() and (bias != 0).any()              # they learn, by the plain update
    found, entropy = example_lm.alternatives(model, 7)
    assert len(found) == 5 and entropy > 0
    # without the norm the model is what it was
    assert example_lm.Model(64, 32, 64).d == 64 * 32 + 32 * 64 + 64 * 64


def test_a_run_captured_and_replayed():
    """Forward, checkpoints and all gradients of a layer in one graph: new inputs, same buffers."""
    rows, width, out = 700, 96, 130
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    new = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, add, dz = (new(*s).bfloat16() for s in ((rows, width), (rows, width), (rows, out)))
    w, weight, bias = new(out, width).bfloat16(), new(width), new(width)
    flat = torch.zeros(out * width + out + 2 * width, device="cuda")
    dw, db = flat[:out * width].view(out, width), flat[out * width:out * width + out]
    d_weight, d_bias = flat[out * width + out:out * width + out + width], flat[out * width + out + width:]
    total, y, dx = (torch.empty_like(x) for _ in range(3))
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    t8, y8 = B.packed8_empty(rows, width), B.packed8_empty(rows, width)

    def step():
        B.deco_layernorm(x, weight, bias, y, mean=mean, rstd=rstd, add=add, total=total, packed=t8)
        B.deco_pack8(y, y8)
        B.deco_weight_grad8(dz, y8, dw, db=db)
        dy = dz @ w
        B.deco_layernorm_grad(t8, mean, rstd, weight, dy, dx, dweight=d_weight, dbias=d_bias, add=add)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(2):
        x.copy_(new(rows, width))
        dz.copy_(new(rows, out))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (flat, dx, total, y, *t8, *y8)]
        for t in (flat, dx, total, y):
            t.fill_(7.0)
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (flat, dx, total, y, *t8, *y8)))
