"""The example's model with 8-bit checkpoints: its forward and its backward pass are of one function, and nothing but checkpoints is
kept between them.

Tolerance of the logits: a product of n terms in fp32 is off by at most (n + 2) 2^-24 of the terms' magnitudes."""
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


def model_with_small_units(vocab, width, hidden):
    """A sixteenth of the hidden units is a thousandth of the others: active, but 0 in 8 bits."""
    model = example_lm.NormModel(vocab, width, hidden)
    model.views(model.params)[1][:, ::16] *= 1e-3
    return model


@pytest.mark.parametrize("vocab,width,hidden,rows", [(64, 32, 64, 100), (101, 45, 70, 333), (512, 128, 256, 1024)])
def test_the_head_is_given_what_the_backward_pass_has(vocab, width, hidden, rows):
    model = model_with_small_units(vocab, width, hidden)
    tokens, targets = example_lm.Chain(vocab).sample(rows)
    _, logits, (_, _, _, y8, h8) = model.forward(tokens)
    _, hid, head = (t.double() for t in model.views(model.params))
    h = values(h8, hidden)
    lost = (values(y8, width) @ hid > 0) & (h == 0)
    assert lost[:, ::16].any()                                     # (else nothing is tested)
    want, total = h @ head.t(), h.abs() @ head.abs().t()
    assert ((logits.double() - want).abs() <= (hidden + 2) * 2.0 ** -24 * total + 1e-30).all()
    # so a unit that the checkpoint has as 0 adds nothing to the loss, and passes no gradient on
    flat = torch.empty(model.d, device="cuda")
    model.gradient(tokens, targets, flat)
    d_head = model.views(flat)[2]
    never = (h == 0).all(0)
    assert (d_head[:, never] == 0).all() and (model.views(flat)[1][:, never] == 0).all()


def test_only_checkpoints_outlive_the_forward_pass(monkeypatch):
    vocab, width, hidden, rows = 512, 128, 256, 4096
    model = example_lm.NormModel(vocab, width, hidden)
    tokens, targets = example_lm.Chain(vocab).sample(rows)
    flat = torch.empty(model.d, device="cuda")
    model.gradient(tokens, targets, flat)                          # (libraries make their workspaces)
    held, plain = [], B.deco_token_logprobs

    def loss(*args, **kw):
        held.append(torch.cuda.memory_allocated())
        plain(*args, **kw)

    monkeypatch.setattr(B, "deco_token_logprobs", loss)
    before = torch.cuda.memory_allocated()
    model.gradient(tokens, targets, flat)
    kept = rows * (2 * width + hidden) * 33 // 32 + 4 * 4 * rows   # three checkpoints; mean, rstd and the loss's two
    assert held[0] - before <= 4 * rows * vocab + kept + (1 << 16)
