"""A small language model trained by simulated workers over the compressed exchange.

    python -m paper_2507_17346_b200.example_lm [--steps N] [--workers N] [--delta R] [--tau T]

Every worker computes the loss of its own tokens and the gradient of its logits
(``deco_token_logprobs``, ``deco_token_logprobs_grad``), the messages are compressed and summed
(``deco_ef_compress``, ``deco_aggregate_stale``), and the server updates the parameters with
orthogonalised directions (``deco_apply_update_orth``).  The model is an embedding, one hidden
layer and a head over a synthetic Markov chain whose entropy rate is known, so that the loss has
something to fall to; its few products are torch's.
"""
import argparse

import torch

from . import binding as B


class Model:
    """logits = relu(embed[token] @ hidden) @ head^T, parameters and gradients as flat vectors."""

    def __init__(self, vocab, width, hidden, seed=0, device="cuda"):
        self.shapes = [("embed", vocab, width), ("hidden", width, hidden), ("head", vocab, hidden)]
        self.matrices, at = [], 0
        for _, rows, cols in self.shapes:
            self.matrices.append((at, rows, cols))
            at += rows * cols
        self.d = at
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.params = torch.zeros(self.d, device=device)
        for (_, rows, cols), w in zip(self.shapes, self.views(self.params)):
            w.copy_(torch.randn(rows, cols, generator=g, device=device) * cols ** -0.5)

    def views(self, flat):
        return [flat[at:at + rows * cols].view(rows, cols) for at, rows, cols in self.matrices]

    def logits(self, tokens):
        embed, hidden, head = self.views(self.params)
        x = embed[tokens]
        h = torch.relu(x @ hidden)
        return x, h, h @ head.t()

    def gradient(self, tokens, targets, out):
        """Gradient of the mean negative log probability of `targets` into the flat vector `out`;
        returns the log probabilities."""
        rows = len(tokens)
        x, h, logits = self.logits(tokens)
        logprob, lse = torch.empty(rows, device=x.device), torch.empty(rows, device=x.device)
        B.deco_token_logprobs(logits, targets, logprob, lse=lse)
        weight = torch.full((rows,), -1.0 / rows, device=x.device)
        B.deco_token_logprobs_grad(logits, targets, lse, logits, g_logprob=weight)     # in place
        _, hidden, head = self.views(self.params)
        d_embed, d_hidden, d_head = self.views(out)
        torch.mm(logits.t(), h, out=d_head)
        dh = (logits @ head) * (h > 0)
        torch.mm(x.t(), dh, out=d_hidden)
        d_embed.zero_().index_add_(0, tokens, dh @ hidden.t())
        return logprob


class Chain:
    """A Markov chain in which every token has a few likely successors."""

    def __init__(self, vocab, seed=1, device="cuda"):
        self.generator = torch.Generator(device=device)
        self.generator.manual_seed(seed)
        logits = 3.0 * torch.randn(vocab, vocab, generator=self.generator, device=device)
        self.p = torch.softmax(logits, 1)

    def sample(self, count):
        now = torch.randint(0, len(self.p), (count,), generator=self.generator, device=self.p.device)
        return now, torch.multinomial(self.p[now], 1, generator=self.generator).squeeze(1)

    def entropy_rate(self):
        return float(-(self.p * self.p.log()).sum(1).mean())


def train(steps=200, workers=4, vocab=512, width=128, hidden=256, batch=1024, delta=0.05, tau=1,
          lr=0.02, momentum=0.9, weight_decay=0.0, log=None):
    """-> (losses per step, model, chain): the mean loss over the workers' batches."""
    model, chain = Model(vocab, width, hidden), Chain(vocab)
    ctx = B.deco_init(model.d, workers, delta, tau, lr, lr_at_server=True, params=model.params)
    orth = B.deco_orth_init(model.d, model.matrices, momentum=momentum,
                            scale=B.DECO_ORTH_SCALE_SPECTRAL)
    moment = torch.zeros(model.d, device="cuda")
    grads = torch.zeros(workers, model.d, device="cuda")
    losses = []
    try:
        for step in range(steps):
            loss = 0.0
            for i in range(workers):
                tokens, targets = chain.sample(batch)
                loss = loss - model.gradient(tokens, targets, grads[i]).mean()
            B.deco_ef_compress(ctx, grads)
            B.deco_aggregate_stale(ctx)
            B.deco_apply_update_orth(ctx, orth, moment, weight_decay)
            losses.append(loss / workers)
            if log and (step % 20 == 0 or step + 1 == steps):
                log("step %4d  loss %.4f" % (step, float(losses[-1])))
        assert B.deco_get_stats(ctx)["device_status"] == 0
        B.deco_orth_get_stats(orth)
    finally:
        B.deco_orth_destroy(orth)
        B.deco_destroy(ctx)
    return [float(v) for v in losses], model, chain


def alternatives(model, token, top=5):
    """The most likely successors of one token: [(token, probability)], and the entropy."""
    tokens = torch.tensor([token], device="cuda")
    logits = model.logits(tokens)[2]
    idx = torch.empty(1, top, dtype=torch.int32, device="cuda")
    logprob, entropy = torch.empty(1, top, device="cuda"), torch.empty(1, device="cuda")
    B.deco_token_logprobs(logits, None, None, entropy=entropy, top_idx=idx, top_logprob=logprob)
    return list(zip(idx[0].tolist(), logprob[0].exp().tolist())), float(entropy)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--delta", type=float, default=0.05)
    ap.add_argument("--tau", type=int, default=1)
    args = ap.parse_args()
    losses, model, chain = train(steps=args.steps, workers=args.workers, delta=args.delta,
                                 tau=args.tau, log=print)
    print("loss %.4f -> %.4f (the chain's entropy rate: %.4f)"
          % (losses[0], losses[-1], chain.entropy_rate()))
    found, entropy = alternatives(model, 7)
    print("after token 7 (entropy %.3f): %s" % (entropy, ", ".join("%d %.3f (true %.3f)" % (t, p, chain.p[7, t])
                                                                   for t, p in found)))


if __name__ == "__main__":
    main()
