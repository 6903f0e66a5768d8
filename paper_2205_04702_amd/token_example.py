"""A small next-token model, trained and then served from 8-bit rows: the operators of
tokens.py together.

    python -m paper_2205_04702_amd.token_example [--vocab 512] [--dim 64] [--steps 300]

Tokens follow a permutation (the next one is perm[token], now and then any other).  The
model is a table of embeddings E and one of outputs W: logits = dropout(lookup(E)) W^T.
Training takes the gradients by hand: the cross entropy's to the logits, the dropout's
again from its generator, the table's by sorted tokens.  Serving keeps E in a cache of 8
bits and W as 8-bit rows: read the token's row back, quantise it, score it against W.
"""
import argparse
import math

import torch

from . import tokens as tk


def sequences(perm, n, vocab, noise, g):
    """n tokens and the ones that follow them."""
    now = torch.randint(vocab, (n,), generator=g, device="cuda")
    other = torch.randint(vocab, (n,), generator=g, device="cuda")
    jump = torch.rand(n, generator=g, device="cuda") < noise
    return now, torch.where(jump, other, perm[now])


def train(vocab, dim, steps, batch, lr=1.0, p=0.1, noise=0.05, seed=0):
    """The trained tables, the rule that the tokens followed and the loss of every step."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    perm = torch.randperm(vocab, generator=g, device="cuda")
    E = torch.randn((vocab, dim), generator=g, device="cuda") / math.sqrt(dim)
    W = torch.randn((vocab, dim), generator=g, device="cuda") / math.sqrt(dim)
    scale = math.sqrt(dim)
    grad = torch.empty_like(E)
    losses = []
    for step in range(steps):
        now, following = sequences(perm, batch, vocab, noise, g)
        x = tk.lookup(now, E, scale)
        h = tk.dropout(x, p, seed, offset=step)
        logp = torch.log_softmax(h @ W.t(), dim=1)
        losses.append(-logp.gather(1, following[:, None]).mean())
        d = logp.exp()
        d[torch.arange(batch, device="cuda"), following] -= 1.0
        dx = tk.dropout(d @ W, p, seed, offset=step)  # the mask is drawn again
        tk.lookup_grad(now, dx, vocab, scale, out=grad)
        W -= lr / batch * vocab / dim * (d.t() @ h)
        E -= lr / batch * vocab / dim * grad
    return E, W, perm, torch.stack(losses)


class Served:
    """The trained tables in 8 bits."""

    def __init__(self, E, W):
        vocab, dim = E.shape
        self.scale = math.sqrt(dim)
        self.rows, self.row_scales = tk.empty_cache(vocab, dim)
        tk.cache_write(self.rows, self.row_scales, E, torch.arange(vocab, device="cuda"))
        self.out, self.out_scales = tk.quantize(W)

    def scores(self, now):
        x = tk.cache_read(self.rows, self.row_scales, now, dtype=torch.float32) * self.scale
        return tk.product(*tk.quantize(x), self.out, self.out_scales, dtype=torch.float32)


def run(vocab=512, dim=64, steps=300, batch=4096, seed=0):
    E, W, perm, losses = train(vocab, dim, steps, batch, seed=seed)
    every = torch.arange(vocab, device="cuda")
    full = (E * math.sqrt(dim)) @ W.t()
    served = Served(E, W).scores(every)
    return {"first_loss": losses[0].item(), "last_loss": losses[-1].item(),
            "right": (full.argmax(1) == perm).double().mean().item(),
            "right_in_8_bits": (served.argmax(1) == perm).double().mean().item(),
            "off_in_8_bits": ((served - full).norm() / full.norm()).item()}


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, value in (("vocab", 512), ("dim", 64), ("steps", 300), ("batch", 4096), ("seed", 0)):
        ap.add_argument("--" + name, type=int, default=value)
    for k, v in run(**vars(ap.parse_args())).items():
        print(f"{k}: {v:.4f}")


if __name__ == "__main__":
    main()
