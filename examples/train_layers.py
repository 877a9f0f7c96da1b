"""A small language model on n workers of a tree: forward and backward pass
with the layer operators on 8-bit rows, then a RelaySum round.

Every worker has its own text (a Markov chain over the tokens, its rows mixed
with a chain that all share) and its own model, a row of x[n, d]: a token
embedding, `blocks` sub-layers

    s = h + r;  y = norm(s);  h = W2 relu(W1 y);  r = s

and a projection of the last norm onto the tokens.  There is no attention: a
token is predicted from the one before it, which is all that a Markov chain
needs.  Weights are views into the
rows of x, packed once a round; their gradients are written into the rows of
g.  What the backward pass needs stays in 8 bits: y and relu(W1 y), which the
products multiply anyway, and s for the norm.  Activations and gradients
between the operators are bfloat16.

    python examples/train_layers.py [--workers 16] [--rounds 200]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2110_04175_amd as rs  # noqa: E402
import workloads as wl  # noqa: E402
from paper_2110_04175_amd import layer  # noqa: E402


class Model:
    """The layout of a model in a row: named views of x or g."""

    def __init__(self, vocab: int, width: int, hidden: int, blocks: int):
        self.vocab, self.width, self.hidden, self.blocks = vocab, width, hidden, blocks
        shapes = {"embedding": (vocab, width)}
        for b in range(blocks):
            shapes |= {f"norm{b}": (width,), f"up{b}": (hidden, width), f"down{b}": (width, hidden)}
        shapes |= {"norm": (width,), "out": (vocab, width)}
        self.at, self.d = {}, 0
        for name, shape in shapes.items():
            size = torch.Size(shape).numel()
            self.at[name] = (self.d, size, shape)
            self.d += size

    def view(self, rows, name: str):
        start, size, shape = self.at[name]
        part = rows[:, start:start + size]
        return part if len(shape) == 1 else part.unflatten(1, shape)

    def init(self, rows, seed: int) -> None:
        """The same values in every row."""
        gen = torch.Generator(device=rows.device).manual_seed(seed)
        for name, (_, _, shape) in self.at.items():
            if len(shape) == 1:
                self.view(rows, name).fill_(1.0)
            else:
                std = 1.0 if name == "embedding" else shape[1] ** -0.5
                v = torch.empty(shape, device=rows.device).normal_(0.0, std, generator=gen)
                self.view(rows, name).copy_(v.expand(rows.shape[0], *shape))

    def gradients(self, x, g, tokens, targets):
        """Writes every worker's gradient at x into g; the workers' losses."""
        bf = torch.bfloat16
        n = x.shape[0]
        packed = {name: layer.pack(self.view(x, name)) for name in self.at
                  if name.startswith(("up", "down", "out"))}
        r = torch.gather(self.view(x, "embedding"), 1,
                         tokens.unsqueeze(-1).expand(-1, -1, self.width)).to(bf)
        h, kept = None, []

        def norm(name):
            # The first norm has no sub-layer before it to add.
            if h is None:
                return layer.rmsnorm(r, None, self.view(x, name))
            return layer.rmsnorm(h, r, self.view(x, name))

        for b in range(self.blocks):
            r, y, rstd, saved = norm(f"norm{b}")
            u = layer.linear(y, packed[f"up{b}"])
            a = layer.pack(torch.relu(u))
            h = layer.linear(a, packed[f"down{b}"])
            kept.append((y, rstd, saved, u > 0, a))
        _, y, rstd, saved = norm("norm")
        logits = layer.linear(y, packed["out"], torch.float32)

        log_p = torch.log_softmax(logits, -1)
        at = targets.unsqueeze(-1)
        losses = -log_p.gather(2, at)[..., 0].mean(1)
        dlogits = log_p.exp()
        dlogits.scatter_add_(2, at, torch.full(at.shape, -1.0, device=x.device))
        dlogits = dlogits.div_(tokens.shape[1]).to(bf)

        layer.linear_backward_weight(dlogits, y, self.view(g, "out"))
        dy = layer.linear_backward_input(dlogits, packed["out"])
        ds = layer.rmsnorm_backward(dy, None, saved, rstd, self.view(x, "norm"), self.view(g, "norm"))
        for b in reversed(range(self.blocks)):
            y, rstd, saved, positive, a = kept[b]
            layer.linear_backward_weight(ds, a, self.view(g, f"down{b}"))
            du = layer.linear_backward_input(ds, packed[f"down{b}"]) * positive
            layer.linear_backward_weight(du, y, self.view(g, f"up{b}"))
            dy = layer.linear_backward_input(du, packed[f"up{b}"])
            ds = layer.rmsnorm_backward(dy, ds, saved, rstd, self.view(x, f"norm{b}"),
                                        self.view(g, f"norm{b}"))
        # The embedding's gradient: each token's rows of ds summed, in 32 bits.
        picked = torch.nn.functional.one_hot(tokens, self.vocab).float().transpose(1, 2).contiguous()
        self.view(g, "embedding").copy_(torch.bmm(picked, ds.float()))
        return losses


def chains(n: int, vocab: int, own: float, seed: int, device):
    """Transition probabilities [n, vocab, vocab]: a chain that all workers
    share, mixed with `own` parts of a worker's own."""
    gen = torch.Generator(device=device).manual_seed(seed)

    def chain(k):
        return torch.softmax(3.0 * torch.randn(k, vocab, vocab, generator=gen, device=device), -1)

    return (1 - own) * chain(1) + own * chain(n)


def sample(p, length: int, gen):
    """Tokens [n, length + 1] of each worker's chain."""
    n, vocab, _ = p.shape
    out = [torch.randint(vocab, (n, 1), generator=gen, device=p.device)]
    for _ in range(length):
        row = p[torch.arange(n, device=p.device), out[-1][:, 0]]
        out.append(torch.multinomial(row, 1, generator=gen))
    return torch.cat(out, 1)


def train(workers=16, rounds=200, vocab=61, width=96, hidden=200, blocks=2, tokens=256, seed=0,
          lr=2e-3, report=None):
    """Trains and returns the mean loss of every round."""
    dev = torch.device("cuda")
    model = Model(vocab, width, hidden, blocks)
    x = torch.empty(workers, model.d, device=dev)
    model.init(x, seed)
    g = torch.zeros_like(x)
    m, v = torch.zeros_like(x), torch.zeros_like(x)
    p = chains(workers, vocab, 0.3, seed + 1, dev)
    gen = torch.Generator(device=dev).manual_seed(seed + 2)
    losses = []
    with rs.RelaySum(workers, model.d, wl.heap_edges(workers)) as h:
        for t in range(rounds):
            text = sample(p, tokens, gen)
            loss = model.gradients(x, g, text[:, :-1], text[:, 1:].contiguous())
            h.step_ex(x, g, m, v, optimizer="adam", lr=lr, beta1=0.9, beta2=0.999, eps=1e-8,
                      adam_step=t + 1)
            losses.append(float(loss.mean()))
            if report and (t % 20 == 0 or t == rounds - 1):
                report(f"round {t:4d}  loss {losses[-1]:.4f}  "
                       f"consensus distance {h.consensus_distance(x)[0]:.4g}")
    return losses


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n", 1)[0])
    ap.add_argument("--workers", type=int, default=16)
    ap.add_argument("--rounds", type=int, default=200)
    a = ap.parse_args()
    train(a.workers, a.rounds, report=lambda line: print(line, flush=True))


if __name__ == "__main__":
    main()
