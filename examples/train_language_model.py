"""A small language model trained by sketched gradients, end to end on one GPU.

Every worker (simulated on the one device) takes tokens of its own: embedding, a linear layer, layer norm, logits.  The
framework's operators stand on both sides of the gradient:

    LayerNorm.forward / .backward     the hidden rows and the gradients of norm weight and bias
    TokenLogprobs.loss                loss and the gradient of the logits, in place
    HotPath.step                      the workers' gradients sketched, merged, queried; of P k candidates the k with the largest
                                      exact sums
    AdamW.step                        the recovered update applied to all tensors, moments in 8 bits, clipped
    TokenLogprobs.forward             what the trained model says about single tokens: entropy and alternatives

The data are a Markov chain in which every token has a few likely successors, so the best possible loss is known.

    python examples/train_language_model.py --steps 200
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1903_04488_amd.pipeline import HotPath  # noqa: E402
from paper_1903_04488_amd.training import AdamW, LayerNorm, TokenLogprobs  # noqa: E402


class Chain:
    """tokens whose successor is one of `likely` with probability 0.9"""

    def __init__(self, vocab, likely, device, seed):
        self.gen = torch.Generator(device=device).manual_seed(seed)
        self.vocab, self.device = vocab, device
        self.next = torch.randint(0, vocab, (vocab, likely), device=device, generator=self.gen)
        self.entropy = 0.9 * math.log(likely / 0.9) + 0.1 * math.log(vocab / 0.1)

    def draw(self, n):
        token = torch.randint(0, self.vocab, (n,), device=self.device, generator=self.gen)
        which = torch.randint(0, self.next.shape[1], (n,), device=self.device, generator=self.gen)
        other = torch.randint(0, self.vocab, (n,), device=self.device, generator=self.gen)
        chance = torch.rand(n, device=self.device, generator=self.gen)
        return token, torch.where(chance < 0.9, self.next[token, which], other)


class Model:
    """hidden = layer_norm(table[token] @ mix), logits = hidden @ head^T; parameters and gradients are views of flat vectors"""

    def __init__(self, vocab, width, rows, workers, device, seed):
        gen = torch.Generator(device=device).manual_seed(seed)
        shapes = {"table": (vocab, width), "mix": (width, width), "weight": (width,), "bias": (width,), "head": (vocab, width)}
        self.d = sum(math.prod(s) for s in shapes.values())
        flat = torch.zeros(self.d, device=device)
        self.params = self.views(flat, shapes)
        for name in ("table", "mix", "head"):
            self.params[name].normal_(0.0, width ** -0.5, generator=gen)
        self.params["weight"].fill_(1.0)
        # every worker's gradient, and the update that is recovered from their sketches
        self.worker_grads = [torch.zeros(self.d, device=device) for _ in range(workers)]
        self.worker_views = [self.views(g, shapes) for g in self.worker_grads]
        self.update = torch.zeros(self.d, device=device)
        self.update_views = self.views(self.update, shapes)
        p = self.params
        self.norms = [LayerNorm(p["weight"], p["bias"], rows, dweight=g["weight"], dbias=g["bias"]) for g in self.worker_views]
        self.loss = TokenLogprobs(rows, vocab, device=device)
        self.coefficient = torch.full((rows,), -1.0 / rows, device=device)

    @staticmethod
    def views(flat, shapes):
        parts = flat.split([math.prod(s) for s in shapes.values()])
        return {name: part.view(shape) for (name, shape), part in zip(shapes.items(), parts)}

    def hidden(self, token, worker=0):
        p = self.params
        rows = p["table"][token]
        return rows, self.norms[worker].forward(rows @ p["mix"])

    def gradients(self, worker, token, target):
        """fills the worker's flat gradient; -log probabilities of its targets"""
        p, g = self.params, self.worker_views[worker]
        rows, hidden = self.hidden(token, worker)
        logits = hidden @ p["head"].t()
        logp, dlogits = self.loss.loss(logits, target, self.coefficient, out=logits)
        torch.mm(dlogits.t(), hidden, out=g["head"])
        dmixed = self.norms[worker].backward(dlogits @ p["head"])
        torch.mm(rows.t(), dmixed, out=g["mix"])
        g["table"].zero_().index_add_(0, token, dmixed @ p["mix"].t())
        return -logp


def train(steps=200, vocab=2000, width=64, rows=1024, workers=4, columns=1 << 14, k=4000, P=4, lr=2e-2, seed=1, device="cuda:0",
          tell=None):
    """(mean loss of every step, the data's entropy, the model, the chain)"""
    chain = Chain(vocab, 4, device, seed)
    model = Model(vocab, width, rows, workers, device, seed + 1)
    path = HotPath(model.d, workers, 5, columns, k, seed=190304488, device=device, P=P)
    names = list(model.params)
    opt = AdamW([model.params[n] for n in names], [model.update_views[n] for n in names], lr=lr, betas=(0.9, 0.98),
                weight_decay=0.0, max_norm=1.0, bits=8)
    losses = []
    for step in range(steps):
        loss = [model.gradients(w, *chain.draw(rows)).mean() for w in range(workers)]
        idx, x = path.step(model.worker_grads)
        model.update.zero_().index_copy_(0, idx, x)
        opt.step()
        losses.append(torch.stack(loss).mean())
        if tell and step % 20 == 19:
            tell(f"step {step + 1}: loss {float(losses[-1]):.3f}, norm of the update {float(opt.norm):.3f}")
    return torch.stack(losses), chain.entropy, model, chain


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--top", type=int, default=5)
    a = ap.parse_args()
    losses, entropy, model, chain = train(a.steps, tell=print)
    print(f"loss {float(losses[0]):.3f} -> {float(losses[-10:].mean()):.3f}; the data's entropy is {entropy:.3f}")
    says = TokenLogprobs(1, chain.vocab, top=a.top)
    for token in (0, 1):
        token = torch.tensor([token], device=model.update.device)
        _, hidden = model.hidden(token)
        says.forward(hidden @ model.params["head"].t(), token)
        print(f"after {int(token)} (entropy {float(says.entropy):.2f}; likely {sorted(chain.next[token][0].tolist())}): "
              + ", ".join(f"{int(i)} {math.exp(float(p)):.2f}" for i, p in zip(says.top_idx[0], says.top_logp[0])))


if __name__ == "__main__":
    main()
