"""Train a small language model with the library's operators.

  python examples/train_lm.py [--steps 200] [--teacher]

The model predicts a token from the one before it: a table's rows, layers of a norm and a
perceptron on a skip connection, a last norm, and a head whose weights are the table
(tied).  A step is what a training program does: oz2_embedding, oz2_layer_norm and
oz2_linear forward, oz2_linear_xent for the loss without its logits, then the gradients
from the loss back, the head's and the table's added up in one float32 gradient, and one
oz2_adamw over all parameters.  With --teacher the model learns from another's top logits
(oz2_linear_distill) in place of the tokens.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_06510_gb300 as oz  # noqa: E402


class Lm:
    """`layers` blocks h + w2·gelu(w1·norm(h) + b1) + b2 between a table and its transpose;
    parameters in bf16 with float32 masters."""

    def __init__(self, vocabulary: int, width: int, hidden: int, layers: int = 2, seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, std):
            return torch.randn(shape, generator=g, device="cuda") * std

        self.vocabulary, self.width, self.layers, self.steps = vocabulary, width, layers, 0
        self.master = [normal(vocabulary, width, std=0.05)]
        decay = [1.0]
        for _ in range(layers):
            self.master += [torch.ones(width, device="cuda"), torch.zeros(width, device="cuda"),
                            normal(hidden, width, std=width ** -0.5), torch.zeros(hidden, device="cuda"),
                            normal(width, hidden, std=hidden ** -0.5 * 0.2), torch.zeros(width, device="cuda")]
            decay += [0.0, 0.0, 1.0, 0.0, 1.0, 0.0]
        self.master += [torch.ones(width, device="cuda"), torch.zeros(width, device="cuda")]
        decay += [0.0, 0.0]
        self.param = [t.to(torch.bfloat16) for t in self.master]
        self.grad = [torch.zeros_like(t) for t in self.master]
        self.plan = oz.oz2_adamw_plan(self.param, self.grad, masters=self.master, decay_scales=decay,
                                      **oz.oz2_adamw_states(self.param))

    def forward(self, tokens):
        """The last norm's output, and what the backward pass wants."""
        h, kept = oz.oz2_embedding(tokens, self.param[0], scale=self.width ** 0.5), []
        for layer in range(self.layers):
            gain, shift, w1, b1, w2, b2 = self.param[1 + 6 * layer:7 + 6 * layer]
            n, mean, rstd = oz.oz2_layer_norm(h, gain, shift, save_stats=True)
            a, z = oz.oz2_linear(n, w1, bias=b1, act="gelu", save_pre=True)
            kept.append((h, mean, rstd, n, a, z))
            h = oz.oz2_linear(a, w2, bias=b2, residual=h)
        y, mean, rstd = oz.oz2_layer_norm(h, self.param[-2], self.param[-1], save_stats=True)
        return y, (tokens, kept, h, mean, rstd)

    def backward(self, dy, state):
        """Adds up the gradients of all parameters but the head's share of the table's."""
        tokens, kept, h, mean, rstd = state
        dh, _, _ = oz.oz2_layer_norm_grad(dy, h, mean, rstd, self.param[-2], dweight=self.grad[-2], dbias=self.grad[-1],
                                          accumulate=True)
        for layer in reversed(range(self.layers)):
            gain, _, w1, _, w2, _ = self.param[1 + 6 * layer:7 + 6 * layer]
            g_gain, g_shift, g1, gb1, g2, gb2 = self.grad[1 + 6 * layer:7 + 6 * layer]
            x, mean, rstd, n, a, z = kept[layer]
            da, _, _ = oz.oz2_linear_grad(dh, a, w2, dw=g2, db=gb2, accumulate=True)
            dn, _, _ = oz.oz2_linear_grad(da, n, w1, pre=z, act="gelu", dw=g1, db=gb1, accumulate=True)
            dh, _, _ = oz.oz2_layer_norm_grad(dn, x, mean, rstd, gain, residual=dh, dx=dh, dweight=g_gain, dbias=g_shift,
                                              accumulate=True)
        oz.oz2_embedding_grad(dh, tokens, self.vocabulary, scale=self.width ** 0.5, out=self.grad[0], accumulate=True)

    def step(self, tokens, targets, z_loss=1e-4):
        """The mean loss of the targets that count (not below 0), with its gradients added up."""
        y, state = self.forward(tokens)
        loss, lse, _ = oz.oz2_linear_xent(y, self.param[0], targets, z_loss=z_loss)
        share = 1 / (targets >= 0).sum().clamp_min(1).float()
        dy, _ = oz.oz2_linear_xent_grad(share, y, self.param[0], targets, lse, z_loss=z_loss, dw=self.grad[0], accumulate=True)
        self.backward(dy, state)
        return loss.sum() * share

    def learn_from(self, tokens, ids, teacher, temperature=2.0):
        """The mean distance from a teacher's listed logits, with its gradients added up."""
        y, state = self.forward(tokens)
        loss, lse, _ = oz.oz2_linear_distill(y, self.param[0], ids, teacher, temperature=temperature)
        share = 1 / (ids >= 0).any(dim=1).sum().clamp_min(1).float()
        dy, _ = oz.oz2_linear_distill_grad(share, y, self.param[0], ids, teacher, lse, temperature=temperature,
                                           dw=self.grad[0], accumulate=True)
        self.backward(dy, state)
        return loss.sum() * share

    def update(self, lr):
        self.steps += 1
        oz.oz2_adamw(self.plan, step=self.steps, lr=lr, weight_decay=0.01)
        for t in self.grad:
            t.zero_()


def text(g, tokens, vocabulary):
    """Pairs of neighbours in a made-up language: a token is mostly followed by one of four."""
    first = torch.randint(0, vocabulary, (tokens,), generator=g, device="cuda")
    follow = (first * 7 + 13 * torch.randint(0, 4, (tokens,), generator=g, device="cuda")) % vocabulary
    stray = torch.rand(tokens, generator=g, device="cuda") < 0.1
    return first, torch.where(stray, torch.randint(0, vocabulary, (tokens,), generator=g, device="cuda"), follow)


def train(steps=200, teacher=False, vocabulary=1000, width=128, hidden=512, tokens=4096, lr=2e-3, report=None):
    """(the model, its losses)"""
    g = torch.Generator(device="cuda").manual_seed(1)
    net, losses = Lm(vocabulary, width, hidden), []
    for step in range(steps):
        first, follow = text(g, tokens, vocabulary)
        if teacher:  # of the four followers it is sure alike; a list may have less
            ids = (first[:, None] * 7 + 13 * torch.arange(4, device="cuda")) % vocabulary
            ids = torch.where(torch.rand(ids.shape, generator=g, device="cuda") < 0.1, torch.full_like(ids, -1), ids)
            loss = net.learn_from(first, ids, torch.zeros(ids.shape, device="cuda"))
        else:
            follow = torch.where(torch.rand(tokens, generator=g, device="cuda") < 0.05, torch.full_like(follow, -100), follow)
            loss = net.step(first, follow)
        net.update(lr)
        losses.append(loss)
        if report and (step % report == 0 or step == steps - 1):
            print(f"step {step:4d}  loss {loss.item():.4f}")
    return net, torch.stack(losses)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--teacher", action="store_true")
    a = ap.parse_args()
    train(a.steps, a.teacher, report=20)
    assert oz.oz2_check_device_status() == 0


if __name__ == "__main__":
    main()
