"""Train a two-layer perceptron with the library's layer operators, then serve it.

  python examples/train_mlp.py [--steps 200] [--bits 8]

A step is what a training program does with them: oz2_linear forward (the hidden
layer keeps its z), oz2_linear_grad backward (gradients of the weights added up in
float32 over micro-batches), and one oz2_adamw over all parameters, whose bf16
copies the next forward pass reads.  Serving runs the trained network on single
tokens, in bf16 and with its weights in E4M3.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_06510_gb300 as oz  # noqa: E402


class Mlp:
    """y = x + w2·gelu(w1·x + b1) + b2, parameters in bf16 with float32 masters."""

    def __init__(self, width: int, hidden: int, bits: int, seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.master = [torch.randn(hidden, width, generator=g, device="cuda") * width ** -0.5,
                       torch.zeros(hidden, device="cuda"),
                       torch.randn(width, hidden, generator=g, device="cuda") * hidden ** -0.5 * 0.1,
                       torch.zeros(width, device="cuda")]
        self.param = [t.to(torch.bfloat16) for t in self.master]
        self.grad = [torch.zeros_like(t) for t in self.master]  # float32: added up over micro-batches
        self.states = oz.oz2_adamw_states(self.param, bits=bits)
        self.plan = oz.oz2_adamw_plan(self.param, self.grad, masters=self.master,
                                      decay_scales=[1.0, 0.0, 1.0, 0.0], **self.states)
        self.steps = 0

    def forward(self, x):
        w1, b1, w2, b2 = self.param
        h, z = oz.oz2_linear(x, w1, bias=b1, act="gelu", save_pre=True)
        return oz.oz2_linear(h, w2, bias=b2, residual=x), (x, h, z)

    def backward(self, dy, kept):
        x, h, z = kept
        g1, gb1, g2, gb2 = self.grad
        dh, _, _ = oz.oz2_linear_grad(dy, h, self.param[2], dw=g2, db=gb2, accumulate=True)
        dx, _, _ = oz.oz2_linear_grad(dh, x, self.param[0], pre=z, act="gelu", dw=g1, db=gb1, accumulate=True)
        return dx + dy  # the residual's share

    def update(self, lr):
        self.steps += 1
        oz.oz2_adamw(self.plan, step=self.steps, lr=lr, weight_decay=0.01, seed=self.steps)
        for t in self.grad:
            t.zero_()


def e4m3(w):
    """A weight's rows as E4M3 values and their scales."""
    scale = w.float().abs().amax(dim=1).clamp_min(1e-12) / 448
    return (w.float() / scale[:, None]).to(torch.float8_e4m3fn), scale


def serve(net, x, quantized):
    """The network's output for one token at a time."""
    w1, b1, w2, b2 = net.param
    out = []
    if quantized:
        (q1, s1), (q2, s2) = e4m3(w1), e4m3(w2)
    for t in x.split(1):
        if quantized:
            xq, xs = e4m3(t)
            h = oz.oz2_linear(xq, q1, bias=b1, act="gelu", x_scale=xs, w_scale=s1)
            hq, hs = e4m3(h)
            out.append(oz.oz2_linear(hq, q2, bias=b2, residual=t, x_scale=hs, w_scale=s2))
        else:
            h = oz.oz2_linear(t, w1, bias=b1, act="gelu")
            out.append(oz.oz2_linear(h, w2, bias=b2, residual=t))
    return torch.cat(out)


def train(steps=200, bits=8, width=256, hidden=1024, tokens=2048, micro=2, lr=2e-3, report=None):
    """Fit a fixed random map of the tokens; returns (net, losses)."""
    g = torch.Generator(device="cuda").manual_seed(1)
    target = torch.randn(width, width, generator=g, device="cuda") * width ** -0.5
    net, losses = Mlp(width, hidden, bits), []
    for step in range(steps):
        loss = torch.zeros((), device="cuda")
        for _ in range(micro):
            x = torch.randn(tokens // micro, width, generator=g, device="cuda").to(torch.bfloat16)
            want = torch.tanh(x.float() @ target) + x.float()
            y, kept = net.forward(x)
            diff = y.float() - want
            loss += diff.square().mean() / micro
            net.backward((diff * (2 / (tokens * width) * 64)).to(torch.bfloat16), kept)
        net.update(lr)
        losses.append(loss)
        if report and (step % report == 0 or step == steps - 1):
            print(f"step {step:4d}  loss {loss.item():.4f}")
    return net, torch.stack(losses)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--bits", type=int, default=8, choices=(8, 32))
    a = ap.parse_args()
    net, _ = train(a.steps, a.bits, report=20)
    x = torch.randn(4, net.param[0].shape[1], device="cuda").to(torch.bfloat16)
    whole, _ = net.forward(x)
    for name, q in (("bf16", False), ("E4M3", True)):
        y = serve(net, x, q)
        print(f"served singly in {name}: {((y - whole).float().norm() / whole.float().norm()).item():.1e} "
              "from the batch's output")
    torch.cuda.synchronize()
    assert oz.oz2_check_device_status() == 0


if __name__ == "__main__":
    main()
