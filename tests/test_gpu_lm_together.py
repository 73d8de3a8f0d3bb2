"""The operators at a language model's ends together with the layers' between them, as
examples/train_lm.py uses them."""
import importlib.util
import os

import pytest

from helpers import ROOT, ensure_built

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    ensure_built()
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    spec = importlib.util.spec_from_file_location("train_lm", os.path.join(ROOT, "examples", "train_lm.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod, torch


@pytest.mark.parametrize("teacher", [False, True])
def test_it_runs_and_repeats(example, teacher):
    mod, torch = example
    net, losses = mod.train(steps=5, teacher=teacher, vocabulary=333, width=72, hidden=200, tokens=700)
    assert torch.isfinite(losses).all()
    again, _ = mod.train(steps=5, teacher=teacher, vocabulary=333, width=72, hidden=200, tokens=700)
    assert all(torch.equal(a, b) for a, b in zip(net.master + net.param, again.master + again.param))


def reference(torch, net, tokens, loss_of):
    """The gradients of a step by autograd in 64 bits on the same bf16 weights."""
    p = [t.double().requires_grad_() for t in net.param]
    h = p[0][tokens] * net.width ** 0.5
    F = torch.nn.functional
    for layer in range(net.layers):
        gain, shift, w1, b1, w2, b2 = p[1 + 6 * layer:7 + 6 * layer]
        n = F.layer_norm(h, (net.width,), gain, shift, 1e-5)
        h = h + F.gelu(n @ w1.t() + b1) @ w2.t() + b2
    y = F.layer_norm(h, (net.width,), p[-2], p[-1], 1e-5)
    loss = loss_of(y @ p[0].t())
    loss.backward()
    return loss.detach(), [t.grad for t in p]


# bf16 activations and gradients carry 2^-8 of rounding each: the longest way to a weight has some
# sixteen of them in a row (nine activations, dz, and six gradients between the layers), which in the
# 2-norm add up as independent ones, 4·2^-8, and as aligned ones no further than 16·2^-8.
def near(a, b):
    return ((a.double() - b).norm() / b.norm()).item() < 16 * 2.0 ** -8


@pytest.mark.parametrize("tokens", [1, 300])
def test_a_step_against_64_bits(example, tokens):
    mod, torch = example
    net = mod.Lm(515, 64, 192)
    g = torch.Generator(device="cuda").manual_seed(3)
    first, follow = mod.text(g, tokens, 515)
    if tokens > 1:
        first[::9], follow[::5] = first[0].clone(), -100
    zl = 1e-2

    def loss_of(z):
        lse = torch.logsumexp(z, 1)
        there = follow >= 0
        loss = lse - z.gather(1, follow.clamp_min(0)[:, None])[:, 0] + zl * lse * lse
        return (loss * there).sum() / there.sum()

    want, grads = reference(torch, net, first, loss_of)
    got = net.step(first, follow, z_loss=zl)
    assert near(got[None], want[None])
    for a, b in zip(net.grad, grads):
        assert near(a, b)


def test_distillation_against_64_bits(example):
    mod, torch = example
    net = mod.Lm(515, 64, 192)
    g = torch.Generator(device="cuda").manual_seed(4)
    first, _ = mod.text(g, 300, 515)
    ids = torch.rand(300, 515, generator=g, device="cuda").topk(9, dim=1)[1]
    ids[torch.rand(ids.shape, generator=g, device="cuda") < 0.3] = -1
    ids[::11] = -1
    teacher = 2 * torch.randn(ids.shape, generator=g, device="cuda")

    def loss_of(z):
        there = ids >= 0
        q = torch.nan_to_num(torch.softmax((teacher.double() / 2).masked_fill(~there, -float("inf")), 1))
        log_p = torch.log_softmax(z / 2, 1).gather(1, ids.clamp_min(0))
        return (torch.xlogy(q, q) - q * log_p).sum() / there.any(1).sum()

    want, grads = reference(torch, net, first, loss_of)
    got = net.learn_from(first, ids, teacher)
    assert near(got[None], want[None])
    for a, b in zip(net.grad, grads):
        assert near(a, b)


def test_a_captured_step(example):
    """A whole step's gradients captured into a graph beside an eager one of the same model, and
    replayed on other tokens."""
    mod, torch = example
    net, other = mod.Lm(515, 64, 192), mod.Lm(515, 64, 192)
    g = torch.Generator(device="cuda").manual_seed(5)
    batches = [mod.text(g, 300, 515) for _ in range(3)]
    first, follow = (t.clone() for t in batches[0])
    net.step(first, follow)
    for t in net.grad:
        t.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = net.step(first, follow)
    for a, b in batches:
        first.copy_(a)
        follow.copy_(b)
        for t in net.grad + other.grad:
            t.zero_()
        graph.replay()
        want = other.step(a, b)
        assert torch.equal(loss, want)
        assert all(torch.equal(u, v) for u, v in zip(net.grad, other.grad))
