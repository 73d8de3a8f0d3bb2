"""The layer operators together, as examples/train_mlp.py uses them."""
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
    spec = importlib.util.spec_from_file_location("train_mlp", os.path.join(ROOT, "examples", "train_mlp.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod, torch


@pytest.mark.parametrize("bits", [32, 8])
def test_training_learns_and_repeats(example, bits):
    """The loss falls by 4 (a map of this width takes it further), and a second run
    gives the same weights bit for bit."""
    mod, torch = example
    net, losses = mod.train(steps=60, bits=bits)
    assert torch.isfinite(losses).all()
    assert losses[-5:].mean() < 0.25 * losses[0]
    again, _ = mod.train(steps=60, bits=bits)
    assert all(torch.equal(a, b) for a, b in zip(net.param + net.master, again.param + again.master))


def test_one_step_against_64_bits(example):
    """Gradients and updated weights of a whole step against autograd in 64 bits on
    the same bf16 weights: bf16 activations and dz carry 2^-8 of rounding each, three
    of them in a row at most; the first AdamW step is a sign but for small gradients."""
    mod, torch = example
    width, hidden, tokens = 64, 192, 300
    net = mod.Mlp(width, hidden, 32)
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(tokens, width, generator=g, device="cuda").to(torch.bfloat16)
    dy = torch.randn(tokens, width, generator=g, device="cuda").to(torch.bfloat16)
    leaves = [p.double().requires_grad_() for p in net.param]
    xd = x.double().requires_grad_()
    h = torch.nn.functional.gelu(xd @ leaves[0].t() + leaves[1])
    y = xd + h @ leaves[2].t() + leaves[3]
    y.backward(dy.double())
    got, kept = net.forward(x)
    dx = net.backward(dy, kept)
    near = lambda a, b: ((a.double() - b).norm() / b.norm()).item() < 3 * 2.0 ** -8  # noqa: E731
    assert near(got, y.detach()) and near(dx, xd.grad)
    for a, b in zip(net.grad, leaves):
        assert near(a, b.grad)
    before = [t.clone() for t in net.master]
    grads = [t.clone() for t in net.grad]
    net.update(1e-3)
    for i, (a, b, gr) in enumerate(zip(net.master, before, grads)):
        decay = 0.01 if i % 2 == 0 else 0.0
        want = b.double() - 1e-3 * (decay * b.double() + gr.double() / (gr.double().abs() + 1e-8))
        assert ((a.double() - want).abs() <= 2.0 ** -22 * (b.double().abs() + 4e-3)).all()
        assert torch.equal(net.param[i], a.to(torch.bfloat16)) and not net.grad[i].any()


def test_serving_matches_the_batch(example):
    """Single tokens give the batch's rows: within two bf16 roundings in bf16, and
    within E4M3's 2^-4 of the branch added to the residual with its weights in E4M3."""
    mod, torch = example
    net, _ = mod.train(steps=20, bits=8)
    x = torch.randn(5, 256, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda").to(torch.bfloat16)
    whole, _ = net.forward(x)
    rel = lambda a: ((a - whole).float().norm() / whole.float().norm()).item()  # noqa: E731
    assert rel(mod.serve(net, x, False)) < 2 * 2.0 ** -8
    assert rel(mod.serve(net, x, True)) < 2.0 ** -4
