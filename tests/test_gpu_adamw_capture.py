"""A captured AdamW step, replayed, is that step again."""
import pytest

from helpers import ensure_built

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
def test_a_replay_is_the_same_step_again(bits):
    """Each replay gives the bits of a call with the step and seed that were captured; the
    gradients and their factor are those of the replay."""
    ensure_built()
    import torch
    import paper_2606_06510_gb300 as oz

    def start():
        g = torch.Generator(device="cuda").manual_seed(21)
        p = [torch.randn(e, generator=g, device="cuda") for e in (1000, 33)]
        grads = [torch.randn(e, generator=g, device="cuda") for e in (1000, 33)]
        states = oz.oz2_adamw_states(p, bits=bits)
        return p, grads, states, oz.oz2_adamw_plan(p, grads, **states), torch.ones((), device="cuda")

    def change(grads, factor, i):
        for t in grads:
            t.mul_(-0.5)
        factor.fill_(1 + i)

    call = dict(step=4, lr=1e-2, seed=7)
    p, grads, states, plan, factor = start()
    for i in range(3):
        change(grads, factor, i)
        oz.oz2_adamw(plan, grad_scale=factor, **call)
    want = p + states["m"] + states["v"]
    p, grads, states, plan, factor = start()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        oz.oz2_adamw(plan, grad_scale=factor, **call)
    for i in range(3):
        change(grads, factor, i)
        graph.replay()
    torch.cuda.synchronize()
    got = p + states["m"] + states["v"]
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, want))
