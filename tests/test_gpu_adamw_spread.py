"""8-bit AdamW states where a block's gradients span many decades: the steps beside
those of 32-bit states."""
import math

import pytest

from helpers import ensure_built

pytestmark = pytest.mark.gpu

BLOCK = 256
H = dict(lr=1.0, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0)
# AdamW's own step is at most this many lr for any gradients (Cauchy and Schwarz over
# the two sums, without bias corrections, which only lower it after the first steps).
MOST = (1 - H["beta1"]) / math.sqrt(1 - H["beta2"]) / math.sqrt(1 - H["beta1"] ** 2 / H["beta2"])


@pytest.fixture(scope="module")
def env():
    ensure_built()
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2606_06510_gb300 as oz
    yield oz, torch
    torch.cuda.synchronize()


def steps(oz, torch, small, kind, bits, count=400, n=8 * BLOCK):
    """(largest step, root mean square) of the small elements, in lr: a weight of zero
    before each step is minus the step after it."""
    g = torch.Generator(device="cuda").manual_seed(11)
    p, grad = [torch.zeros(n, device="cuda")], [torch.zeros(n, device="cuda")]
    plan = oz.oz2_adamw_plan(p, grad, **oz.oz2_adamw_states(p, bits=bits))
    size = torch.full((n,), small, device="cuda")
    size[::BLOCK] = 1.0
    top, square = 0.0, 0.0
    for t in range(1, count + 1):
        r = torch.randn(n, generator=g, device="cuda")
        grad[0].copy_((r if kind == "random" else 1 + 0.1 * r) * size)
        p[0].zero_()
        oz.oz2_adamw(plan, step=t, seed=5, **H)
        u = p[0][size < 1].double()
        top, square = max(top, u.abs().max().item()), square + u.square().mean().item() / count
    return top, math.sqrt(square)


@pytest.mark.parametrize("kind", ["steady", "random"])
@pytest.mark.parametrize("small", [1e-3, 1e-4, 1e-5, 3e-6, 1e-6, 1e-8])
def test_steps_stay_those_of_adamw(env, small, kind):
    """One gradient of a block at 1, the others small.  An m and a √v that are rounded
    can be up to twice as far apart as unrounded ones (√v from just under two of its
    smallest units to one), so a step is at most 2·MOST = 14.5 lr.  Down to 1e-4 the
    states hold every element to 1/8 of itself or better, and the steps' mean square is
    that of 32-bit states within what two such errors make of it."""
    oz, torch = env
    top, rms = steps(oz, torch, small, kind, 8)
    top32, rms32 = steps(oz, torch, small, kind, 32)
    assert top32 <= MOST
    assert top <= 2 * MOST, (top, top32)
    if small >= 1e-4:
        assert abs(rms / rms32 - 1) <= 0.25, (rms, rms32)


@pytest.mark.parametrize("offset", [0, 1])
def test_without_a_root_there_is_no_m(env, offset):
    """Codes of every kind: a step is that of the state with m's code cleared where √v's
    is zero, bit for bit (weights, codes and scales)."""
    oz, torch = env
    n = 2 * BLOCK + 77
    g = torch.Generator(device="cuda").manual_seed(12)
    codes = [torch.randint(0, 256, (n,), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2)]
    codes[1] &= 0x7F
    codes[1][torch.rand(n, generator=g, device="cuda") < 0.4] = 0
    codes[1][5:60:7] = 0x80  # -0
    for c in codes:
        c[(c & 0x7F) == 0x7F] -= 1  # finite
    grad = torch.randn(n, generator=g, device="cuda") * 1e-3
    out = []
    for clear in (False, True):
        m, v = codes[0].clone(), codes[1].clone()
        if clear:
            m[(v & 0x7F) == 0] = 0
        hold = [torch.empty(n + offset, dtype=torch.uint8, device="cuda")[offset:] for _ in range(2)]
        hold[0].copy_(m)
        hold[1].copy_(v)
        p = torch.ones(n, device="cuda")
        blocks = (n + BLOCK - 1) // BLOCK
        scales = [torch.full((blocks,), 2.0 ** -10, device="cuda") for _ in range(2)]
        plan = oz.oz2_adamw_plan([p], [grad], *([h.view(torch.float8_e4m3fn)] for h in hold), m_scales=scales[:1],
                                 v_scales=scales[1:])
        oz.oz2_adamw(plan, step=3, lr=1e-2, seed=9)
        out.append((p, *hold, *scales))
    assert int(((codes[1] & 0x7F) == 0).sum()) > 100
    assert all(torch.equal(a, b) for a, b in zip(*out))
