"""Types, sizes and sums of the layer operators that their own tests leave out."""
import math

import pytest

import layers_ref as ref
from helpers import ensure_built
from test_gpu_adamw import BLOCK, HYPER, SIZES, check_8bit, pow2, tensors

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    ensure_built()
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2606_06510_gb300 as oz
    yield oz, torch
    torch.cuda.synchronize()
    assert oz.oz2_check_device_status() == 0


TYPES = [("bf16", "f32"), ("f16", "f16"), ("f16", "f32")]


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("param, grad", TYPES)
def test_8_bit_states_of_other_types(env, param, grad, offset):
    oz, torch = env
    types = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
    check_8bit(oz, torch, SIZES, types[param], types[grad], seed=15, steps=3, offset=offset, master=True)


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("param, grad", TYPES)
def test_weights_without_masters(env, param, grad, bits, offset):
    """One step from the same values is the step of a master, rounded: the same bits of
    the weights and of the states."""
    oz, torch = env
    types = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
    out = []
    for master in (False, True):
        p, g, _, _ = tensors(torch, SIZES, types[param], types[grad], 16, offset)
        st = oz.oz2_adamw_states(p, bits=bits)
        plan = oz.oz2_adamw_plan(p, g, masters=[t.float() for t in p] if master else None, **st)
        oz.oz2_adamw(plan, step=1, seed=8, **HYPER)
        out.append(p + [t for name in sorted(st) for t in st[name]])
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(*out))


def test_rounding_of_both_states_is_unbiased(env):
    """The mean over seeds of m and of √v is the unrounded one: within 5 deviations of a
    mean of N values that are each off by up to a spacing s (variance ≤ s²/4), and the
    2^-16 that a draw of 16 bits resolves."""
    oz, torch = env
    e, seeds = BLOCK, 400
    g = torch.randn(e, device="cuda", generator=torch.Generator(device="cuda").manual_seed(17)) * 0.02
    total = {s: torch.zeros(e, dtype=torch.float64, device="cuda") for s in "mv"}
    for seed in range(seeds):
        p = [torch.zeros(e, device="cuda")]
        st = oz.oz2_adamw_states(p, bits=8)
        oz.oz2_adamw(oz.oz2_adamw_plan(p, [g], **st), step=1, seed=seed, **HYPER)
        for s in "mv":
            total[s] += st[s][0].double() * st[s + "_scales"][0].double()
    want = {"m": (1 - HYPER["beta1"]) * g.double(), "v": math.sqrt(1 - HYPER["beta2"]) * g.double().abs()}
    for s in "mv":
        scale = st[s + "_scales"][0].double()
        spacing = pow2(torch, torch.frexp((want[s].abs() / scale).clamp_min(2.0 ** -6))[1] - 4) * scale
        dev = spacing / 2 / math.sqrt(seeds)
        assert ((total[s] / seeds - want[s]).abs() <= 5 * dev + spacing * 2.0 ** -15).all(), s


@pytest.mark.parametrize("m, n, k", [(700, 2304, 2304), (300, 4096, 2500), (40, 5000, 3001)])
def test_accumulation_over_many_tiles(env, m, n, k):
    """dw of more tiles than run at once, stored and added to in float32."""
    oz, torch = env
    g = torch.Generator(device="cuda").manual_seed(m)
    dy, x, w = (torch.randn(s, generator=g, device="cuda").to(torch.bfloat16) for s in ((m, n), (m, k), (n, k)))
    want, (_, _, bb), ew = ref.grad(dy, x, w, None, "none")
    plain = oz.oz2_linear_grad(dy, x, w, dw_dtype=torch.float32, need=("dw",))[1]
    ref.close(plain, want[1], ew + 2.0 ** -23 * want[1].abs(), "dw")
    held = torch.full((n, k + 4), 5.0, device="cuda")
    dw, db = held[:, 1:1 + k], torch.full((n,), 1.0, device="cuda")
    oz.oz2_linear_grad(dy, x, w, dw=dw, db=db, accumulate=True)
    ref.close(dw, want[1] + 5, ew + 2.0 ** -23 * (want[1].abs() + 5), "dw added to")
    ref.close(db, want[2] + 1, bb + 2.0 ** -23 * (want[2].abs() + 1), "db added to")
    assert (held[:, 0] == 5).all() and (held[:, 1 + k:] == 5).all()
