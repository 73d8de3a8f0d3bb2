"""oz2_linear records no graph, and says so where a gradient would be lost."""
import pytest
import torch

from helpers import ensure_built


@pytest.fixture(scope="module")
def oz():
    ensure_built()
    import paper_2606_06510_gb300 as oz
    return oz


WHAT = ("x", "w", "bias", "residual", "x_scale", "w_scale")


def operands(device, what):
    dt = torch.float8_e4m3fn if "scale" in what else torch.bfloat16
    t = {"x": torch.ones(4, 8, device=device).to(dt), "w": torch.ones(6, 8, device=device).to(dt),
         "bias": torch.ones(6, device=device), "residual": torch.ones(4, 6, device=device).bfloat16()}
    if "scale" in what:
        t["x_scale"], t["w_scale"] = torch.ones(4, device=device), torch.ones(6, device=device)
    t[what].requires_grad_()
    return t


@pytest.mark.parametrize("what", WHAT)
def test_a_lost_gradient_is_refused(oz, what):
    """Before anything else of the call is looked at (these are no CUDA tensors)."""
    with pytest.raises(AssertionError, match="requires its gradient"):
        oz.oz2_linear(**operands("cpu", what))
    with torch.no_grad(), pytest.raises(AssertionError, match="CUDA"):
        oz.oz2_linear(**operands("cpu", what))
    with torch.inference_mode(), pytest.raises(AssertionError, match="CUDA"):
        oz.oz2_linear(**operands("cpu", what))


@pytest.mark.gpu
@pytest.mark.parametrize("what", WHAT)
def test_without_a_graph_it_runs(oz, what):
    t = operands("cuda", what)
    with torch.no_grad():
        y = oz.oz2_linear(**t)
    assert not y.requires_grad
    assert torch.equal(y, oz.oz2_linear(**{k: v.detach() for k, v in t.items()}))


@pytest.mark.gpu
def test_the_gradients_of_parameters_are_had(oz):
    """oz2_linear_grad takes them as they are: it is what gives their gradients."""
    x, w = torch.ones(4, 8, device="cuda").bfloat16(), torch.ones(6, 8, device="cuda").bfloat16().requires_grad_()
    dx, dw, db = oz.oz2_linear_grad(torch.ones(4, 6, device="cuda").bfloat16(), x, w)
    assert (dx == 6).all() and (dw == 4).all() and (db == 4).all()
