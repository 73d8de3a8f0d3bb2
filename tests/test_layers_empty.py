"""Empty linear layers do nothing, whichever of their pointers are null: a framework's
empty array, an empty scale among them, has none."""
import pytest
import torch

from helpers import ensure_built


@pytest.fixture(scope="module")
def oz():
    ensure_built()
    import paper_2606_06510_gb300 as oz
    oz.lib()
    return oz


BF16, E4M3, N = 1, 3, None


def linear(oz, m, n, xs, ws, type=E4M3):
    return oz.lib().oz2_linear(m, n, 8, type, 16, 8, 16, 8, xs, ws, N, 0, 0, N, 0, N, 0, 16, 8, BF16, N)


def test_empty_with_scales_is_nothing(oz):
    assert linear(oz, 0, 8, N, 16) == 0  # no tokens: their scales are an empty array
    assert linear(oz, 8, 0, 16, N) == 0
    assert linear(oz, 0, 0, N, N) == 0
    assert linear(oz, 0, 8, 16, 16) == 0


def test_what_is_refused_stays_refused(oz):
    assert linear(oz, 8, 8, N, 16) == -1
    assert linear(oz, 8, 8, 16, N) == -1
    assert linear(oz, 8, 8, 16, 16, BF16) == -1
    assert linear(oz, 0, 8, N, 16, BF16) == -1
    assert linear(oz, 8, 0, 16, N, BF16) == -1


@pytest.mark.gpu
def test_no_tokens_with_scales(oz):
    """Through the binding: a slice without tokens, and weights without outputs."""
    e4m3 = torch.float8_e4m3fn
    x, w = (torch.ones(s, device="cuda").to(e4m3) for s in ((4, 64), (32, 64)))
    xs, ws = torch.ones(4, device="cuda"), torch.ones(32, device="cuda")
    assert oz.oz2_linear(x[:0], w, x_scale=xs[:0], w_scale=ws).shape == (0, 32)
    assert oz.oz2_linear(x, w[:0], x_scale=xs, w_scale=ws[:0]).shape == (4, 0)
    y, z = oz.oz2_linear(x[:0], w, x_scale=xs[:0], w_scale=ws, save_pre=True)
    assert y.shape == z.shape == (0, 32)
