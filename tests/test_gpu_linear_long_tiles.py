"""A gradient whose dX has fewer tiles than there are CTA pairs, and long ones: they go one to a
pair beside dW's many.  Each tile is whole, so both products have the bits that they have alone."""
import pytest
import torch

from helpers import ensure_built

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def oz():
    ensure_built()
    import paper_2606_06510_gb300 as oz
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    return oz


@pytest.mark.parametrize("m,n,k", [(2500, 30000, 1100), (4096, 20000, 1024), (1111, 32003, 2000), (2049, 9001, 1288)])
def test_together_and_alone(oz, m, n, k):
    g = torch.Generator(device="cuda").manual_seed(m)
    dy = torch.randn(m, n, generator=g, device="cuda").bfloat16()
    x, w = (torch.randn(s, k, generator=g, device="cuda").bfloat16() for s in (m, n))
    dx, dw, _ = oz.oz2_linear_grad(dy, x, w, need=("dx", "dw"))
    assert torch.equal(dx, oz.oz2_linear_grad(dy, x, w, need=("dx",))[0])
    assert torch.equal(dw, oz.oz2_linear_grad(dy, x, w, need=("dw",))[1])
    rows, cols = torch.tensor([0, 255, 256, m - 1]), torch.tensor([0, 255, 256, n // 2, n - 1])
    want = dy[rows].double() @ w.double()
    assert ((dx[rows].double() - want).abs() <= 2.0 ** -8 * want.abs() +
            (n / 16 + 16) * 2.0 ** -22 * (dy[rows].double().abs() @ w.double().abs())).all()
    want = dy[:, cols].double().t() @ x.double()
    assert ((dw[cols].double() - want).abs() <= 2.0 ** -8 * want.abs() +
            (m / 16 + 16) * 2.0 ** -22 * (dy[:, cols].double().abs().t() @ x.double().abs())).all()
    assert oz.oz2_check_device_status() == 0
