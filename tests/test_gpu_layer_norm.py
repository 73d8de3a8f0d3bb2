"""oz2_layer_norm and its gradient against their formulas in 64 bits."""
import pytest
import torch

import lm_ref as ref
from helpers import ensure_built
from layers_ref import close

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]


@pytest.fixture(scope="module")
def oz():
    ensure_built()
    import paper_2606_06510_gb300 as oz
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    return oz


def rng(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def view(t, how):
    if how == "whole":
        return t
    pad = torch.full((t.shape[0], t.shape[1] + (3 if how == "odd" else 8)), float("nan"), dtype=t.dtype, device="cuda")
    at = 1 if how == "odd" else 0
    pad[:, at:at + t.shape[1]] = t
    return pad[:, at:at + t.shape[1]]


# Every number of threads and pieces a row has, with rows that end inside a piece.
SHAPES = [(1, 1), (1, 16), (3, 7), (7, 64), (5, 250), (9, 512), (40, 777), (65, 1024), (33, 1031), (130, 2048), (4, 4000),
          (64, 4096), (3, 8192), (2, 12345), (2, 16384), (3, 16392), (2, 20001), (400, 100), (700, 1000), (400, 2056),
          (330, 4104), (320, 9000), (310, 16384), (309, 17000), (5000, 40),
          (1001, 64), (1001, 63), (1003, 128), (2005, 24), (777, 33), (1500, 5), (333, 9001), (200, 16383)]


def inputs(m, k, dt, how, affine, center, seed):
    g = rng(seed)
    x = view((torch.randn(m, k, generator=g, device="cuda") * 1.5 + torch.randn(m, 1, generator=g, device="cuda")).to(dt), how)
    wt = (dt, torch.float32)[affine - 1] if affine else dt
    w = (1 + 0.3 * torch.randn(k, generator=g, device="cuda")).to(wt) if affine else None
    b = torch.randn(k, generator=g, device="cuda").to(wt) if affine and center else None
    return g, x, w, b


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("at", range(len(SHAPES)))
@pytest.mark.parametrize("center", [True, False])
def test_both_ways(oz, dt, at, center):
    m, k = SHAPES[at]
    how, affine = ("whole", "odd", "strided")[at % 3], (at + center) % 3
    g, x, w, b = inputs(m, k, dt, how, affine, center, m + k)
    if k == 1:
        w = b = None
    (y, mean, rstd), (ey, em, er) = ref.layer_norm(x, w, b, 1e-5, center)
    gy, gm, gr = oz.oz2_layer_norm(x, w, b, eps=1e-5, center=center, save_stats=True)
    close(gy, y, ey, "y")
    close(gr, rstd, er, "rstd")
    assert (gm is None) == (not center)
    if center:
        close(gm, mean, em, "mean")
    assert torch.equal(gy, oz.oz2_layer_norm(x, w, b, center=center))
    # The gradient, from these statistics.
    dy = view(torch.randn(m, k, generator=g, device="cuda").to(dt), how)
    r = view(torch.randn(m, k, generator=g, device="cuda").to(dt), how) if at % 2 else None
    want, bound = ref.layer_norm_grad(dy, x, gm, gr, w, r)
    got = oz.oz2_layer_norm_grad(dy, x, gm, gr, w, residual=r)
    for a, v, e, what in zip(got, want, bound, ("dx", "dweight", "dbias")):
        close(a, v, e, what)
    again = oz.oz2_layer_norm_grad(dy, x, gm, gr, w, residual=r)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("need", [("dx",), ("dweight",), ("dbias",), ("dx", "dbias"), ("dweight", "dbias"), ()])
@pytest.mark.parametrize("k", [96, 3000, 17000])
def test_what_is_wanted(oz, need, k):
    g, x, w, _ = inputs(50, k, torch.bfloat16, "whole", 1, True, k)
    _, mean, rstd = oz.oz2_layer_norm(x, w, save_stats=True)
    dy = torch.randn(50, k, generator=g, device="cuda").bfloat16()
    whole = oz.oz2_layer_norm_grad(dy, x, mean, rstd, w)
    got = oz.oz2_layer_norm_grad(dy, x, mean, rstd, w, need=need)
    for a, b, name in zip(got, whole, ("dx", "dweight", "dbias")):
        assert torch.equal(a, b) if name in need else a is None


def test_accumulate_and_given_outputs(oz):
    g, x, w, _ = inputs(300, 520, torch.float16, "whole", 2, True, 3)
    _, mean, rstd = oz.oz2_layer_norm(x, w, save_stats=True)
    dy = torch.randn(300, 520, generator=g, device="cuda").half()
    want = oz.oz2_layer_norm_grad(dy, x, mean, rstd, w)
    dw, db = torch.randn(520, generator=g, device="cuda"), torch.randn(520, generator=g, device="cuda")
    sums = dw + want[1], db + want[2]
    dx = torch.full((302, 528), 9.0, device="cuda").half()
    got = oz.oz2_layer_norm_grad(dy, x, mean, rstd, w, dx=dx[1:301, :520], dweight=dw, dbias=db, accumulate=True)
    assert torch.equal(got[0], want[0]) and torch.equal(dw, sums[0]) and torch.equal(db, sums[1])
    dx[1:301, :520] = 9
    assert (dx == 9).all()  # what lies beside it is left as it was
    with pytest.raises(AssertionError, match="accumulate"):
        oz.oz2_layer_norm_grad(dy, x, mean, rstd, w, accumulate=True)


@pytest.mark.parametrize("k", [520, 4096, 20000])
def test_in_place(oz, k):
    """y over x, and dx over the skip connection's gradient."""
    g, x, w, b = inputs(70, k, torch.bfloat16, "whole", 1, True, 5)
    y, mean, rstd = oz.oz2_layer_norm(x, w, b, save_stats=True)
    own = x.clone()
    assert oz.oz2_layer_norm(own, w, b, out=own) is own and torch.equal(own, y)
    dy, r = (torch.randn(70, k, generator=g, device="cuda").bfloat16() for _ in range(2))
    want = oz.oz2_layer_norm_grad(dy, x, mean, rstd, w, residual=r)
    got = oz.oz2_layer_norm_grad(dy, x, mean, rstd, w, residual=r, dx=r)
    assert got[0] is r and torch.equal(r, want[0]) and torch.equal(got[1], want[1])


def test_hard_rows(oz):
    """Constant rows, a mean far above the spread, large and infinite values, NaN."""
    x = torch.zeros(8, 512, device="cuda")
    x[1] = 3.0
    x[2] = 1000 + torch.randn(512, generator=rng(1), device="cuda")
    x[3] = 1e15 * torch.randn(512, generator=rng(2), device="cuda")
    x[4] = 1e-15 * torch.randn(512, generator=rng(3), device="cuda")
    (y, mean, rstd), (ey, em, er) = ref.layer_norm(x[:5], None, None, 1e-5, True)
    gy, gm, gr = oz.oz2_layer_norm(x, save_stats=True)
    close(gy[:5], y, ey, "y")
    close(gr[:5], rstd, er, "rstd")
    x[5, 7], x[6, 9] = float("inf"), float("nan")
    y = oz.oz2_layer_norm(x)
    assert y[5:7].isnan().any(1).all() and torch.equal(y[[0, 1, 2, 3, 4, 7]], gy[[0, 1, 2, 3, 4, 7]])


@pytest.mark.parametrize("m", [3, 8, 700])
@pytest.mark.parametrize("k", [1, 2, 16, 128])
def test_constant_rows_of_large_values(oz, m, k):
    """mean·rstd passes FP32's range, but no row deviates from its mean (exact: k is a power of two,
    and equal values are added): dx = rstd·(dy - mean dy), dw = 0."""
    x = torch.full((m, k), 2.0 ** 120, device="cuda")
    y, mean, rstd = oz.oz2_layer_norm(x, save_stats=True)
    assert not y.any() and torch.equal(mean, x[:, 0])
    dy = torch.randn(m, k, generator=rng(k), device="cuda")
    dx, dw, db = oz.oz2_layer_norm_grad(dy, x, mean, rstd)
    dev, r = dy.double() - dy.double().mean(1, keepdim=True), rstd.double()[:, None]
    # The mean of k, its product and difference: k + 3 roundings of what is no larger than Σ|dy|/k + |dy|.
    close(dx, r * dev, r * (k + 3) * ref.u * (dy.double().abs() + dy.double().abs().mean(1, keepdim=True)), "dx")
    assert not dw.any()
    close(db, dy.double().sum(0), m * ref.u * dy.double().abs().sum(0), "db")


def test_empty(oz):
    x = torch.zeros(0, 8, device="cuda")
    y, mean, rstd = oz.oz2_layer_norm(x, save_stats=True)
    assert y.shape == (0, 8) and mean.shape == rstd.shape == (0,)
    dx, dw, db = oz.oz2_layer_norm_grad(x, x, mean, rstd)
    assert dx.shape == (0, 8) and not dw.any() and not db.any()
    old = torch.ones(8, device="cuda")
    oz.oz2_layer_norm_grad(x, x, mean, rstd, need=("dweight",), dweight=old, accumulate=True)
    assert (old == 1).all()
    assert oz.oz2_layer_norm(torch.zeros(3, 0, device="cuda")).shape == (3, 0)


@pytest.mark.parametrize("center", [True, False])
def test_against_differences(oz, center):
    """dL of L = Σ y·c along random directions: differences of h leave h²·|L'''|/6, far below
    1e-3 of these derivatives for h = 2^-7, and FP32 noise of 2^-24·Σ|y·c|/h, some 5e-4."""
    g = rng(8)
    m, k = 6, 40
    x, w, b, c = (torch.randn(s, generator=g, device="cuda") for s in ((m, k), (k,), (k,), (m, k)))
    loss = lambda x, w, b: (oz.oz2_layer_norm(x, w, b, center=center).double() * c.double()).sum()  # noqa: E731
    _, mean, rstd = oz.oz2_layer_norm(x, w, b, center=center, save_stats=True)
    dx, dw, db = oz.oz2_layer_norm_grad(c, x, mean, rstd, w)
    h = 2.0 ** -7
    for _ in range(4):
        v = [torch.randn(t.shape, generator=g, device="cuda") for t in (x, w, b)]
        for i, grad in enumerate((dx, dw, db)):
            p = [t + h * v[j] if j == i else t for j, t in enumerate((x, w, b))]
            q = [t - h * v[j] if j == i else t for j, t in enumerate((x, w, b))]
            num = (loss(*p) - loss(*q)) / (2 * h)
            assert abs(num - (grad.double() * v[i].double()).sum()) < 5e-3 * (1 + grad.double().norm() * v[i].double().norm())


def test_streams_and_graphs(oz):
    g, x, w, b = inputs(600, 1000, torch.bfloat16, "whole", 1, True, 6)
    dy = torch.randn(600, 1000, generator=g, device="cuda").bfloat16()
    y, mean, rstd = oz.oz2_layer_norm(x, w, b, save_stats=True)
    want = oz.oz2_layer_norm_grad(dy, x, mean, rstd, w)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [oz.oz2_layer_norm_grad(dy, x, mean, rstd, w, stream=s) for _ in range(4) for s in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for r in got for a, b in zip(r, want))
    graph = torch.cuda.CUDAGraph()
    xs = torch.zeros_like(x)
    with torch.cuda.graph(graph):
        y2, m2, r2 = oz.oz2_layer_norm(xs, w, b, save_stats=True)
        got = oz.oz2_layer_norm_grad(dy, xs, m2, r2, w)
    xs.copy_(x)
    for _ in range(2):
        graph.replay()
        assert torch.equal(y2, y) and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("k", [5, 33, 777, 4097, 8201, 20001])
def test_in_place_off_the_grid(oz, dt, k):
    """y over x where the words around a piece hold others' values, of the same row or of the next:
    rows of their own stride that begin anywhere, and rows without a gap."""
    g, x, w, b = inputs(203, k, dt, "odd", 1, True, 5)
    y, mean, rstd = oz.oz2_layer_norm(x, w, b, save_stats=True)
    for own in (view(x, "odd"), x.contiguous()):
        got, m2, r2 = oz.oz2_layer_norm(own, w, b, out=own, save_stats=True)
        assert got is own and torch.equal(own, y) and torch.equal(m2, mean) and torch.equal(r2, rstd)
    dy, r = (view(torch.randn(203, k, generator=g, device="cuda").to(dt), "odd") for _ in range(2))
    want = oz.oz2_layer_norm_grad(dy, x, mean, rstd, w, residual=r)
    for own in (view(r, "odd"), r.contiguous()):
        got = oz.oz2_layer_norm_grad(dy, x, mean, rstd, w, residual=own, dx=own)
        assert got[0] is own and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("center", [True, False])
def test_statistics_of_no_features(oz, center):
    """They are NaN, not what the memory held before."""
    x = torch.zeros(3, 0, device="cuda")
    for _ in range(4):
        del_me = torch.full((3,), 7.0, device="cuda"), torch.full((3,), 7.0, device="cuda")
        del del_me
        y, mean, rstd = oz.oz2_layer_norm(x, center=center, save_stats=True)
        assert y.shape == (3, 0) and rstd.isnan().all() and (mean.isnan().all() if center else mean is None)
    dx, dw, db = oz.oz2_layer_norm_grad(x, x, mean, rstd)
    assert dx.shape == (3, 0) and dw.shape == db.shape == (0,)
