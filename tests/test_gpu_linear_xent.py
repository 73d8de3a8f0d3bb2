"""oz2_linear_xent and its gradient against their formulas in 64 bits."""
import pytest
import torch

import lm_ref as ref
from helpers import ensure_built
from layers_ref import close

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


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
    beside = float("nan") if t.is_floating_point() else 1 << 30
    pad = torch.full((t.shape[0], t.shape[1] + (3 if how == "odd" else 8)), beside, dtype=t.dtype, device="cuda")
    at = 1 if how == "odd" else 0
    pad[:, at:at + t.shape[1]] = t
    return pad[:, at:at + t.shape[1]]


def inputs(m, n, k, dt, how="whole", masked=True, seed=0, ids=torch.int64):
    g = rng(seed + m + n + k)
    w = view((torch.randn(n, k, generator=g, device="cuda") * 2 * max(k, 1) ** -0.5).to(dt), how)
    t = torch.randint(0, n, (m,), generator=g, device="cuda")
    x = (torch.randn(m, k, generator=g, device="cuda") + 3 * torch.rand(m, 1, generator=g, device="cuda") * w[t].float()).to(dt)
    if masked and m > 1:
        t[torch.rand(m, generator=g, device="cuda") < 0.2] = -100
    return g, view(x, how), w, t.to(ids)


# Tokens, rows and depth inside a tile, at its ends, over several; rows off the grid.
SHAPES = [(1, 1, 1, "whole"), (1, 64, 64, "whole"), (2, 65, 8, "whole"), (5, 1000, 100, "whole"), (31, 63, 72, "odd"),
          (128, 256, 64, "whole"), (129, 257, 65, "odd"), (256, 512, 256, "strided"), (257, 513, 96, "whole"),
          (300, 1003, 256, "whole"), (1, 20000, 512, "whole"), (17, 5000, 1031, "odd"), (700, 3001, 128, "strided"),
          (2100, 129, 40, "whole"), (1500, 10007, 64, "whole")]


@pytest.mark.parametrize("dt", [BF16, F16])
@pytest.mark.parametrize("m,n,k,how", SHAPES)
def test_forward(oz, dt, m, n, k, how):
    g, x, w, t = inputs(m, n, k, dt, how, ids=torch.int32 if m % 2 else torch.int64)
    for scale, zl in ((1.0, 0.0), (0.25, 1e-2), (-1.5, 0.0)):
        want, bound = ref.xent(x, w, t, scale, zl)
        got = oz.oz2_linear_xent(x, w, t, scale=scale, z_loss=zl)
        for a, v, e, what in zip(got, want, bound, ("loss", "lse", "picked")):
            close(a, v, e, what)
        assert all(torch.equal(a, b) for a, b in zip(got, oz.oz2_linear_xent(x, w, t, scale=scale, z_loss=zl)))


@pytest.mark.parametrize("dt", [BF16, F16])
@pytest.mark.parametrize("m,n,k,how", SHAPES)
def test_gradient(oz, dt, m, n, k, how):
    g, x, w, t = inputs(m, n, k, dt, how, ids=torch.int32 if m % 2 else torch.int64)
    dloss = torch.rand(m, generator=g, device="cuda") / m
    for scale, zl, wt in ((1.0, 0.0, dt), (0.5, 1e-2, torch.float32)):
        lse = ref.xent(x, w, t, scale, zl)[0][1].float()
        want, bound = ref.xent_grad(dloss, x, w, t, lse, scale, zl, wt)
        got = oz.oz2_linear_xent_grad(dloss, x, w, t, lse, scale=scale, z_loss=zl, dw_dtype=wt)
        for a, v, e, what in zip(got, want, bound, ("dx", "dw")):
            close(a, v, e, what)
        assert got[1].dtype == wt and not got[0][t < 0].any()
        again = oz.oz2_linear_xent_grad(dloss, x, w, t, lse, scale=scale, z_loss=zl, dw_dtype=wt)
        assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_no_depth(oz):
    """k = 0: every logit is 0."""
    x, w = torch.zeros(3, 0, device="cuda").to(BF16), torch.zeros(700, 0, device="cuda").to(BF16)
    t = torch.tensor([5, -1, 699], device="cuda")
    loss, lse, picked = oz.oz2_linear_xent(x, w, t)
    log_n = torch.tensor(700.0).log().item()
    assert ((lse - log_n).abs() < 1e-4).all() and loss[1] == 0 and ((loss - log_n)[[0, 2]].abs() < 1e-4).all()
    assert not picked.any()
    dx, dw = oz.oz2_linear_xent_grad(torch.ones(3, device="cuda"), x, w, t, lse)
    assert dx.shape == (3, 0) and dw.shape == (700, 0)


def test_no_tokens(oz):
    w = torch.randn(90, 64, device="cuda").to(BF16)
    x, t, f = w[:0], torch.zeros(0, dtype=torch.int64, device="cuda"), torch.zeros(0, device="cuda")
    assert all(v.shape == (0,) for v in oz.oz2_linear_xent(x, w, t))
    dx, dw = oz.oz2_linear_xent_grad(f, x, w, t, f)
    assert dx.shape == (0, 64) and dw.shape == (90, 64) and not dw.any()
    old = torch.ones(90, 64, device="cuda")
    oz.oz2_linear_xent_grad(f, x, w, t, f, need=("dw",), dw=old, accumulate=True)
    assert (old == 1).all()


@pytest.mark.parametrize("dt", [BF16, F16])
def test_masked_tokens_hold_anything(oz, dt):
    """Tokens that do not count: no loss, no gradient, whatever x, lse and dloss hold there."""
    g, x, w, t = inputs(600, 900, 128, dt)
    dead = t < 0
    lse = oz.oz2_linear_xent(x, w, t)[1]
    dloss = torch.rand(600, generator=g, device="cuda") / 600
    want = oz.oz2_linear_xent_grad(dloss, x, w, t, lse)
    loss = oz.oz2_linear_xent(x, w, t)[0]
    for bad in (float("nan"), float("inf"), -float("inf"), torch.finfo(dt).max):
        x2, l2, d2 = x.clone(), lse.clone(), dloss.clone()
        x2[dead], l2[dead], d2[dead] = bad, bad, bad
        got = oz.oz2_linear_xent(x2, w, t)
        assert torch.equal(got[0], loss) and not got[2][dead].any()
        assert all(torch.equal(a, b) for a, b in zip(want, oz.oz2_linear_xent_grad(d2, x2, w, t, l2)))
    none = torch.full_like(t, -1)
    assert not oz.oz2_linear_xent(x, w, none)[0].any()
    assert not any(v.any() for v in oz.oz2_linear_xent_grad(dloss, x, w, none, lse))


def test_a_target_beyond_is_nan(oz):
    g, x, w, t = inputs(300, 500, 64, BF16, masked=False)
    good = oz.oz2_linear_xent(x, w, t)
    t2 = t.clone()
    t2[7], t2[9] = 500, 1 << 40
    loss, lse, picked = oz.oz2_linear_xent(x, w, t2)
    bad = t2 >= 500
    assert loss[bad].isnan().all() and picked[bad].isnan().all() and torch.equal(lse, good[1])
    assert torch.equal(loss[~bad], good[0][~bad])
    dx, dw = oz.oz2_linear_xent_grad(torch.ones(300, device="cuda"), x, w, t2, lse)
    assert dx[bad].isnan().all() and dw.isnan().all() and dx[~bad].isfinite().all()


def test_hard_logits(oz):
    """Logits that are all alike, far apart, masked by the type's lowest value, infinite."""
    w = torch.zeros(300, 64, device="cuda").to(BF16)
    w[:, 0] = torch.linspace(-1, 1, 300, device="cuda").to(BF16)
    x = torch.zeros(6, 64, device="cuda").to(BF16)
    x[1, 0], x[2, 0], x[3, 0] = 1000, -1000, 1e-3
    t = torch.tensor([0, 299, 0, 17, 5, 5], device="cuda")
    want, bound = ref.xent(x, w, t)
    for a, v, e in zip(oz.oz2_linear_xent(x, w, t), want, bound):
        close(a, v, e)
    lse = want[1].float()
    dloss = torch.ones(6, device="cuda")
    for a, v, e in zip(oz.oz2_linear_xent_grad(dloss, x, w, t, lse), *ref.xent_grad(dloss, x, w, t, lse)):
        close(a, v, e)
    # Rows that a mask takes out: their logits are the lowest or minus infinity.
    x[:, 1] = 1
    for low in (torch.finfo(BF16).min, -float("inf")):
        w[100:, 1] = low
        t = torch.tensor([0, 99, 0, 17, 5, 5], device="cuda")
        loss, lse, picked = oz.oz2_linear_xent(x, w, t)
        want, bound = ref.xent(x, w[:100], t)
        for a, v, e in zip((loss, lse, picked), want, bound):
            close(a, v, e)
    # A logit of plus infinity: lse is, too; NaN stays NaN.
    w[:, 1] = 0
    w[3, 1] = float("inf")
    loss, lse, _ = oz.oz2_linear_xent(x, w, t)
    assert lse.isinf().all() and loss.isinf().all()
    w[3, 1] = float("nan")
    assert oz.oz2_linear_xent(x, w, t)[1].isnan().all()


def test_nearly_certain_tokens(oz):
    """p of the target within 2^-20 of 1: its gradient is that of p - 1, not of two FP32 numbers'
    difference.  Relative to the value, for z and lse given as they are."""
    w = torch.zeros(64, 64, device="cuda").to(BF16)
    w[0, 0] = 1
    x = torch.zeros(4, 64, device="cuda").to(BF16)
    x[:, 0] = torch.tensor([8.0, 12.0, 16.0, 4.0])
    t = torch.zeros(4, dtype=torch.int64, device="cuda")
    lse = torch.logsumexp(x.double() @ w.double().t(), 1)
    lse32 = lse.float()
    dx, _ = oz.oz2_linear_xent_grad(torch.ones(4, device="cuda"), x, w, t, lse32)
    want = torch.expm1(x[:, 0].double() - lse32.double())  # dz of the target; w picks it alone
    # (An ulp of 16's logarithmic sum in FP32 is 2^-20: the exponent is known to that much.)
    assert ((dx[:, 0].double() - want).abs() <= 2 * 2.0 ** -8 * want.abs() + 2.0 ** -19).all()


@pytest.mark.parametrize("dt", [BF16, F16])
def test_small_gradients_stay(oz, dt):
    """Losses' gradients far below F16's range: dw in float32 has them, relative to the whole.  (The
    same outputs are wanted of every call: how the sums are split goes by that.)"""
    g, x, w, t = inputs(500, 700, 64, dt, masked=False)
    lse = ref.xent(x, w, t)[0][1].float()
    whole = oz.oz2_linear_xent_grad(torch.full((500,), 1.0, device="cuda"), x, w, t, lse, dw_dtype=torch.float32,
                                    need=("dw",))[1]
    for scale in (2.0 ** -30, 2.0 ** 20):
        small = oz.oz2_linear_xent_grad(torch.full((500,), scale, device="cuda"), x, w, t, lse, dw_dtype=torch.float32,
                                        need=("dw",))[1]
        assert torch.equal(small / scale, whole)  # powers of two: the same bits


def test_dloss_of_one_for_all(oz):
    g, x, w, t = inputs(300, 700, 128, BF16)
    lse = oz.oz2_linear_xent(x, w, t)[1]
    one = torch.tensor(0.5, device="cuda")
    want = oz.oz2_linear_xent_grad(torch.full((300,), 0.5, device="cuda"), x, w, t, lse)
    for d in (one, one.expand(300)):
        assert all(torch.equal(a, b) for a, b in zip(want, oz.oz2_linear_xent_grad(d, x, w, t, lse)))


def test_what_is_wanted_and_given(oz):
    g, x, w, t = inputs(400, 1000, 200, BF16)
    lse = oz.oz2_linear_xent(x, w, t)[1]
    dloss = torch.rand(400, generator=g, device="cuda")
    dx, dw = oz.oz2_linear_xent_grad(dloss, x, w, t, lse, dw_dtype=torch.float32)
    a = oz.oz2_linear_xent_grad(dloss, x, w, t, lse, need=("dx",))
    b = oz.oz2_linear_xent_grad(dloss, x, w, t, lse, need=("dw",), dw_dtype=torch.float32)
    bx, bw = ref.xent_grad(dloss, x, w, t, lse, dw_dtype=torch.float32)[1]
    assert a[1] is None and b[0] is None
    close(a[0], dx.double(), 2 * bx)
    close(b[1], dw.double(), 2 * bw)
    to, tw = torch.full((402, 208), 3.0, device="cuda").to(BF16), torch.full((1001, 232), 3.0, device="cuda")
    got = oz.oz2_linear_xent_grad(dloss, x, w, t, lse, dx=to[1:401, 3:203], dw=tw[:1000, 5:205])
    assert torch.equal(got[0], dx) and torch.equal(got[1], dw)
    to[1:401, 3:203] = 3
    tw[:1000, 5:205] = 3
    assert (to == 3).all() and (tw == 3).all()
    old = torch.randn(1000, 200, generator=g, device="cuda")
    want, bound = ref.xent_grad(dloss, x, w, t, lse, dw_dtype=torch.float32, old=old)
    oz.oz2_linear_xent_grad(dloss, x, w, t, lse, dw=old, accumulate=True)
    close(old, want[1], bound[1])
    with pytest.raises(AssertionError, match="accumulate"):
        oz.oz2_linear_xent_grad(dloss, x, w, t, lse, accumulate=True)


@pytest.mark.parametrize("dt", [BF16, F16])
def test_pieces_of_the_vocabulary(oz, dt):
    """So many tokens and rows that dz is formed in pieces, the last one short."""
    m, n, k = 9000, 70001, 24
    g, x, w, t = inputs(m, n, k, dt)
    x, w = x.contiguous(), w.contiguous()
    loss, lse, picked = oz.oz2_linear_xent(x, w, t)
    dloss = torch.rand(m, generator=g, device="cuda") / m
    dx, dw = oz.oz2_linear_xent_grad(dloss, x, w, t, lse, dw_dtype=torch.float32)
    rows = torch.tensor([0, 1, 4500, 8999], device="cuda")  # of dx, of all pieces
    want, bound = ref.xent(x[rows], w, t[rows])
    for a, v, e in zip((loss, lse, picked), want, bound):
        close(a[rows], v, e)
    big = dloss.max() / dloss[rows].max()  # (f16's scale is that of all tokens)
    want, bound = ref.xent_grad(dloss[rows], x[rows], w, t[rows], lse[rows])
    close(dx[rows], want[0], bound[0] * float(max(1, big)))
    cols = torch.cat([torch.arange(0, 40), torch.arange(34900, 35300, 7), torch.arange(69950, 70001)]).cuda()
    p = torch.exp(x.double() @ w[cols].double().t() - lse.double()[:, None])
    dz = dloss.double()[:, None] * (p - (t[:, None] == cols).double()) * (t >= 0)[:, None]
    want = dz.t() @ x.double()
    # dz's rounding, the logits' error (a depth of 24: 18 steps of 2^-22) and the sums of 9000.
    size = dz.abs().t() @ x.double().abs()
    near = ref.U[dt] + 1e-4 + (9000 / 16 + 16) * 2.0 ** -22
    close(dw[cols], want, near * size + 2.0 ** -38 * float(dloss.max()) * x.double().abs().sum(0))


def test_against_differences(oz):
    """dL of L = Σ c·loss along a direction of bf16 steps that are exact: the loss is smooth, and a
    central difference of steps h leaves h²·|L'''|/6."""
    g = rng(3)
    m, n, k = 40, 100, 64
    x = (torch.randint(-64, 65, (m, k), generator=g, device="cuda") / 64).to(BF16)
    w = (torch.randint(-64, 65, (n, k), generator=g, device="cuda") / 256).to(BF16)
    t = torch.randint(0, n, (m,), generator=g, device="cuda")
    c = torch.rand(m, generator=g, device="cuda")
    zl = 1e-2
    _, lse, _ = oz.oz2_linear_xent(x, w, t, z_loss=zl)
    dx, dw = oz.oz2_linear_xent_grad(c, x, w, t, lse, z_loss=zl, dw_dtype=torch.float32)
    loss = lambda x, w: (oz.oz2_linear_xent(x, w, t, z_loss=zl)[0].double() * c.double()).sum()  # noqa: E731
    for grad, which in ((dx, 0), (dw, 1)):
        base = (x, w)[which]
        v = (torch.randint(0, 2, base.shape, generator=g, device="cuda") * 2 - 1).to(BF16) * 2.0 ** -7
        p, q = base + v, base - v
        moved = (p.double() - q.double())  # what the rounding left of it
        args = [(p, w), (q, w)] if which == 0 else [(x, p), (x, q)]
        num = loss(*args[0]) - loss(*args[1])
        want = (grad.double() * moved).sum()
        # dz's rounding 2^-8 of each term, in random directions; the third order (2^-7·√k)³/6 a token.
        room = 2.0 ** -7 * (grad.double().abs() * moved.abs()).sum() + m * (2.0 ** -7 * 8 * 8) ** 3 / 6 * 1e-2
        assert abs(num - want) < room


def test_streams_and_graphs(oz):
    g, x, w, t = inputs(700, 3000, 128, BF16)
    dloss = torch.rand(700, generator=g, device="cuda")
    fwd = oz.oz2_linear_xent(x, w, t)
    want = oz.oz2_linear_xent_grad(dloss, x, w, t, fwd[1])
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [(oz.oz2_linear_xent(x, w, t, stream=s), oz.oz2_linear_xent_grad(dloss, x, w, t, fwd[1], stream=s))
           for _ in range(4) for s in streams]
    torch.cuda.synchronize()
    for a, b in got:
        assert all(torch.equal(u, v) for u, v in zip(a, fwd)) and all(torch.equal(u, v) for u, v in zip(b, want))
    xs, ts = torch.zeros_like(x), torch.zeros_like(t)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f2 = oz.oz2_linear_xent(xs, w, ts)
        g2 = oz.oz2_linear_xent_grad(dloss, xs, w, ts, f2[1])
    xs.copy_(x)
    ts.copy_(t)
    for _ in range(2):
        graph.replay()
        assert all(torch.equal(u, v) for u, v in zip(f2, fwd)) and all(torch.equal(u, v) for u, v in zip(g2, want))
    assert oz.oz2_check_device_status() == 0


@pytest.mark.parametrize("dt", [BF16, F16])
@pytest.mark.parametrize("scale", [1.0, 0.3, -0.7])
@pytest.mark.parametrize("z_loss", [0.0, 1e-3])
def test_a_certain_targets_gradient_keeps_its_accuracy(oz, dt, scale, z_loss):
    """dz of targets whose p is within 1e-6 to 1e-3 of 1, or 1, for z and lse as they are given: z - lse
    is rounded once, so dz is off by its rounding to 16 bits, the result's, and a few steps of FP32
    relative to itself (with z_loss, to its terms); where z = lse it is 0 but for z_loss's term."""
    z = torch.tensor([4.0, 8, 12, 16, 20, 22, 27, 30], device="cuda")
    w = torch.zeros(64, 64, device="cuda").to(dt)  # (the other rows are 0 in the one feature looked at)
    w[0, 0] = 1 if scale > 0 else -1
    x = torch.zeros(8, 64, device="cuda").to(dt)
    x[:, 0] = (z / abs(scale)).round()  # whole numbers: the products are exact
    t = torch.zeros(8, dtype=torch.int64, device="cuda")
    s, c = torch.tensor([scale, z_loss], dtype=torch.float32).double().cuda()
    z = s * x.double() @ w[0].double()
    for off in (0.0, 1e-6, 5e-6, 2e-5, 1e-3):
        lse = (z + off).float()
        e = 2 * c * lse.double()
        dx, _ = oz.oz2_linear_xent_grad(torch.ones(8, device="cuda"), x, w, t, lse, scale=scale, z_loss=z_loss)
        want = s * ((1 + e) * torch.expm1(z - lse.double()) + e) * w[0, 0].double()
        # (f16: dz and results below its normal range.)
        err = 2 * ref.U[dt] * want.abs() + 16 * ref.u * (s.abs() * e + want.abs()) + (2.0 ** -25 + 2.0 ** -38 if dt == F16 else 0)
        assert ((dx[:, 0].double() - want).abs() <= err).all()


def test_nan_beside_infinity(oz):
    """A token with a logit of plus infinity and one that is NaN: lse is NaN, wherever they are; with
    the infinity alone it is that."""
    w = torch.zeros(700, 64, device="cuda").to(BF16)
    x = torch.zeros(5, 64, device="cuda").to(BF16)
    x[:, 0] = 1
    t = torch.zeros(5, dtype=torch.int64, device="cuda")
    for a, b in ((3, 5), (5, 3), (0, 63), (3, 600), (600, 3), (130, 699), (699, 698)):
        for scale in (1.0, -1.0):
            w[:, 0] = 0
            w[a, 0], w[b, 0] = scale * float("inf"), float("nan")
            loss, lse, _ = oz.oz2_linear_xent(x, w, t, scale=scale)
            assert lse.isnan().all() and loss.isnan().all()
            w[b, 0] = 1
            assert (oz.oz2_linear_xent(x, w, t, scale=scale)[1] == float("inf")).all()


@pytest.mark.parametrize("dloss", [1.9999, 1.0, 3.9999 * 2.0 ** -9])
def test_f16_scale_has_room_for_negative_z_loss(oz, dloss):
    """1 + 2·z_loss·lse at -1: a certain target's dz is -2·dloss, twice any other's, and stays in
    f16's range under the scale that the largest dloss gets (one row of w: p is 1)."""
    x = torch.full((3, 1), 10.0, device="cuda").half()
    w = torch.ones(1, 1, device="cuda").half()
    t = torch.zeros(3, dtype=torch.int64, device="cuda")
    d, lse = torch.full((3,), dloss, device="cuda"), torch.full((3,), 10.0, device="cuda")
    dx, dw = oz.oz2_linear_xent_grad(d, x, w, t, lse, z_loss=-0.1, dw_dtype=torch.float32)
    dz = d.double() * 2 * -0.1 * 10
    assert ((dx[:, 0].double() - dz).abs() <= 2 * ref.U[F16] * dz.abs()).all()
    want = (dz * 10).sum()
    assert abs(dw[0, 0].double() - want) <= (ref.U[F16] + 8 * ref.u) * abs(want)


@pytest.mark.parametrize("how", ["whole", "odd"])
def test_added_to_over_pieces(oz, how):
    """dw in float32 added to where dz is formed in pieces of the vocabulary: what is stored, and one
    addition; what lies beside it stays."""
    m, n, k = 9000, 70001, 40
    g, x, w, t = inputs(m, n, k, BF16)
    lse = oz.oz2_linear_xent(x, w, t)[1]
    d = torch.rand(m, generator=g, device="cuda") / m
    dx, dw = oz.oz2_linear_xent_grad(d, x, w, t, lse, dw_dtype=torch.float32)
    old = view(torch.randn(n, k, generator=g, device="cuda"), how)
    whole, sums = old._base, old + dw
    dx2, to = oz.oz2_linear_xent_grad(d, x, w, t, lse, dw=old, accumulate=True)
    assert to is old and torch.equal(old, sums) and torch.equal(dx, dx2)
    if how == "odd":
        old[:] = float("nan")
        assert whole.isnan().all()
