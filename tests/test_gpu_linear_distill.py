"""oz2_linear_distill and its gradient against their formulas in 64 bits."""
import pytest
import torch

import lm_ref as ref
from helpers import ensure_built
from layers_ref import close
from test_gpu_linear_xent import rng, view

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def oz():
    ensure_built()
    import paper_2606_06510_gb300 as oz
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    return oz


def inputs(m, n, k, top, dt, how="whole", seed=0, ragged=True, repeated=False, teacher=torch.float32, ids=torch.int64):
    g = rng(seed + m + n + k + top)
    w = view((torch.randn(n, k, generator=g, device="cuda") * 2 * k ** -0.5).to(dt), how)
    x = view(torch.randn(m, k, generator=g, device="cuda").to(dt), how)
    if repeated or top > n:
        at = torch.randint(0, min(n, 3 * top), (m, top), generator=g, device="cuda")
    else:
        at = torch.rand(m, n, generator=g, device="cuda").topk(top, dim=1)[1]
    if ragged:  # some entries not there, some lists empty
        at = torch.where(torch.rand(m, top, generator=g, device="cuda") < torch.rand(m, 1, generator=g, device="cuda"),
                         torch.full_like(at, -1), at)
        at[::7] = -1
    logits = (3 * torch.randn(m, top, generator=g, device="cuda")).to(teacher)
    return g, x, w, view(at.to(ids), how), view(logits, how)


CASES = [
    (1, 1, 64, 1, {}), (2, 64, 64, 1, {}), (3, 100, 72, 2, dict(teacher=BF16)), (40, 300, 128, 33, dict(how="odd")),
    (130, 700, 96, 64, dict(teacher=F16, ids=torch.int32)), (257, 513, 65, 5, dict(how="odd", ids=torch.int32)),
    (300, 2000, 256, 128, dict(how="strided")), (20, 50, 64, 50, dict(ragged=False)), (30, 200, 64, 100, dict(repeated=True)),
    (9, 5000, 64, 1024, {}), (70, 300, 128, 300, dict(ragged=False)),
    (20, 400000, 8, 40, {}), (600, 9000, 40, 17, dict(ragged=False)), (5, 64, 64, 300, dict(repeated=True))]


@pytest.mark.parametrize("dt", [BF16, F16])
@pytest.mark.parametrize("at", range(len(CASES)))
@pytest.mark.parametrize("temperature", [1.0, 2.5])
def test_both_ways(oz, dt, at, temperature):
    m, n, k, top, more = CASES[at]
    g, x, w, ids, teacher = inputs(m, n, k, top, dt, **more)
    want, bound = ref.distill(x, w, ids, teacher, temperature)
    got = oz.oz2_linear_distill(x, w, ids, teacher, temperature=temperature)
    for a, v, e, what in zip(got, want, bound, ("loss", "lse", "picked")):
        close(a, v, e, what)
    again = oz.oz2_linear_distill(x, w, ids, teacher, temperature=temperature)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    lse = want[1].float()
    dloss = torch.rand(m, generator=g, device="cuda") / m
    for wt in (dt, torch.float32):
        want, bound = ref.distill_grad(dloss, x, w, ids, teacher, lse, temperature, wt)
        got = oz.oz2_linear_distill_grad(dloss, x, w, ids, teacher, lse, temperature=temperature, dw_dtype=wt)
        for a, v, e, what in zip(got, want, bound, ("dx", "dw")):
            close(a, v, e, what)
    again = oz.oz2_linear_distill_grad(dloss, x, w, ids, teacher, lse, temperature=temperature, dw_dtype=wt)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_one_certain_row_is_cross_entropy(oz):
    """A teacher that lists one row: the loss and gradient of that target, bit for bit but for the
    loss's order of additions."""
    g, x, w, ids, teacher = inputs(300, 800, 128, 1, BF16)
    loss, lse, picked = oz.oz2_linear_distill(x, w, ids, teacher)
    l2, lse2, p2 = oz.oz2_linear_xent(x, w, ids[:, 0].contiguous())
    assert torch.equal(lse, lse2) and torch.equal(picked[:, 0], p2)
    assert ((loss - l2).abs() <= 4 * ref.u * (lse.abs() + p2.abs())).all()


def test_what_is_not_listed_holds_anything(oz):
    g, x, w, ids, teacher = inputs(200, 500, 64, 20, BF16)
    none = ids < 0
    dead = none.all(1)
    assert dead.any() and not dead.all()
    fwd = oz.oz2_linear_distill(x, w, ids, teacher)
    dloss = torch.rand(200, generator=g, device="cuda")
    want = oz.oz2_linear_distill_grad(dloss, x, w, ids, teacher, fwd[1])
    assert not fwd[0][dead].any() and not want[0][dead].any() and not fwd[2][none].any()
    for bad in (float("nan"), float("inf"), -float("inf"), torch.finfo(torch.float32).min):
        t2, x2, l2, d2 = teacher.clone(), x.clone(), fwd[1].clone(), dloss.clone()
        t2[none], x2[dead], l2[dead], d2[dead] = bad, bad, bad, bad
        got = oz.oz2_linear_distill(x2, w, ids, t2)
        assert torch.equal(got[0], fwd[0]) and torch.equal(got[2], fwd[2])
        assert all(torch.equal(a, b) for a, b in zip(want, oz.oz2_linear_distill_grad(d2, x2, w, ids, t2, l2)))


def test_hard_teachers(oz):
    """Rows that the teacher rules out, by minus infinity or the lowest value, weigh nothing; a
    teacher that is lowest everywhere is even."""
    g, x, w, ids, teacher = inputs(60, 300, 64, 16, BF16, ragged=False)
    for low in (-float("inf"), torch.finfo(torch.float32).min):
        t = teacher.clone()
        t[:, 8:] = low
        got, want = oz.oz2_linear_distill(x, w, ids, t), oz.oz2_linear_distill(x, w, ids[:, :8], t[:, :8])
        assert ((got[0] - want[0]).abs() <= 64 * ref.u * (got[1].abs() + 20)).all() and torch.equal(got[1], want[1])
        d = torch.ones(60, device="cuda")
        a = oz.oz2_linear_distill_grad(d, x, w, ids, t, got[1])
        b = oz.oz2_linear_distill_grad(d, x, w, ids[:, :8], t[:, :8], got[1])
        bound = ref.distill_grad(d, x, w, ids[:, :8], t[:, :8], got[1], 1.0)[1]
        for u, v, e in zip(a, b, bound):
            close(u, v.double(), 2 * e)
    even = torch.full_like(teacher, torch.finfo(torch.float32).min)
    got, want = oz.oz2_linear_distill(x, w, ids, even), oz.oz2_linear_distill(x, w, ids, torch.zeros_like(even))
    assert torch.equal(got[0], want[0])


def test_an_entry_beyond_is_nan(oz):
    g, x, w, ids, teacher = inputs(100, 300, 64, 10, BF16, ragged=False)
    good = oz.oz2_linear_distill(x, w, ids, teacher)
    i2 = ids.clone()
    i2[5, 3], i2[6, 0] = 300, 1 << 50
    i2[7, 1], teacher[7, 1] = 301, -float("inf")  # nor does it matter what the teacher thinks of it
    loss, lse, picked = oz.oz2_linear_distill(x, w, i2, teacher)
    bad = (i2 >= 300).any(1)
    assert loss[bad].isnan().all() and torch.equal(loss[~bad], good[0][~bad])
    assert torch.equal(picked.isnan(), i2 >= 300)
    dx, dw = oz.oz2_linear_distill_grad(torch.ones(100, device="cuda"), x, w, i2, teacher, lse)
    assert dx[bad].isnan().all() and dw.isnan().all() and dx[~bad].isfinite().all()


def test_no_tokens(oz):
    w = torch.randn(90, 64, device="cuda").to(BF16)
    ids, f = torch.zeros(0, 4, dtype=torch.int64, device="cuda"), torch.zeros(0, device="cuda")
    loss, lse, picked = oz.oz2_linear_distill(w[:0], w, ids, torch.zeros(0, 4, device="cuda"))
    assert loss.shape == lse.shape == (0,) and picked.shape == (0, 4)
    dx, dw = oz.oz2_linear_distill_grad(f, w[:0], w, ids, torch.zeros(0, 4, device="cuda"), f)
    assert dx.shape == (0, 64) and not dw.any()


def test_against_differences(oz):
    g = rng(3)
    m, n, k, top = 40, 100, 64, 6
    x = (torch.randint(-64, 65, (m, k), generator=g, device="cuda") / 64).to(BF16)
    w = (torch.randint(-64, 65, (n, k), generator=g, device="cuda") / 256).to(BF16)
    ids = torch.rand(m, n, generator=g, device="cuda").topk(top, dim=1)[1]
    teacher = torch.randn(m, top, generator=g, device="cuda")
    c = torch.rand(m, generator=g, device="cuda")
    _, lse, _ = oz.oz2_linear_distill(x, w, ids, teacher, temperature=2.0)
    dx, dw = oz.oz2_linear_distill_grad(c, x, w, ids, teacher, lse, temperature=2.0, dw_dtype=torch.float32)
    loss = lambda x, w: (oz.oz2_linear_distill(x, w, ids, teacher, temperature=2.0)[0].double() * c.double()).sum()  # noqa: E731
    for grad, which in ((dx, 0), (dw, 1)):
        base = (x, w)[which]
        v = (torch.randint(0, 2, base.shape, generator=g, device="cuda") * 2 - 1).to(BF16) * 2.0 ** -7
        p, q = base + v, base - v
        moved = p.double() - q.double()
        args = [(p, w), (q, w)] if which == 0 else [(x, p), (x, q)]
        num, want = loss(*args[0]) - loss(*args[1]), (grad.double() * moved).sum()
        room = 2.0 ** -7 * (grad.double().abs() * moved.abs()).sum() + m * (2.0 ** -7 * 8 * 8) ** 3 / 6 * 1e-2
        assert abs(num - want) < room


@pytest.mark.parametrize("teacher_type", [torch.float32, BF16, F16])
@pytest.mark.parametrize("temperature", [0.5, 1e-3, 3.0])
def test_lowest_logits_at_any_temperature(oz, teacher_type, temperature):
    """A list of the teacher's lowest values is even, though they pass FP32's range once divided;
    beside others they weigh nothing."""
    g, x, w, ids, _ = inputs(60, 300, 64, 16, BF16, ragged=False)
    d = torch.ones(60, device="cuda")
    even = torch.full((60, 16), torch.finfo(teacher_type).min, device="cuda", dtype=teacher_type)
    got = oz.oz2_linear_distill(x, w, ids, even, temperature=temperature)
    want = oz.oz2_linear_distill(x, w, ids, torch.zeros_like(even), temperature=temperature)
    assert got[0].isfinite().all() and all(torch.equal(a, b) for a, b in zip(got, want))
    a = oz.oz2_linear_distill_grad(d, x, w, ids, even, got[1], temperature=temperature)
    b = oz.oz2_linear_distill_grad(d, x, w, ids, torch.zeros_like(even), got[1], temperature=temperature)
    assert all(v.isfinite().all() and torch.equal(v, u) for v, u in zip(a, b))
    one = even.clone()
    one[:, 3] = 1
    sure = torch.full_like(even, -float("inf"))
    sure[:, 3] = 1
    got = oz.oz2_linear_distill(x, w, ids, one, temperature=temperature)
    assert torch.equal(got[0], oz.oz2_linear_distill(x, w, ids, sure, temperature=temperature)[0])


@pytest.mark.parametrize("dt", [BF16, F16])
def test_pieces_of_the_vocabulary(oz, dt):
    """dz formed in pieces of the vocabulary (three of 23552 rows here), with listed rows on both sides
    of their borders; dw stored, and added to in float32."""
    m, n, k, top, T = 9000, 70001, 24, 9, 1.5
    g, x, w, ids, teacher = inputs(m, n, k, top, dt, repeated=True)
    ids[:, :top] = torch.randint(0, n, (m, top), generator=g, device="cuda")
    borders = torch.tensor([0, 23551, 23552, 47103, 47104, 70000], device="cuda")
    ids[:, 2:5] = borders[torch.randint(0, 6, (m, 3), generator=g, device="cuda")]
    ids[torch.rand(ids.shape, generator=g, device="cuda") < 0.2] = -1
    ids[::11] = -1
    live = (ids >= 0).any(1)
    loss, lse, picked = oz.oz2_linear_distill(x, w, ids, teacher, temperature=T)
    d = torch.rand(m, generator=g, device="cuda") / m
    dx, dw = oz.oz2_linear_distill_grad(d, x, w, ids, teacher, lse, temperature=T, dw_dtype=torch.float32)
    rows = torch.tensor([0, 1, 5, 4500, 8990, 8999], device="cuda")
    want, bound = ref.distill(x[rows], w, ids[rows], teacher[rows], T)
    for a, v, e in zip((loss, lse, picked), want, bound):
        close(a[rows], v, e)
    big = float(max(1, d.max() / d[rows].max()))  # (f16's scale is that of all tokens)
    want, bound = ref.distill_grad(d[rows], x[rows], w, ids[rows], teacher[rows], lse[rows], T)
    close(dx[rows], want[0], bound[0] * big)
    # dw of rows of w around the borders: dz's rounding, the logits' error (a depth of 24: 18 steps of
    # 2^-22), the weights' and the sums' of 9000.
    cols = torch.cat([torch.arange(a, b) for a, b in ((0, 40), (23500, 23600), (47050, 47160), (69950, 70001))]).cuda()
    p = torch.exp(x.double() @ w[cols].double().t() / T - lse.double()[:, None])
    q = ref.teacher(ids, teacher, T, n)[0]
    hot = torch.zeros(m, n, device="cuda").double().scatter_add_(1, ids.clamp_min(0), q)[:, cols]
    c = (d.double() / T * live)[:, None]
    dz, parts = c * (p - hot), c * (p + hot)
    near = ref.U[dt] + 1e-4 + (m / 16 + 16) * 2.0 ** -22
    size = dz.abs().t() @ x.double().abs() * near + 2e-4 * (parts.t() @ x.double().abs()) + \
        2.0 ** -38 * float(d.max()) * x.double().abs().sum(0)
    close(dw[cols], dz.t() @ x.double(), size)
    old = torch.randn(n, k, generator=g, device="cuda")
    sums = old + dw  # (the same sums, then one addition)
    _, to = oz.oz2_linear_distill_grad(d, x, w, ids, teacher, lse, temperature=T, dw=old, accumulate=True)
    assert to is old and torch.equal(old, sums)
    only = oz.oz2_linear_distill_grad(d, x, w, ids, teacher, lse, temperature=T, need=("dx",))
    close(only[0][rows], want[0], bound[0] * big)


def test_long_lists_of_a_large_vocabulary(oz):
    """Lists whose keys, a row and a place among 1024, take more than 32 bits."""
    m, n, k, top = 2, 4200000, 8, 1024
    g = rng(9)
    w = (torch.randn(n, k, generator=g, device="cuda") / 2).to(BF16)
    x = torch.randn(m, k, generator=g, device="cuda").to(BF16)
    ids = torch.randint(0, n, (m, top), generator=g, device="cuda")
    ids[:, :300] = n - 1 - torch.arange(300, device="cuda")
    ids[:, 300:310] = torch.arange(10, device="cuda")
    ids = ids[:, torch.randperm(top, generator=g, device="cuda")].contiguous()
    ids[1, ::3] = -1
    teacher = 3 * torch.randn(m, top, generator=g, device="cuda")
    want, bound = ref.distill(x, w, ids, teacher, 1.0)
    got = oz.oz2_linear_distill(x, w, ids, teacher)
    for a, v, e, what in zip(got, want, bound, ("loss", "lse", "picked")):
        close(a, v, e, what)
    d = torch.ones(m, device="cuda")
    lse = want[1].float()
    want, bound = ref.distill_grad(d, x, w, ids, teacher, lse, 1.0, torch.float32)
    for a, v, e, what in zip(oz.oz2_linear_distill_grad(d, x, w, ids, teacher, lse, dw_dtype=torch.float32), want, bound,
                             ("dx", "dw")):
        close(a, v, e, what)
