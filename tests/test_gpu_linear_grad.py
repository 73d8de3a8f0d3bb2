"""oz2_linear_grad against its formula in 64 bits and against differences."""
import pytest

import layers_ref as ref
from helpers import ensure_built

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


def make(torch, m, n, k, dtype, seed=0, pad=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000 * seed + m + 3 * n + 7 * k)

    def normal(rows, cols):
        return torch.randn((rows, cols + pad), generator=g, device="cuda").to(dtype)[:, pad // 2:pad // 2 + cols]

    return normal(m, n), normal(m, k), normal(n, k) * max(n, 1) ** -0.5, normal(m, n)


def check(got, dy, x, w, z, name, torch):
    want, bounds, _ = ref.grad(dy, x, w, z, name)
    for a, b, e, what in zip(got, want, bounds, ("dx", "dw", "db")):
        ref.close(a, b, e, what)


@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 300, 200), (8, 128, 64), (17, 257, 130), (100, 64, 1032), (128, 128, 128),
                                   (129, 255, 129), (256, 256, 256), (300, 1000, 72), (513, 257, 1027),
                                   (5000, 96, 130), (8192, 256, 192), (1000, 1333, 777), (16384, 512, 512),
                                   (20000, 200, 1000), (40, 2000, 3000), (2304, 1536, 1280), (2304, 2200, 2304),
                                   (1000, 2500, 5000)])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_shapes(env, shape, kind):
    oz, torch = env
    dt = {"bf16": torch.bfloat16, "f16": torch.float16}[kind]
    m, n, k = shape
    name = ref.ACTS[(m + n + k) % 5]
    dy, x, w, z = make(torch, m, n, k, dt)
    got = oz.oz2_linear_grad(dy, x, w, pre=z, act=name)
    check(got, dy, x, w, z, name, torch)
    again = oz.oz2_linear_grad(dy, x, w, pre=z, act=name)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("name", ref.ACTS)
def test_activations(env, name):
    oz, torch = env
    m, n, k = 200, 144, 96
    for dt in (torch.bfloat16, torch.float16):
        dy, x, w, z = make(torch, m, n, k, dt, seed=1)
        z = (z.float() * 4).to(dt)
        z[0, :8] = torch.tensor([0.0, -0.0, 100.0, -100.0, 6e4, -6e4, 1e-7, -1e-7], device="cuda").to(dt)
        check(oz.oz2_linear_grad(dy, x, w, pre=z, act=name), dy, x, w, z, name, torch)


@pytest.mark.parametrize("pad", [2, 6, 16])
def test_strided(env, pad):
    oz, torch = env
    for m, n, k in ((150, 120, 88), (151, 121, 89)):
        dy, x, w, z = make(torch, m, n, k, torch.bfloat16, seed=2, pad=pad)
        for name in ("none", "gelu"):
            hold = torch.full((n, k + pad), 7.0, dtype=torch.bfloat16, device="cuda")
            dw = hold[:, 1:1 + k]
            dx, dw, db = oz.oz2_linear_grad(dy, x, w, pre=z, act=name, dw=dw)
            check((dx, dw, db), dy, x, w, z, name, torch)
            assert (hold[:, 0] == 7).all() and (hold[:, 1 + k:] == 7).all()


def test_each_gradient_alone(env):
    oz, torch = env
    dy, x, w, z = make(torch, 300, 200, 100, torch.float16, seed=3)
    whole = oz.oz2_linear_grad(dy, x, w, pre=z, act="silu")
    for i, name in enumerate(("dx", "dw", "db")):
        alone = oz.oz2_linear_grad(dy, x, w, pre=z, act="silu", need=(name,))
        assert torch.equal(alone[i], whole[i])
        assert all(alone[j] is None for j in range(3) if j != i)


def test_f32_weights_gradient_and_accumulation(env):
    """A weight's gradient over four parts of the tokens, added up in float32."""
    oz, torch = env
    m, n, k = 512, 130, 70
    dy, x, w, z = make(torch, m, n, k, torch.bfloat16, seed=4)
    want, (_, _, bb), ew = ref.grad(dy, x, w, z, "gelu_tanh")
    dw = torch.full((n, k), 3.0, device="cuda")
    db = torch.full((n,), -2.0, device="cuda")
    for a in range(0, m, 128):
        s = slice(a, a + 128)
        oz.oz2_linear_grad(dy[s], x[s], w, pre=z[s], act="gelu_tanh", dw=dw, db=db, accumulate=True)
    size = want[1].abs() + 3
    ref.close(dw, want[1] + 3, ew + 8 * 2.0 ** -23 * size, "dw")
    ref.close(db, want[2] - 2, bb + 8 * 2.0 ** -23 * (want[2].abs() + 2), "db")
    one = oz.oz2_linear_grad(dy, x, w, pre=z, act="gelu_tanh", dw_dtype=torch.float32)[1]
    ref.close(one, want[1], ew + 2.0 ** -23 * size, "dw in one")
    dw2, db2 = dw.clone(), db.clone()
    oz.oz2_linear_grad(dy[:0], x[:0], w, pre=z[:0], act="gelu_tanh", dw=dw2, db=db2, accumulate=True)
    assert torch.equal(dw, dw2) and torch.equal(db, db2)


def test_empty_problems(env):
    oz, torch = env
    bf = torch.bfloat16
    e = lambda *s: torch.ones(s, dtype=bf, device="cuda")  # noqa: E731
    dx, dw, db = oz.oz2_linear_grad(e(0, 24), e(0, 16), e(24, 16))
    assert dx.shape == (0, 16) and not dw.any() and not db.any()
    dx, dw, db = oz.oz2_linear_grad(e(7, 0), e(7, 16), e(0, 16))
    assert not dx.any() and dx.shape == (7, 16) and dw.shape == (0, 16) and db.shape == (0,)
    dx, dw, db = oz.oz2_linear_grad(e(7, 24), e(7, 0), e(24, 0))
    assert dx.shape == (7, 0) and dw.shape == (24, 0) and torch.equal(db, torch.full((24,), 7.0, device="cuda"))


@pytest.mark.parametrize("name", ref.ACTS)
def test_against_differences(env, name):
    """⟨gradient, direction⟩ against (L(+h) - L(-h))/2h of L = Σ dy∘y in 64 bits,
    at the formula's truncation error h²·|L'''|/6 and the gradients' own bounds."""
    oz, torch = env
    m, n, k, h = 24, 40, 32, 1e-4
    g = torch.Generator(device="cuda").manual_seed(5)
    x, w, dy = (torch.randn(s, generator=g, device="cuda").to(torch.float16) for s in ((m, k), (n, k), (m, n)))
    w = w * 0.25
    b = torch.randn(n, generator=g, device="cuda").to(torch.float16)
    z = ref.linear(x, w, b)[1].to(torch.float16)
    if name == "relu":  # away from its corner
        z = torch.where(z.abs() < 0.05, torch.full_like(z, 0.05), z)
    got = oz.oz2_linear_grad(dy, x, w, pre=z, act=name)
    want, bounds, _ = ref.grad(dy, x, w, z, name)
    Z, DY = z.to(ref.D), dy.to(ref.D)
    X, W = x.to(ref.D), w.to(ref.D)
    for i in range(3):
        d = torch.randn(got[i].shape, generator=g, device="cuda", dtype=ref.D)
        change = d @ W.t() if i == 0 else X @ d.t() if i == 1 else d.expand(m, n)  # of z
        change, scale = change / change.abs().max(), change.abs().max()
        loss = lambda t: (DY * ref.act(Z + t * change, name)).sum()  # noqa: E731
        numeric = (loss(h) - loss(-h)) / (2 * h) * scale
        ours = (got[i].to(ref.D) * d).sum()
        bound = (bounds[i] * d.abs()).sum() + scale * (h * h * 4 * DY.abs().sum() + 1e-16 / h * 20 * DY.abs().sum())
        assert abs(ours - numeric) <= bound, (i, ours.item(), numeric.item(), bound.item())


def test_on_another_stream_and_in_a_graph(env):
    oz, torch = env
    dy, x, w, z = make(torch, 129, 203, 77, torch.bfloat16, seed=6)
    want = oz.oz2_linear_grad(dy, x, w, pre=z, act="silu")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = oz.oz2_linear_grad(dy, x, w, pre=z, act="silu")
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    outs = [torch.empty_like(t) for t in want]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        oz.oz2_linear_grad(dy, x, w, pre=z, act="silu", dx=outs[0], dw=outs[1], db=outs[2])
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_accumulation_with_split_depths(env):
    """Many tokens into small weights: the parts of the depth and what was there."""
    oz, torch = env
    m, n, k = 16384, 512, 300
    dy, x, w, _ = make(torch, m, n, k, torch.bfloat16, seed=7)
    want, (_, _, bb), ew = ref.grad(dy, x, w, None, "none")
    dw, db = torch.full((n, k), 5.0, device="cuda"), torch.full((n,), 1.0, device="cuda")
    oz.oz2_linear_grad(dy, x, w, dw=dw, db=db, accumulate=True)
    ref.close(dw, want[1] + 5, ew + 2.0 ** -23 * (want[1].abs() + 5), "dw")
    ref.close(db, want[2] + 1, bb + 2.0 ** -23 * (want[2].abs() + 1), "db")


def test_db_of_many_rows(env):
    """One column block, rows beyond a cluster's: sums in a fixed order."""
    oz, torch = env
    for m, n in ((2048, 40), (2049, 40), (100000, 24), (3000, 1001)):
        dy = torch.randn(m, n, generator=torch.Generator(device="cuda").manual_seed(m), device="cuda").to(torch.float16)
        x, w = torch.zeros(m, 8, dtype=torch.float16, device="cuda"), torch.zeros(n, 8, dtype=torch.float16, device="cuda")
        db = oz.oz2_linear_grad(dy, x, w, need=("db",))[2]
        d = dy.double()
        ref.close(db, d.sum(0), (m / 8 + 16) * 2.0 ** -23 * d.abs().sum(0), (m, n))
        assert torch.equal(db, oz.oz2_linear_grad(dy, x, w, need=("db",))[2])


@pytest.mark.parametrize("shape", [(3400, 2504, 2504), (40, 72, 104)])
def test_rows_on_16_bytes_only(env, shape):
    """dY, X and W all on odd multiples of 16 bytes: the larger products take a copy of
    dY; either way the bits of the same values on whole lines."""
    oz, torch = env
    dy, x, w, _ = make(torch, *shape, torch.bfloat16, seed=8)

    def lined(t):
        return torch.nn.functional.pad(t, (0, -t.shape[1] % 64))[:, :t.shape[1]]

    assert all(t.stride(0) * 2 % 32 == 16 for t in (dy, x, w))
    want = oz.oz2_linear_grad(lined(dy), lined(x), lined(w))
    got = oz.oz2_linear_grad(dy, x, w)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    got = oz.oz2_linear_grad(dy, x, w, need=("dx", "dw"))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    (wx, ww, wb), (bx, bw, bb), _ = ref.grad(dy, x, w, None, "none")
    ref.close(want[0], wx, bx, "dx")
    ref.close(want[1], ww, bw, "dw")
    ref.close(want[2], wb, bb, "db")
