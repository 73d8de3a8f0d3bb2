"""oz2_linear against its formula in 64 bits."""
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


def make(torch, m, n, k, dtype, seed=0, pad=(0, 0)):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000 * seed + m + 3 * n + 7 * k)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    x, w = normal(m, k + pad[0]), normal(n, k + pad[1]) * max(k, 1) ** -0.5
    xs = ws = None
    if dtype == torch.float8_e4m3fn:
        x, xs = ref.e4m3_rows(x) if x.numel() else (x.to(dtype), normal(m))
        w, ws = ref.e4m3_rows(w) if w.numel() else (w.to(dtype), normal(n))
    else:
        x, w = x.to(dtype), w.to(dtype)
    return x[:, :k], w[:, :k], xs, ws, normal


SHAPES = [(1, 1, 1), (1, 128, 64), (2, 129, 63), (3, 4096, 4096), (8, 1000, 520), (16, 640, 16384), (17, 257, 130),
          (33, 96, 1032), (64, 2048, 512), (100, 300, 257), (128, 128, 128), (129, 255, 129), (256, 256, 256),
          (257, 513, 1027), (500, 64, 8192), (1000, 777, 1333), (1024, 2304, 640),
          (128, 4096, 4096), (300, 1024, 12288), (512, 4096, 16384), (2500, 3001, 500), (5000, 2600, 72), (4096, 4096, 200), (5000, 4200, 72)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind", ["bf16", "f16", "e4m3"])
def test_shapes(env, shape, kind):
    oz, torch = env
    dt = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}[kind]
    m, n, k = shape
    x, w, xs, ws, normal = make(torch, m, n, k, dt)
    out = torch.bfloat16 if kind == "e4m3" else dt
    name = ref.ACTS[(m + n + k) % 5]
    bias, r = normal(n).to(out), normal(m, n).to(out)
    y, z = oz.oz2_linear(x, w, bias=bias, act=name, residual=r, x_scale=xs, w_scale=ws, save_pre=True)
    wy, wz, by, bz = ref.linear(x, w, bias, name, r, xs, ws)
    ref.close(y, wy, by, "y")
    ref.close(z, wz, bz, "z")
    # Without its options, and again: the same bits.
    y0 = oz.oz2_linear(x, w, x_scale=xs, w_scale=ws)
    wy, _, by, _ = ref.linear(x, w, x_scale=xs, w_scale=ws)
    ref.close(y0, wy, by, "plain")
    assert torch.equal(y0, oz.oz2_linear(x, w, x_scale=xs, w_scale=ws))


@pytest.mark.parametrize("name", ref.ACTS)
@pytest.mark.parametrize("m", [1, 24, 300])
def test_activations_at_all_magnitudes(env, name, m):
    """z from bias alone (k = 0) and from products, tiny to huge."""
    oz, torch = env
    n = 777
    bias = torch.linspace(-12, 12, n, device="cuda")
    bias[:8] = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 300.0, -300.0, 60000.0, -60000.0])
    for dt in (torch.bfloat16, torch.float16):
        x, w = torch.zeros(m, 0, dtype=dt, device="cuda"), torch.zeros(n, 0, dtype=dt, device="cuda")
        y = oz.oz2_linear(x, w, bias=bias, act=name)
        wy, _, by, _ = ref.linear(x, w, bias, name, out=dt)
        ref.close(y, wy, by, "k = 0")
        x, w = torch.ones(m, 40, dtype=dt, device="cuda"), torch.zeros(n, 40, dtype=dt, device="cuda")
        w[:, 7] = bias.clamp(-200, 200).to(dt)
        y = oz.oz2_linear(x, w, act=name)
        wy, _, by, _ = ref.linear(x, w, None, name)
        ref.close(y, wy, by, "products")


@pytest.mark.parametrize("m,n,k", [(1, 300, 200), (20, 300, 200), (300, 300, 200), (300, 333, 201)])
def test_strided_operands_and_outputs(env, m, n, k):
    """Rows inside larger arrays, bases off the 16-byte grid, residual and out
    the same array; what lies beside the rows keeps its values."""
    oz, torch = env
    for pad in ((8, 16), (1, 3), (2, 5)):
        x, w, _, _, normal = make(torch, m, n, k, torch.bfloat16, seed=2, pad=pad)
        x, w = x[:, 1:], w[:, 1:]
        hold = normal(m, n + 2 * pad[0]).to(torch.bfloat16)
        keep = hold.clone()
        y = hold[:, pad[0]:pad[0] + n]
        r = keep[:, pad[0]:pad[0] + n]
        got = oz.oz2_linear(x, w, act="silu", residual=y, out=y)
        wy, _, by, _ = ref.linear(x, w, None, "silu", r)
        assert got.data_ptr() == y.data_ptr()
        ref.close(y, wy, by, "y")
        assert torch.equal(hold[:, :pad[0]], keep[:, :pad[0]]) and torch.equal(hold[:, pad[0] + n:], keep[:, pad[0] + n:])


@pytest.mark.parametrize("m,n,k", [(1, 256, 512), (20, 256, 512), (300, 256, 512)])
def test_nothing_outside_the_operands_matters(env, m, n, k):
    """NaN beside and behind the operands' rows and around the outputs."""
    oz, torch = env
    nan = float("nan")
    for dt in (torch.bfloat16, torch.float8_e4m3fn):
        x, w, xs, ws, _ = make(torch, m, n, k, dt, seed=3)
        k2 = k - 5
        X = torch.full((m + 1, k + 16), nan, device="cuda").to(dt)
        W = torch.full((n + 1, k + 16), nan, device="cuda").to(dt)
        X[:m, :k2], W[:n, :k2] = x[:, :k2], w[:, :k2]
        y = oz.oz2_linear(X[:m, :k2], W[:n, :k2], x_scale=xs, w_scale=ws)
        wy, _, by, _ = ref.linear(x[:, :k2], w[:, :k2], x_scale=xs, w_scale=ws)
        ref.close(y, wy, by)


@pytest.mark.parametrize("m", [1, 5, 200])
def test_non_finite_values_stay_in_their_rows(env, m):
    oz, torch = env
    n, k = 260, 192
    x, w, _, _, _ = make(torch, m, n, k, torch.float16, seed=4)
    w[7, 3] = float("nan")
    w[9, 5] = float("inf")
    x[:, 5] = 1.0
    y = oz.oz2_linear(x, w)
    assert torch.isnan(y[:, 7]).all()
    assert torch.isposinf(y[:, 9]).all()
    y[:, 7] = y[:, 9] = 0
    assert torch.isfinite(y).all()
    assert torch.isnan(oz.oz2_linear(x, w, act="relu")[:, 7]).all()


def test_empty_problems(env):
    oz, torch = env
    bf = torch.bfloat16
    e = lambda *s: torch.empty(s, dtype=bf, device="cuda")  # noqa: E731
    assert oz.oz2_linear(e(0, 64), e(32, 64)).shape == (0, 32)
    assert oz.oz2_linear(e(5, 64), e(0, 64)).shape == (5, 0)
    assert torch.equal(oz.oz2_linear(e(5, 0), e(9, 0)), torch.zeros(5, 9, dtype=bf, device="cuda"))


def test_e4m3_without_scales_and_with_f16_results(env):
    oz, torch = env
    x, w, _, _, normal = make(torch, 70, 90, 300, torch.float8_e4m3fn, seed=5)
    x, w = (x.float() / 64).to(x.dtype), (w.float() / 64).to(w.dtype)
    y = oz.oz2_linear(x, w, out_dtype=torch.float16)
    wy, _, by, _ = ref.linear(x, w, out=torch.float16)
    ref.close(y, wy, by)


def test_zero_tokens_and_zero_scales(env):
    """Padding tokens: rows of zeros, with a scale of zero."""
    oz, torch = env
    x, w, xs, ws, normal = make(torch, 40, 90, 300, torch.float8_e4m3fn, seed=6)
    x[10:20] = 0
    xs[10:20] = 0
    b = normal(90)
    y = oz.oz2_linear(x, w, bias=b, x_scale=xs, w_scale=ws)
    assert torch.equal(y[10:20], b.to(torch.bfloat16).expand(10, 90))


def test_on_another_stream_and_in_a_graph(env):
    oz, torch = env
    x, w, _, _, normal = make(torch, 37, 515, 333, torch.bfloat16, seed=7)
    want = oz.oz2_linear(x, w, act="gelu")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = oz.oz2_linear(x, w, act="gelu")
    s.synchronize()
    assert torch.equal(got, want)
    out = torch.empty_like(want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        oz.oz2_linear(x, w, act="gelu", out=out)
    x2 = normal(37, 333).to(torch.bfloat16)
    x.copy_(x2)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, oz.oz2_linear(x2, w, act="gelu"))


def test_offsets_beyond_32_bits(env):
    """A token array and a result of more than 2^31 elements' extent."""
    oz, torch = env
    m, n, k = 3, 136, 128
    ld = (1 << 30) + 64
    big = torch.empty(2 * ld + k + n, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(8)
    xs = torch.randn(m, k, generator=g, device="cuda").to(torch.bfloat16)
    w = torch.randn(n, k, generator=g, device="cuda").to(torch.bfloat16)
    x = big.as_strided((m, k), (ld, 1), 0)
    y = big.as_strided((m, n), (ld, 1), k)
    x.copy_(xs)
    oz.oz2_linear(x, w, out=y)
    wy, _, by, _ = ref.linear(xs, w)
    ref.close(y, wy, by)


@pytest.mark.parametrize("m,n,k", [(1, 4096, 4096), (7, 640, 8192), (40, 4672, 6016), (16, 16384, 8192), (200, 2048, 2048),
                                   (512, 4096, 16384), (3000, 2500, 512), (9, 8200, 64), (1000, 72, 4000)])
def test_calls_repeat_bit_for_bit_beside_others(env, m, n, k):
    """Each way that a product runs (few rows, many, split depths): the same bits
    alone, and while other products run on another stream."""
    oz, torch = env
    x, w, _, _, normal = make(torch, m, n, k, torch.bfloat16, seed=9)
    b = normal(n)
    want = oz.oz2_linear(x, w, bias=b, act="silu")
    x2, w2, _, _, _ = make(torch, 700, 900, 1100, torch.bfloat16, seed=10)
    other = oz.oz2_linear(x2, w2, act="gelu")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got, beside = [], []
    for _ in range(4):
        with torch.cuda.stream(s):
            beside.append(oz.oz2_linear(x2, w2, act="gelu"))
        got.append(oz.oz2_linear(x, w, bias=b, act="silu"))
    torch.cuda.synchronize()
    assert all(torch.equal(a, want) for a in got) and all(torch.equal(a, other) for a in beside)


def test_a_given_stream_owns_the_outputs(env):
    """Outputs of a call on another stream come from that stream's memory: freed at
    once and allocated again there, they are not handed to the current stream."""
    oz, torch = env
    x, w, _, _, _ = make(torch, 300, 200, 100, torch.bfloat16, seed=11)
    dy = torch.ones(300, 200, dtype=torch.bfloat16, device="cuda")
    want = oz.oz2_linear(x, w, act="silu"), oz.oz2_linear_grad(dy, x, w)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = oz.oz2_linear(x, w, act="silu", stream=s), oz.oz2_linear_grad(dy, x, w, stream=s)
    at = got[0].data_ptr()
    s.synchronize()
    assert torch.equal(got[0], want[0]) and all(torch.equal(a, b) for a, b in zip(got[1], want[1]))
    del got
    with torch.cuda.stream(s):
        again = [torch.empty(300, 200, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    assert at in [t.data_ptr() for t in again]


@pytest.mark.parametrize("kind, shape", [("bf16", (2000, 5000, 4104)), ("f16", (5000, 2100, 4104)),
                                         ("e4m3", (4200, 5000, 4112)), ("bf16", (40, 96, 1032))])
def test_rows_on_16_bytes_only(env, kind, shape):
    """Both operands' rows on odd multiples of 16 bytes: the larger products copy one
    of them; either way the bits of the same values on whole lines."""
    oz, torch = env
    dt = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}[kind]
    x, w, xs, ws, _ = make(torch, *shape, dt, seed=12)
    es = x.element_size()

    def lined(t):
        """The same values on rows of whole 128-byte lines."""
        rows = torch.zeros(t.shape[0], -(-t.shape[1] * es // 128) * 128, dtype=torch.uint8, device="cuda")
        rows[:, :t.shape[1] * es] = t.contiguous().view(torch.uint8)
        return rows.view(dt)[:, :t.shape[1]]

    assert x.stride(0) * es % 32 == 16 and w.stride(0) * es % 32 == 16
    want = oz.oz2_linear(lined(x), lined(w), x_scale=xs, w_scale=ws, act="relu")
    assert torch.equal(oz.oz2_linear(x, w, x_scale=xs, w_scale=ws, act="relu"), want)
    wy, _, by, _ = ref.linear(x, w, None, "relu", None, xs, ws)
    ref.close(want, wy, by, shape)


@pytest.mark.parametrize("m, n, k, pad", [(2500, 3001, 200, 0), (2500, 3002, 64, 0), (4099, 2048, 300, 3), (600, 9000, 1024, 1)])
def test_large_results_in_place_of_unaligned_residuals(env, m, n, k, pad):
    """Tiles whose residual is fetched value by value, ahead of the stores over it."""
    oz, torch = env
    x, w, _, _, normal = make(torch, m, n, k, torch.bfloat16, seed=13)
    hold = normal(m, n + pad).to(torch.bfloat16)
    r = hold[:, pad:].clone()
    y = hold[:, pad:]
    beside = hold[:, :pad].clone()
    want, z = oz.oz2_linear(x, w, act="gelu_tanh", residual=r, save_pre=True)
    oz.oz2_linear(x, w, act="gelu_tanh", residual=y, out=y)
    assert torch.equal(y, want) and torch.equal(hold[:, :pad], beside)
    wy, wz, by, bz = ref.linear(x, w, None, "gelu_tanh", r)
    ref.close(y, wy, by, "y")
    ref.close(z, wz, bz, "z")


@pytest.mark.parametrize("kind", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("m, n, k", [(1, 1, 3), (1, 4096, 4097), (3, 15, 31), (7, 17, 33), (8, 333, 395), (9, 100, 2049),
                                     (16, 64, 16383), (13, 2001, 1000 + 3), (2, 5000, 257), (16, 16384, 101), (5, 40, 8191)])
def test_few_tokens_and_unaligned_weights(env, kind, m, n, k):
    """Weights that are read where they lie: depths that end inside a piece, deep and
    narrow ones, NaN around the rows, residuals in place."""
    oz, torch = env
    dt = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}[kind]
    out = torch.bfloat16 if kind == "e4m3" else dt
    x, w, xs, ws, normal = make(torch, m, n, k, dt, seed=14)
    bias, r = normal(n), normal(m, n).to(out)
    name = ref.ACTS[(m + n + k) % 5]
    wy, wz, by, bz = ref.linear(x, w, bias, name, r, xs, ws)

    def inside_nan(t, left):
        held = torch.full((t.shape[0] + 2, t.shape[1] + left + 2), float("nan"), device="cuda").to(dt)
        held[1:-1, left:left + t.shape[1]] = t
        return held[1:-1, left:left + t.shape[1]]

    for left in (0, 1, 5):
        X, W = inside_nan(x, left), inside_nan(w, left + 1)
        y, z = oz.oz2_linear(X, W, bias=bias, act=name, residual=r, x_scale=xs, w_scale=ws, save_pre=True)
        ref.close(y, wy, by, ("y", left))
        ref.close(z, wz, bz, ("z", left))
        held = r.clone()
        oz.oz2_linear(X, W, bias=bias, act=name, residual=held, out=held, x_scale=xs, w_scale=ws)
        assert torch.equal(held, y)
        again = oz.oz2_linear(X, W, bias=bias, act=name, residual=r, x_scale=xs, w_scale=ws)
        assert torch.equal(again, y)
