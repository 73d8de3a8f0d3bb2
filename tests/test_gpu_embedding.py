"""oz2_embedding and oz2_embedding_grad against their formulas in 64 bits."""
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


def tokens(g, m, n, kind="zipf", dtype=torch.int64):
    if kind == "one":
        ids = torch.full((m,), n - 1, device="cuda", dtype=torch.float64)
    elif kind == "even":
        ids = torch.rand(m, generator=g, device="cuda", dtype=torch.float64) * n
    else:
        ids = torch.exp(torch.rand(m, generator=g, device="cuda", dtype=torch.float64) * torch.log(torch.tensor(n + 1.0))) - 1
    return ids.long().clamp(0, n - 1).to(dtype)


def view(t, how):
    """The same values off the 16-byte grid, or in rows of their own stride."""
    if how == "whole":
        return t
    pad = torch.zeros(t.shape[0], t.shape[1] + (3 if how == "odd" else 8), dtype=t.dtype, device="cuda")
    at = 1 if how == "odd" else 0
    pad[:, at:at + t.shape[1]] = t
    return pad[:, at:at + t.shape[1]]


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("m,n,k,how", [
    (1, 1, 1, "whole"), (1, 7, 8, "whole"), (5, 64, 16, "whole"), (64, 1000, 4096, "whole"), (33, 100, 777, "whole"),
    (300, 50, 129, "odd"), (257, 513, 264, "strided"), (4000, 3000, 96, "whole"), (3, 9, 20001, "whole"), (70, 9, 5, "odd")])
def test_forward(oz, dt, m, n, k, how):
    g = rng(m + n + k)
    table = view(torch.randn(n, k, generator=g, device="cuda").to(dt), how)
    ids = tokens(g, m, n, dtype=torch.int32 if m % 2 else torch.int64)
    for scale in (1.0, 0.5, 32.0):
        y, e = ref.embedding(ids, table, scale)
        close(oz.oz2_embedding(ids, table, scale=scale), y, e, "y")


def test_forward_padding_and_beyond(oz):
    """Negative ids are zeros, ids of n or more NaN, whatever the table holds."""
    table = torch.full((4, 40), float("inf"), device="cuda").bfloat16()
    table[2] = 3.0
    ids = torch.tensor([2, -1, 4, -100, 2, 1 << 40, -(1 << 40)], device="cuda")
    y = oz.oz2_embedding(ids, table)
    assert (y[0] == 3).all() and (y[4] == 3).all() and not y[[1, 3, 6]].any() and y[[2, 5]].isnan().all()
    for scale in (float("inf"), float("nan")):
        y = oz.oz2_embedding(ids, table, scale=scale)
        assert not y[[1, 3, 6]].any() and not y[[0, 2, 4, 5]].isfinite().any()
    assert oz.oz2_embedding(ids[:0], table).shape == (0, 40)
    assert oz.oz2_embedding(torch.tensor([0, -1], device="cuda"), table[:0])[0].isnan().all()


def test_forward_into_a_part(oz):
    """`out` of its own stride: what lies beside it is left as it was."""
    g = rng(1)
    table = torch.randn(50, 100, generator=g, device="cuda").half()
    ids = tokens(g, 30, 50)
    for off in (0, 1, 8):
        whole = torch.full((32, 128), 7.0, device="cuda").half()
        oz.oz2_embedding(ids, table, out=whole[1:31, off:off + 100])
        assert torch.equal(whole[1:31, off:off + 100], table[ids])
        whole[1:31, off:off + 100] = 7
        assert (whole == 7).all()


def test_forward_offsets_pass_32_bits(oz):
    """A table of 2^32 elements and more: its last rows."""
    n, k = (1 << 21) + 5, 2048
    table = torch.empty(n, k, dtype=torch.bfloat16, device="cuda")
    table[-3:] = torch.randn(3, k, device="cuda").bfloat16()
    ids = torch.tensor([n - 1, n - 3, n - 2], device="cuda")
    assert torch.equal(oz.oz2_embedding(ids, table), table[ids])
    dy = torch.randn(3, k, device="cuda").bfloat16()
    table[-4:] = 0
    oz.oz2_embedding_grad(dy, ids, n, out=table, accumulate=True)
    assert torch.equal(table[ids], dy) and not table[-4].any()


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("kind", ["zipf", "even", "one"])
@pytest.mark.parametrize("m,n,k,how", [
    (1, 1, 1, "whole"), (5, 7, 8, "whole"), (31, 40, 33, "odd"), (100, 3, 264, "strided"), (255, 9000, 16, "odd"),
    (256, 300, 4100, "whole"), (257, 300, 4100, "whole"), (200, 131071, 24, "strided"), (300, 511, 64, "whole"),
    (1000, 512, 777, "whole"), (2049, 70000, 40, "whole"), (5000, 131071, 16, "whole"), (20000, 600, 24, "odd")])
def test_gradient(oz, dt, kind, m, n, k, how):
    g = rng(m + n + k)
    dy = view(torch.randn(m, k, generator=g, device="cuda").to(dt), how)
    ids = tokens(g, m, n, kind, torch.int32 if m % 2 else torch.int64)
    ids[torch.rand(m, generator=g, device="cuda") < 0.1] = -1
    if m > 20:
        ids[m // 2] = n
    for scale, out in ((1.0, dt), (0.5, torch.float32)):
        s, e = ref.embedding_grad(dy, ids, n, scale, out)
        got = oz.oz2_embedding_grad(dy, ids, n, scale=scale, out_dtype=out)
        assert got.dtype == out
        close(got, s, e, "dE")
        assert torch.equal(got, oz.oz2_embedding_grad(dy, ids, n, scale=scale, out_dtype=out))  # one order
        old = view(torch.randn(n, k, generator=g, device="cuda").to(out), how)
        whole = old.clone()
        s, e = ref.embedding_grad(dy, ids, n, scale, out, old)
        assert oz.oz2_embedding_grad(dy, ids, n, scale=scale, out=old, accumulate=True) is old
        close(old, s, e, "added to")
        hit = torch.zeros(n + 1, dtype=torch.bool, device="cuda")
        hit[ids.long().clamp(0, n)[ids >= 0]] = True
        assert torch.equal(old[~hit[:n]], whole[~hit[:n]])  # rows without tokens: left as they were


@pytest.mark.parametrize("m", [15, 16, 17, 31, 32, 33, 48, 49, 64, 65, 130, 200])
def test_runs_at_the_chunks_ends(oz, m):
    """Runs of every length around those that are cut, starting anywhere in a chunk."""
    g = rng(m)
    for lead in (0, 1, 15, 16, 17, 31, 32, 40):
        ids = torch.cat([torch.zeros(lead, dtype=torch.int64), torch.ones(m, dtype=torch.int64),
                         torch.full((5,), 2), torch.full((m + 1,), 5)]).cuda()
        ids = ids[torch.randperm(len(ids), generator=g, device="cuda")]
        dy = torch.randn(len(ids), 72, generator=g, device="cuda")
        s, e = ref.embedding_grad(dy, ids, 6, 1.0, torch.float32)
        close(oz.oz2_embedding_grad(dy, ids, 6), s, e, f"lead {lead}")


def test_gradient_nothing_to_do(oz):
    dy = torch.ones(4, 8, device="cuda")
    none = torch.full((4,), -1, device="cuda")
    assert not oz.oz2_embedding_grad(dy, none, 5).any()
    assert not oz.oz2_embedding_grad(dy[:0], none[:0], 5).any()
    old = torch.ones(5, 8, device="cuda")
    assert (oz.oz2_embedding_grad(dy, none, 5, out=old, accumulate=True) == 1).all()
    assert (oz.oz2_embedding_grad(dy[:0], none[:0], 5, out=old, accumulate=True) == 1).all()
    assert oz.oz2_embedding_grad(dy, none, 0).shape == (0, 8)


@pytest.mark.parametrize("m", [40, 400])
def test_nan_stays_with_its_row(oz, m):
    dy = torch.ones(m, 16, device="cuda")
    dy[3] = float("nan")
    dy[7] = float("inf")
    ids = torch.arange(m, device="cuda") % (m // 2)
    ids[9] = -1
    dy[9] = float("nan")
    got = oz.oz2_embedding_grad(dy, ids, m)
    assert got[3].isnan().all() and got[7].isinf().all()
    keep = torch.ones(m, dtype=torch.bool, device="cuda")
    keep[[3, 7]] = False
    assert got[keep].isfinite().all() and (got[9] == 1).all()


def test_forward_and_gradient_are_adjoint(oz):
    """<E[ids], dY> = <E, dE>, and a difference along one entry gives its gradient."""
    g = rng(4)
    table, ids = torch.randn(30, 24, generator=g, device="cuda"), tokens(g, 200, 30)
    dy = torch.randn(200, 24, generator=g, device="cuda")
    grad = oz.oz2_embedding_grad(dy, ids, 30, scale=0.5)
    y = oz.oz2_embedding(ids, table, scale=0.5)
    left, right = (y.double() * dy.double()).sum(), (table.double() * grad.double()).sum()
    assert abs(left - right) < 200 * 24 * 300 * 2 ** -24
    table[2, 3] += 1
    got = ((oz.oz2_embedding(ids, table, scale=0.5) - y).double() * dy.double()).sum()
    assert abs(got - grad[2, 3].double()) < 1e-4


def test_streams_and_graphs(oz):
    """Calls on two streams at once, captured ones, and replays on other inputs."""
    g = rng(5)
    n, k = 3000, 200
    dy = torch.randn(4000, k, generator=g, device="cuda").bfloat16()
    a, b = tokens(g, 4000, n), tokens(g, 4000, n, "even")
    want = [oz.oz2_embedding_grad(dy, t, n) for t in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[oz.oz2_embedding_grad(dy, t, n, stream=s) for t, s in zip((a, b), streams)] for _ in range(5)]
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for r in got for x, y in zip(r, want))
    ids, out = a.clone(), torch.empty_like(want[0])
    y = torch.empty_like(dy)
    graphs = []
    for _ in range(2):  # two captured graphs
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            oz.oz2_embedding_grad(dy, ids, n, out=out)
            oz.oz2_embedding(ids, out, out=y)
        graphs.append(graph)
    for t, w in zip((b, a, b), (want[1], want[0], want[1])):
        ids.copy_(t)
        for graph in graphs:
            out.fill_(5)
            graph.replay()
            assert torch.equal(out, w) and torch.equal(y, w[t])


def test_current_stream_is_used(oz):
    s = torch.cuda.Stream()
    table = torch.zeros(8, 64, device="cuda")
    ids = torch.arange(8, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        table.fill_(2)
        y = oz.oz2_embedding(ids, table)
        d = oz.oz2_embedding_grad(y, ids, 8)
    s.synchronize()
    assert (y == 2).all() and (d == 2).all()


@pytest.mark.parametrize("m", [2048, 2049, 3001, 4096, 8191, 8192, 8193, 16385, 65535, 65537, 140001])
@pytest.mark.parametrize("n", [3, 700, 70001])
def test_sorts_of_all_sizes(oz, m, n):
    """By one block, a cluster of 8 and one of 16; a block's pairs in shared memory (up to 4096) or
    written where they belong; a warp's stretch held (up to 256) or read twice."""
    g = rng(m + n)
    ids = tokens(g, m, n, "zipf" if m % 2 else "even")
    ids[torch.rand(m, generator=g, device="cuda") < 0.05] = -1
    dy = torch.randn(m, 24, generator=g, device="cuda")
    s, e = ref.embedding_grad(dy, ids, n, 1.0, torch.float32)
    got = oz.oz2_embedding_grad(dy, ids, n)
    close(got, s, e, "dE")
    assert torch.equal(got, oz.oz2_embedding_grad(dy, ids, n))


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("k,how", [(200, "whole"), (203, "odd"), (264, "whole"), (520, "strided"), (520, "odd"), (777, "odd"),
                                   (2100, "whole"), (2101, "odd")])
@pytest.mark.parametrize("kind", ["zipf", "even", "one"])
def test_several_pieces_a_lane(oz, dt, kind, k, how):
    """So many tokens that a lane has two or four pieces of a row (from 256 columns of 16 bits on, 128
    and 256 of 32), of one slice or several; short and long runs, stored and added to."""
    m, n = 60000, 20000
    assert (m + 15) // 16 >= 24 * 152
    g = rng(k)
    dy = view(torch.randn(m, k, generator=g, device="cuda").to(dt), how)
    ids = tokens(g, m, n, kind)
    if kind == "zipf":
        ids[torch.rand(m, generator=g, device="cuda") < 0.1] = -1
        ids[m // 2] = n
    for out in {dt, torch.float32}:
        s, e = ref.embedding_grad(dy, ids, n, 0.5, out)
        got = oz.oz2_embedding_grad(dy, ids, n, scale=0.5, out_dtype=out)
        close(got, s, e, "dE")
        assert torch.equal(got, oz.oz2_embedding_grad(dy, ids, n, scale=0.5, out_dtype=out))
        old = view(torch.randn(n, k, generator=g, device="cuda").to(out), how)
        s, e = ref.embedding_grad(dy, ids, n, 0.5, out, old)
        oz.oz2_embedding_grad(dy, ids, n, scale=0.5, out=old, accumulate=True)
        close(old, s, e, "added to")


@pytest.mark.parametrize("m", [1, 2, 14, 15, 16, 17, 18, 31, 32, 33, 47, 48, 49, 64, 65, 130, 200])
@pytest.mark.parametrize("dt,k", [(torch.float32, 72), (torch.bfloat16, 33)])
def test_runs_around_the_cut_at_any_place(oz, m, dt, k):
    """Runs as long as those that are cut, and one less and more, starting at every place of a chunk
    of 16 sorted pairs; what follows brings the tokens over those that are not sorted (256)."""
    g = rng(m)
    for lead in list(range(18)) + [30, 31, 32, 33, 40]:
        ids = torch.cat([torch.zeros(lead, dtype=torch.int64), torch.ones(m, dtype=torch.int64),
                         torch.full((5,), 2), torch.full((m + 1,), 5), torch.arange(6, 306)]).cuda()
        assert len(ids) > 256
        ids = ids[torch.randperm(len(ids), generator=g, device="cuda")]
        dy = torch.randn(len(ids), k, generator=g, device="cuda").to(dt)
        s, e = ref.embedding_grad(dy, ids, 306, 1.0, dt)
        close(oz.oz2_embedding_grad(dy, ids, 306), s, e, f"lead {lead}")
        old = torch.randn(306, k, generator=g, device="cuda").to(dt)
        s, e = ref.embedding_grad(dy, ids, 306, 1.0, dt, old)
        close(oz.oz2_embedding_grad(dy, ids, 306, out=old, accumulate=True), s, e, f"lead {lead}, added to")
