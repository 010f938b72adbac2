"""Rows that no group lists, rows outside all segments and the padding behind rows: whatever they hold, the results are the same bits, and they stay as they are.
The first and the last row are among them, which tiles fetch in place of rows that they have not."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2305_09887_amd import binding
    binding.lib()
    return binding


def rows(n, F, dtype, g, spare):
    """[n, F] in rows with `spare` elements of padding behind each"""
    return torch.randn((n, F + spare), generator=g).to(dtype).cuda()[:, :F]


def poisoned(x, free, value):
    whole = x.new_empty((x.shape[0], x.stride(0))).fill_(value)
    out = whole[:, :x.shape[1]]
    out.copy_(x)
    out[free] = value
    return out


# a few rows a group, tiles of 64 rows, weights in LDS; widths that end in whole pieces and that do not
@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes,F_in,F_out", [([2, 1, 0, 1], 40, 24), ([2, 1, 1], 37, 21), ([90, 0, 31], 64, 96), ([90, 0, 31], 65, 101), ([200_000, 7], 128, 64),
                                              ([200_000, 7], 43, 77)])
def test_grouped_dense(B, sizes, F_in, F_out, dtype, act):
    g = torch.Generator().manual_seed(F_in)
    m, E = sum(sizes), len(sizes)
    n = m + 6
    middle = torch.randperm(n - 2, generator=g) + 1
    listed, free = middle[:m], torch.cat([middle[m:], torch.tensor([0, n - 1])])
    order = torch.cat([listed, torch.zeros(n - m, dtype=torch.long)]).int().cuda()
    offsets = torch.tensor([0] + sizes).cumsum(0).int().cuda()
    X, Y, dY = (rows(n, F, dtype, g, 3 if F % 2 else 4) for F in (F_in, F_out, F_out))
    W, b = torch.randn((E, F_in, F_out), generator=g).cuda(), torch.randn((E, F_out), generator=g).cuda()
    free, listed = free.cuda(), listed.cuda()

    def results(X, Y, dY):
        out, dX = torch.full((n, F_out), 7.0, dtype=dtype, device="cuda"), torch.full((n, F_in), 7.0, dtype=dtype, device="cuda")
        B.tma_grouped_dense_fwd(X, W, b, offsets, act, order=order, Y_out=out)
        dW, db, _ = B.tma_grouped_dense_bwd(X, Y, dY, W, offsets, act, order=order, dX_out=dX)
        assert (out[free] == 7).all() and (dX[free] == 7).all()
        return out, dX, dW, db

    want = results(X, Y, dY)
    assert all(torch.isfinite(t).all() for t in want)
    for value in (NAN, INF, -INF):
        got = results(*(poisoned(t, free, value) for t in (X, Y, dY)))
        assert all(torch.equal(a, c) for a, c in zip(got, want)), value


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("edges", [[3, 90, 90, 800], [17, 20], [1, 30_000]])
@pytest.mark.parametrize("G,cg", [(4, 8), (3, 5), (2, 700)])
def test_group_norm_over_segments(B, edges, G, cg, dtype):
    g = torch.Generator().manual_seed(edges[0])
    if cg > 100 and edges[-1] > 1000:
        edges = [1, 2_000]
    n, F = edges[-1] + 5, G * cg
    free = torch.cat([torch.arange(edges[0]), torch.arange(edges[-1], n)]).cuda()
    X, dY = rows(n, F, dtype, g, 3 if F % 2 else 8), rows(n, F, dtype, g, 3 if F % 2 else 8)
    gamma, beta = torch.rand(F, generator=g).cuda(), torch.randn(F, generator=g).cuda()
    segments = torch.tensor(edges, dtype=torch.int32, device="cuda")

    def results(X, dY):
        out, dX = torch.full((n, F), 7.0, dtype=dtype, device="cuda"), torch.full((n, F), 7.0, dtype=dtype, device="cuda")
        _, stats = B.tma_groupnorm_act_fwd(X, G, gamma, beta, B.TMA_ACT_SILU, segments=segments, out=out)
        _, dga, dbe, _ = B.tma_groupnorm_act_bwd(X, dY, G, gamma, beta, B.TMA_ACT_SILU, segments=segments, stats=stats, dX_out=dX)
        assert (out[free] == 7).all() and (dX[free] == 7).all()
        return out, stats, dX, dga, dbe

    want = results(X, dY)
    assert all(torch.isfinite(t).all() for t in want)
    for value in (NAN, INF, -INF):
        got = results(poisoned(X, free, value), poisoned(dY, free, value))
        assert all(torch.equal(a, c) for a, c in zip(got, want)), value
