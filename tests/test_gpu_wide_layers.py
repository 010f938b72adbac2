"""Gated dense layers and dense layers with a residual against plain fp64 forms of their formulas.

Small whole numbers are exact in every step (their products' sums stay below 2^24), so with them results have to be the reference's, rounded once: any
misplaced, lost or doubled term shows.  Normal values are compared element by element with a bound from the roundings that the calls are allowed:
u_s = 2^-8 of bf16 storage (2^-24 of fp32) for each result and, with bf16, each weight; fp32 sums of K terms K 2^-24 of the sum of magnitudes."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16]


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2305_09887_amd import binding
    binding.lib()
    return binding


def _buffer(values, dtype, pitch, offset=0, fill=math.nan):
    """`values` as rows `pitch` elements apart, `offset` elements into a buffer filled with something else."""
    n, w = values.shape
    flat = torch.full((max(n, 1) * pitch + offset + 16,), fill, dtype=dtype, device="cuda")
    t = flat[offset:offset + max(n, 1) * pitch].view(max(n, 1), pitch)[:n, :w]
    t.copy_(values.to(dtype))
    return t, flat


def _untouched(flat, t, fill):
    """Whether all of `flat` outside the rows of `t` is still `fill`."""
    mask = torch.ones_like(flat, dtype=torch.bool)
    n, w = t.shape
    off = t.storage_offset()
    for_rows = mask[off:off + max(n, 1) * t.stride(0)] if n else mask[:0]
    if n:
        for_rows.view(n, t.stride(0))[:, :w] = False
    return bool((flat[mask] == fill).all())


def _whole(g, *shape, top=3):
    return torch.randint(-top, top + 1, shape, generator=g).double()


def _act(name, z):
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2))
    return z.clamp(min=0) if name == "relu" else z


def _slope(name, z):
    if name == "silu":
        t = torch.sigmoid(z)
        return t * (1 + z * (1 - t))
    if name == "gelu":
        return 0.5 * torch.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return (z > 0).double() if name == "relu" else torch.ones_like(z)


def _code(B, name):
    return {"none": B.TMA_ACT_NONE, "relu": B.TMA_ACT_RELU, "silu": B.TMA_ACT_SILU, "gelu": B.TMA_ACT_GELU}[name]


# (n, F_in, F_out, pitch beyond the width, offset into the buffer): one row, units and tiles that end inside, rows that begin anywhere
SHAPES = [(1, 1, 1, 0, 0), (1, 17, 33, 0, 0), (2, 64, 32, 0, 0), (5, 16, 100, 4, 0), (16, 31, 48, 0, 0), (17, 64, 20, 0, 0), (31, 33, 31, 3, 1), (32, 1030, 16, 2, 2), (64, 600, 50, 0, 0), (65, 600, 50, 0, 0), (33, 100, 47, 0, 0), (70, 8, 130, 8, 8),
          (127, 129, 65, 1, 3), (128, 128, 128, 0, 0), (300, 96, 300, 4, 4), (257, 513, 255, 0, 0), (1030, 40, 72, 0, 0)]


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_gated_whole_numbers(B, shape, act, dtype):
    n, fi, fo, more, off = shape
    g = torch.Generator().manual_seed(fi * 1000 + fo)
    X, Wg, Wu, bg, bu = _whole(g, n, fi), _whole(g, fi, fo), _whole(g, fi, fo), _whole(g, fo), _whole(g, fo)
    G, U = X @ Wg + bg, X @ Wu + bu
    x, _ = _buffer(X, dtype, fi + more, off)
    outs = [_buffer(torch.zeros(n, fo), dtype, fo + more, off, fill=7.0) for _ in range(3)]
    d = lambda t: t.float().cuda()
    h, gg, uu = B.tma_gated_dense_fwd(x, d(Wg), d(Wu), d(bg), d(bu), _code(B, act), G_out=outs[1][0], U_out=outs[2][0], H_out=outs[0][0])
    want = _act(act, G) * U
    for got, w, (t, flat) in zip((h, gg, uu), (want, G, U), outs):
        assert torch.equal(got.cpu(), w.float().to(dtype))       # (below 2^24: exact in fp32)
        assert _untouched(flat, t, 7.0)
    alone, none_g, none_u = B.tma_gated_dense_fwd(x, d(Wg), d(Wu), None, d(bu), _code(B, act), save=False)
    assert none_g is None and none_u is None and torch.equal(alone.cpu(), (_act(act, X @ Wg) * U).float().to(dtype))

    G, U, dH, R = _whole(g, n, fo, top=2), _whole(g, n, fo, top=2), _whole(g, n, fo, top=2), _whole(g, n, fi)
    gg, uu, dh, r = (_buffer(t, dtype, t.shape[1] + more, off)[0] for t in (G, U, dH, R))
    dG, dU = dH * U * _slope(act, G), dH * _act(act, G)
    dx, flat = _buffer(torch.zeros(n, fi), dtype, fi + more, off, fill=7.0)
    got = B.tma_gated_dense_bwd(x, gg, uu, dh, d(Wg), d(Wu), _code(B, act), R=r, dX_out=dx)
    for t, w in zip(got[:4], (X.t() @ dG, X.t() @ dU, dG.sum(0), dU.sum(0))):
        assert torch.equal(t.cpu().double(), w)
    assert torch.equal(got[4].cpu(), (dG @ Wg.t() + dU @ Wu.t() + R).float().to(dtype)) and _untouched(flat, dx, 7.0)
    got = B.tma_gated_dense_bwd(x, gg, uu, dh, d(Wg), d(Wu), _code(B, act), need_dX=False, need_dbias=False)
    assert torch.equal(got[0].cpu().double(), X.t() @ dG) and got[2] is None and got[3] is None and got[4] is None


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_residual_whole_numbers(B, shape, act, dtype):
    n, fi, fo, more, off = shape
    g = torch.Generator().manual_seed(fi * 1000 + fo + 1)
    X, W, b, R = _whole(g, n, fi), _whole(g, fi, fo), _whole(g, fo), _whole(g, n, fo)
    Z = X @ W + b
    x, r = _buffer(X, dtype, fi + more, off)[0], _buffer(R, dtype, fo + more, off)[0]
    (z, z_flat), (y, y_flat) = (_buffer(torch.zeros(n, fo), dtype, fo + more, off, fill=7.0) for _ in range(2))
    d = lambda t: t.float().cuda()
    B.tma_dense_residual_fwd(x, d(W), d(b), _code(B, act), R=r, Z_out=z, Y_out=y)
    want = (_act(act, Z) + R).float().to(dtype)
    assert torch.equal(z.cpu(), Z.float().to(dtype)) and torch.equal(y.cpu(), want)
    assert _untouched(z_flat, z, 7.0) and _untouched(y_flat, y, 7.0)
    B.tma_dense_residual_fwd(x, d(W), d(b), _code(B, act), R=r, Y_out=r)          # in place
    assert torch.equal(r.cpu(), want)
    plain, none_z = B.tma_dense_residual_fwd(x, d(W), act=_code(B, act))
    assert none_z is None and torch.equal(plain.cpu(), _act(act, X @ W).float().to(dtype))

    Z, dY, R = _whole(g, n, fo), _whole(g, n, fo), _whole(g, n, fi)
    z, dy, r = (_buffer(t, dtype, t.shape[1] + more, off)[0] for t in (Z, dY, R))
    dZ = dY * _slope(act, Z)
    dx, flat = _buffer(torch.zeros(n, fi), dtype, fi + more, off, fill=7.0)
    dW, db, _ = B.tma_dense_residual_bwd(x, z if act != "none" else None, dy, d(W), _code(B, act), R=r, dX_out=dx)
    assert torch.equal(dW.cpu().double(), X.t() @ dZ) and torch.equal(db.cpu().double(), dZ.sum(0))
    want = (dZ @ W.t() + R).float().to(dtype)
    assert torch.equal(dx.cpu(), want) and _untouched(flat, dx, 7.0)
    B.tma_dense_residual_bwd(x, z, dy, d(W), _code(B, act), R=r, dX_out=r)          # in place
    assert torch.equal(r.cpu(), want)
    dW, db, dx = B.tma_dense_residual_bwd(x, z, dy, d(W), _code(B, act), need_dX=False, need_dbias=False)
    assert torch.equal(dW.cpu().double(), X.t() @ dZ) and db is None and dx is None


LIPSCHITZ = 1.13          # the steepest slope of silu is 1.0999, of gelu 1.1290
CURVE = 0.80              # the largest |act''|: of silu 1/2, of gelu 2 / sqrt(2 pi)


def _sum_bound(A, W, dtype, K):
    """Of a product's sums: its weights' roundings with bf16, fp32 sums of K terms and of the parts that they come in."""
    m = A.abs() @ W.abs()
    return m * ((2.0 ** -8 if dtype == torch.bfloat16 else 0.0) + (K + 16) * 2.0 ** -24)


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("n,fi,fo", [(1, 40, 70), (77, 130, 96), (400, 64, 258)])
def test_normal_values(B, n, fi, fo, act, dtype):
    g = torch.Generator().manual_seed(n)
    N = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)
    store = lambda t: t.to(dtype).double()
    u = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    X, R = store(N(n, fi)), store(N(n, fo))
    Wg, Wu, bg, bu = ((t / s).float().double() for t, s in ((N(fi, fo), fi ** 0.5), (N(fi, fo), fi ** 0.5), (N(fo), 4), (N(fo), 4)))
    d, s = lambda t: t.float().cuda(), lambda t: t.to(dtype).cuda()
    G, U = X @ Wg + bg, X @ Wu + bu
    eg, eu = _sum_bound(X, Wg, dtype, fi) + 2.0 ** -23 * G.abs(), _sum_bound(X, Wu, dtype, fi) + 2.0 ** -23 * U.abs()
    h, gg, uu = B.tma_gated_dense_fwd(s(X), d(Wg), d(Wu), d(bg), d(bu), _code(B, act))
    a = _act(act, G)
    # (the functions themselves: 2^-20 of z, which is more than their value's error)
    ea = LIPSCHITZ * eg + 2.0 ** -20 * G.abs()
    H, eh = a * U, ea * (U.abs() + eu) + a.abs() * eu + 2.0 ** -23 * (a * U).abs()
    for got, want, e in ((gg, G, eg), (uu, U, eu), (h, H, eh)):
        assert bool(((got.cpu().double() - want).abs() <= e + u * (want.abs() + e)).all())
    y, z = B.tma_dense_residual_fwd(s(X), d(Wg), d(bg), _code(B, act), R=s(R), save=True)
    want = a + R
    assert torch.equal(z, gg)
    assert bool(((y.cpu().double() - want).abs() <= ea + u * (want.abs() + ea) + 2.0 ** -23 * want.abs()).all())

    G, U, dH, R = store(N(n, fo)), store(N(n, fo)), store(N(n, fo) / n), store(N(n, fi) / n)
    a, slope = _act(act, G), _slope(act, G)
    dG, dU, dZ = dH * U * slope, dH * a, dH * slope
    small = 2.0 ** -19          # of the functions, and of the parts that a gradient is held in
    es = small * (1 + G.abs())
    got = B.tma_gated_dense_bwd(s(X), s(G), s(U), s(dH), d(Wg), d(Wu), _code(B, act), R=s(R))
    eG, eU, eZ = (dH * U).abs() * es + dG.abs() * 2.0 ** -16, dH.abs() * es + dU.abs() * 2.0 ** -16, dH.abs() * es + dZ.abs() * 2.0 ** -16
    for t, D, e in zip(got[:2], (dG, dU), (eG, eU)):
        assert bool(((t.cpu().double() - X.t() @ D).abs() <= X.abs().t() @ (e + (n + 16) * 2.0 ** -24 * D.abs())).all())
    for t, D, e in zip(got[2:4], (dG, dU), (eG, eU)):
        assert bool(((t.cpu().double() - D.sum(0)).abs() <= (e + (n + 16) * 2.0 ** -24 * D.abs()).sum(0)).all())
    ub = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0          # of an operand that is rounded

    def close(t, pairs):
        want, e = R.clone(), torch.zeros_like(R)
        for D, eD, W in pairs:
            want += D @ W.t()
            e += (eD + ub * D.abs()) @ W.abs().t() * (1 + ub) + _sum_bound(D, W.t(), dtype, 2 * fo)
        e += 2.0 ** -23 * want.abs()
        return bool(((t.cpu().double() - want).abs() <= e + u * (want.abs() + e)).all())

    assert close(got[4], ((dG, eG, Wg), (dU, eU, Wu)))
    dW, db, dX = B.tma_dense_residual_bwd(s(X), s(G), s(dH), d(Wg), _code(B, act), R=s(R))
    assert bool(((dW.cpu().double() - X.t() @ dZ).abs() <= X.abs().t() @ (eZ + (n + 16) * 2.0 ** -24 * dZ.abs())).all())
    assert bool(((db.cpu().double() - dZ.sum(0)).abs() <= (eZ + (n + 16) * 2.0 ** -24 * dZ.abs()).sum(0)).all())
    assert close(dX, ((dZ, eZ, Wg),))


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gradients_are_the_differences(B, act):
    """Central differences of sum(c H) along random directions, fp32: the step h = 2^-6 leaves an error of h^2 / 6 times a third derivative (of a product of
    a smooth function and a linear one along one direction, some units) and 2^-22 of the loss over 2 h."""
    g = torch.Generator().manual_seed(3)
    n, fi, fo = 40, 24, 56
    N = lambda *s: torch.randn(s, generator=g).cuda()
    X, Wg, Wu, Wd, bg, bu, bd = N(n, fi), N(fi, fo) / 5, N(fi, fo) / 5, N(fo, fi) / 8, N(fo) / 4, N(fo) / 4, N(fi) / 4
    c, code = N(n, fi), _code(B, act)

    def block(t):
        H, G, U = B.tma_gated_dense_fwd(t[0], t[1], t[2], t[3], t[4], code)
        return B.tma_dense_residual_fwd(H, t[5], t[6], R=t[0])[0], H, G, U

    leaves = [X, Wg, Wu, bg, bu, Wd, bd]
    Y, H, G, U = block(leaves)
    dWd, dbd, dH = B.tma_dense_residual_bwd(H, None, c, Wd)
    dWg, dWu, dbg, dbu, dX = B.tma_gated_dense_bwd(X, G, U, dH, Wg, Wu, code, R=c)
    for i, grad in enumerate((dX, dWg, dWu, dbg, dbu, dWd, dbd)):
        v = torch.randn(leaves[i].shape, generator=g).cuda()
        v /= v.norm()
        h = 2.0 ** -6
        loss = [float((block([t + s * h * v if j == i else t for j, t in enumerate(leaves)])[0].double() * c.double()).sum()) for s in (1, -1)]
        want, got = (loss[0] - loss[1]) / (2 * h), float((grad.double() * v.double()).sum())
        scale = float(grad.norm())
        assert abs(got - want) <= 2e-3 * scale, (i, got, want, scale)


# many tiles of both sizes, ranges of the rows that are joined, a block's several tiles one after the other
MANY = [(6_000, 520, 1_500), (16_401, 288, 1_100), (1_000, 64, 300), (9_000, 1_600, 2_048), (20_011, 96, 100), (2_300, 2_050, 600), (300, 4_100, 2_304), (70_000, 33, 1_100), (200, 4_096, 512), (130, 1_536, 1_024), (70, 2_049, 33), (1_100, 1_280, 320), (40_000, 31, 257), (16_400, 260, 1_100)]


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("n,fi,fo", MANY)
def test_many_tiles_of_whole_numbers(B, n, fi, fo, dtype):
    g = torch.Generator(device="cuda").manual_seed(n)
    W = lambda *s: torch.randint(-1, 2, s, generator=g, device="cuda").double()
    s, d = lambda t: t.to(dtype), lambda t: t.float()
    X, Wg, Wu, bg, bu, R = W(n, fi), W(fi, fo), W(fi, fo), W(fo), W(fo), W(n, fo)
    G, U = X @ Wg + bg, X @ Wu + bu
    h, gg, uu = B.tma_gated_dense_fwd(s(X), d(Wg), d(Wu), d(bg), d(bu), B.TMA_ACT_RELU)
    for got, want in ((gg, G), (uu, U), (h, G.clamp(min=0) * U)):
        assert torch.equal(got, want.float().to(dtype))
    y, z = B.tma_dense_residual_fwd(s(X), d(Wg), d(bg), B.TMA_ACT_RELU, R=s(R), save=True)
    assert torch.equal(z, gg) and torch.equal(y, (G.clamp(min=0) + R).float().to(dtype))
    del G, U, h, gg, uu, y, z
    G, U, dH, R = W(n, fo), W(n, fo), W(n, fo), W(n, fi)
    dG, dU = dH * U * (G > 0), dH * G.clamp(min=0)
    want = X.t() @ dG, X.t() @ dU, dG.sum(0), dU.sum(0), (dG @ Wg.t() + dU @ Wu.t() + R).float().to(dtype).double()
    for repeat in range(2):
        got = B.tma_gated_dense_bwd(s(X), s(G), s(U), s(dH), d(Wg), d(Wu), B.TMA_ACT_RELU, R=s(R))
        for t, w in zip(got, want):
            assert torch.equal(t.double(), w)
    for act, D in ((B.TMA_ACT_NONE, dH), (B.TMA_ACT_RELU, dH * (G > 0))):
        dW, db, dX = B.tma_dense_residual_bwd(s(X), s(G), s(dH), d(Wg), act, R=s(R))
        assert torch.equal(dW.double(), X.t() @ D) and torch.equal(db.double(), D.sum(0))
        assert torch.equal(dX, (D @ Wg.t() + R).float().to(dtype))


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_no_rows(B, dtype):
    e = lambda w: torch.empty((0, w), dtype=dtype, device="cuda")
    W = torch.ones((5, 9), device="cuda")
    full = lambda *s: torch.full(s, 7.0, device="cuda")
    assert B.tma_gated_dense_fwd(e(5), W, W)[0].shape == (0, 9)
    assert B.tma_dense_residual_fwd(e(5), W)[0].shape == (0, 9)
    out = [full(5, 9), full(5, 9), full(9), full(9)]
    B.tma_gated_dense_bwd(e(5), e(9), e(9), e(9), W, W, dW_gate=out[0], dW_up=out[1], db_gate=out[2], db_up=out[3])
    assert not any(t.any() for t in out)
    out = [full(5, 9), full(9)]
    B.tma_dense_residual_bwd(e(5), e(9), e(9), W, B.TMA_ACT_SILU, dW=out[0], dbias=out[1])
    assert not any(t.any() for t in out)


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_values_that_are_no_numbers_stay_in_their_row(B, dtype):
    """A NaN and an infinity in one row, and in the padding of all rows, reach that row's results and, backward, the weights' gradients of their columns; nothing else."""
    g = torch.Generator().manual_seed(8)
    n, fi, fo = 150, 50, 70
    N = lambda *s: torch.randn(s, generator=g)
    X, Wg, Wu = N(n, fi), N(fi, fo).cuda(), N(fi, fo).cuda()
    x, _ = _buffer(X, dtype, fi + 14)
    h, gg, uu = B.tma_gated_dense_fwd(x, Wg, Wu)
    y, _ = B.tma_dense_residual_fwd(x, Wg, R=h)
    dh, _ = _buffer(N(n, fo), dtype, fo + 10)
    clean = B.tma_gated_dense_bwd(x, gg, uu, dh, Wg, Wu)
    assert all(bool(t.isfinite().all()) for t in (h, gg, uu, y) + clean)
    for bad in (math.nan, math.inf):
        xb = x.clone()
        xb[33, 7] = bad
        hb, gb, ub = B.tma_gated_dense_fwd(xb, Wg, Wu)
        yb, _ = B.tma_dense_residual_fwd(xb, Wg, R=h)
        keep = torch.arange(n, device="cuda") != 33
        for t, was in ((hb, h), (gb, gg), (ub, uu), (yb, y)):
            assert torch.equal(t[keep], was[keep])
        assert not bool(gb[33].isfinite().any()) and not bool(yb[33].isfinite().any())
        got = B.tma_gated_dense_bwd(xb, gg, uu, dh, Wg, Wu)
        cols = torch.arange(fi, device="cuda") != 7
        for i in (0, 1):
            assert torch.equal(got[i][cols], clean[i][cols]) and not bool(got[i][7].isfinite().any())
        assert torch.equal(got[4], clean[4]) and torch.equal(got[2], clean[2])
        gbad = B._padded(n, fo, dtype, 'cuda').copy_(gg)       # (G and U share a pitch)
        gbad[33, 9] = bad
        got = B.tma_gated_dense_bwd(x, gbad, uu, dh, Wg, Wu)
        other = torch.arange(fo, device="cuda") != 9
        assert torch.equal(got[0][:, other], clean[0][:, other]) and torch.equal(got[4][keep], clean[4][keep])
        assert not bool(got[1][:, 9].isfinite().any()) and not bool(got[4][33].isfinite().any())


def test_large_and_small_fp32_values(B):
    """Values near the end of fp32's range and far below one: 24 bits of each count.  A product of two powers of two is exact."""
    big, small = 2.0 ** 127 * (2 - 2.0 ** -23), 2.0 ** -100 * (1 + 2.0 ** -23)
    X = torch.tensor([[big, 0.0], [0.0, small], [-big, 0.0]], device="cuda")
    W = torch.tensor([[1.0, 0.5, 0.0], [2.0, 0.0, 2.0 ** 60]], device="cuda")
    Y, _ = B.tma_dense_residual_fwd(X, W)
    assert torch.equal(Y, torch.tensor([[big, big / 2, 0.0], [2 * small, 0.0, small * 2.0 ** 60], [-big, -big / 2, 0.0]], device="cuda"))


# few rows of wide weights, whose k blocks share out: ranges of even and of uneven length, last ones that are shorter, columns that end inside a block, rows anywhere
FEW = [(1, 4_096, 1_024, 0, 0), (1, 8_000, 40, 0, 0), (16, 5_003, 77, 3, 1), (17, 4_096, 300, 0, 0), (24, 2_048, 5_632, 0, 0), (31, 8_191, 33, 1, 2), (64, 2_000, 1_001, 0, 0), (48, 1_111, 512, 8, 8),
       (3, 512, 70, 0, 0), (64, 96, 300, 0, 0)]


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("n,fi,fo,more,off", FEW)
def test_few_rows_of_whole_numbers(B, n, fi, fo, more, off, dtype):
    g = torch.Generator().manual_seed(fi)
    W = lambda *s: torch.randint(-1, 2, s, generator=g).double()
    X, Wg, Wu, bg, bu, R = W(n, fi), W(fi, fo), W(fi, fo), W(fo), W(fo), W(n, fo)
    G, U = X @ Wg + bg, X @ Wu + bu
    x, r = _buffer(X, dtype, fi + more, off)[0], _buffer(R, dtype, fo + more, off)[0]
    outs = [_buffer(torch.zeros(n, fo), dtype, fo + more, off, fill=7.0) for _ in range(4)]
    d = lambda t: t.float().cuda()
    want = G.clamp(min=0) * U, G, U, G.clamp(min=0) + R
    for repeat in range(2):
        B.tma_gated_dense_fwd(x, d(Wg), d(Wu), d(bg), d(bu), B.TMA_ACT_RELU, G_out=outs[1][0], U_out=outs[2][0], H_out=outs[0][0])
        B.tma_dense_residual_fwd(x, d(Wg), d(bg), B.TMA_ACT_RELU, R=r, Y_out=outs[3][0])
        for (t, flat), w in zip(outs, want):
            assert torch.equal(t.cpu(), w.float().to(dtype)) and _untouched(flat, t, 7.0)
    alone, _ = B.tma_dense_residual_fwd(x, d(Wu))
    assert torch.equal(alone.cpu(), (X @ Wu).float().to(dtype))
    B.tma_dense_residual_fwd(x, d(Wg), d(bg), B.TMA_ACT_RELU, R=r, Y_out=r)          # in place
    assert torch.equal(r.cpu(), want[3].float().to(dtype))


def test_an_infinite_last_weight_of_few_rows(B):
    """k ends inside a step: what stands for the weights behind it is a zero, whatever the last one is."""
    X, W = torch.ones((2, 37)), torch.ones((37, 20))
    W[36, 3] = math.inf
    for dtype in DTYPES:
        got = B.tma_dense_residual_fwd(X.to(dtype).cuda(), W.cuda())[0].float().cpu()
        rest = [c for c in range(20) if c != 3]
        assert torch.equal(got[:, rest], torch.full((2, 19), 37.0))
        # (fp32 rows come in three parts, and an infinity times a part that is zero is no number: the documented exception)
        assert bool((got[:, 3] == math.inf).all()) if dtype == torch.bfloat16 else not torch.isfinite(got[:, 3]).any()


def _block_step(B, t, ws, stream=None):
    """A residual block's step: forward, backward, clipping of the gradients."""
    H, G, U = B.tma_gated_dense_fwd(t["X"], t["Wg"], t["Wu"], t["bg"], t["bu"], B.TMA_ACT_SILU, G_out=t["G"], U_out=t["U"], H_out=t["H"], ws=ws, stream=stream)
    B.tma_dense_residual_fwd(H, t["Wd"], t["bd"], R=t["X"], Y_out=t["Y"], ws=ws, stream=stream)
    B.tma_dense_residual_bwd(H, None, t["dY"], t["Wd"], dW=t["dWd"], dbias=t["dbd"], dX_out=t["dH"], ws=ws, stream=stream)
    B.tma_gated_dense_bwd(t["X"], G, U, t["dH"], t["Wg"], t["Wu"], B.TMA_ACT_SILU, R=t["dY"], dW_gate=t["dWg"], dW_up=t["dWu"], db_gate=t["dbg"], db_up=t["dbu"],
                          dX_out=t["dX"], ws=ws, stream=stream)
    B.tma_grad_clip([t[k] for k in ("dWd", "dbd", "dWg", "dWu", "dbg", "dbu")], 0.5, norm_out=t["norm"], ws=ws, stream=stream)


RESULTS = ("H", "G", "U", "Y", "dH", "dX", "dWd", "dbd", "dWg", "dWu", "dbg", "dbu", "norm")


def _block_tensors(n, F, K, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: (torch.randn(s, generator=g) / s[0] ** 0.5).cuda()
    e, rows = (lambda *s: torch.empty(s, device="cuda")), lambda w: torch.empty((n, w), dtype=dtype, device="cuda")
    return dict(X=torch.randn((n, F), generator=g).to(dtype).cuda(), dY=torch.randn((n, F), generator=g).to(dtype).cuda(), Wg=r(F, K), Wu=r(F, K), bg=r(K), bu=r(K), Wd=r(K, F),
                bd=r(F), H=rows(K), G=rows(K), U=rows(K), Y=rows(F), dH=rows(K), dX=rows(F), dWd=e(K, F), dbd=e(F), dWg=e(F, K), dWu=e(F, K), dbg=e(K), dbu=e(K), norm=e(1))


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_two_captured_blocks_share_a_workspace(B, dtype):
    """Steps of two sizes captured into a graph each, with one workspace; replayed in turn with eager steps between them, on the capture's and on another stream."""
    sizes = (900, 96, 264), (40, 1_024, 2_048)
    code = B.TMA_BF16 if dtype == torch.bfloat16 else B.TMA_F32
    room = max(max(B.tma_gated_dense_fwd_workspace_bytes(n, F, K, code), B.tma_gated_dense_bwd_workspace_bytes(n, F, K, code), B.tma_dense_residual_fwd_workspace_bytes(n, K, F, code),
                   B.tma_dense_residual_bwd_workspace_bytes(n, K, F, B.TMA_ACT_NONE, code), B.tma_grad_norm_workspace_bytes(6)) for n, F, K in sizes)
    ws = torch.empty(room, dtype=torch.uint8, device="cuda")
    steps, graphs, want = [_block_tensors(*s, dtype, i) for i, s in enumerate(sizes)], [], []
    for t in steps:
        _block_step(B, t, ws)
        want.append({k: t[k].clone() for k in RESULTS})
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for t in steps:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            _block_step(B, t, ws, side)
        graphs.append(graph)
    other = torch.cuda.Stream()
    for turn in range(4):
        for i in (0, 1):
            for k in RESULTS:
                steps[i][k].fill_(math.nan)
            ws.fill_(255)
            torch.cuda.synchronize()
            with torch.cuda.stream(other if turn % 2 else side):
                graphs[i].replay()
            torch.cuda.synchronize()
            for k in RESULTS:
                assert torch.equal(steps[i][k], want[i][k]), (turn, i, k)
            if turn == 2:
                _block_step(B, steps[1 - i], None)
                for k in RESULTS:
                    assert torch.equal(steps[1 - i][k], want[1 - i][k]), (turn, i, k)


def test_two_streams_at_once(B):
    """Steps on two streams at the same time, workspaces and results from the allocator."""
    steps = [_block_tensors(700, 128, 320, torch.bfloat16, 3), _block_tensors(33, 2_048, 1_024, torch.bfloat16, 4)]
    want = []
    for t in steps:
        _block_step(B, t, None)
        want.append({k: t[k].clone() for k in RESULTS})
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(5):
        for t, s in zip(steps, streams):
            _block_step(B, t, None, s)
    torch.cuda.synchronize()
    for t, w in zip(steps, want):
        for k in RESULTS:
            assert torch.equal(t[k], w[k]), k


def test_places_past_32_bits(B):
    """Rows whose places, in elements and more so in bytes, do not fit into 32 bits: of whole numbers, checked at the first and the last ones."""
    n, fi, fo = 270_001, 64, 8_192
    g = torch.Generator(device="cuda").manual_seed(0)
    W = lambda *s, dtype=torch.bfloat16: torch.randint(-1, 2, s, generator=g, device="cuda", dtype=torch.int8).to(dtype)
    X, Wt, dY, R = W(n, fi), W(fi, fo, dtype=torch.float32), W(n, fo), W(n, fi)
    assert dY.numel() > 1 << 31
    Y, _ = B.tma_dense_residual_fwd(X, Wt, R=dY)
    ends = [slice(0, 200), slice(n // 2, n // 2 + 200), slice(n - 200, n)]
    for rows in ends:
        assert torch.equal(Y[rows], (X[rows].float() @ Wt + dY[rows].float()).bfloat16())
    del Y
    H, G, U = B.tma_gated_dense_fwd(X, Wt, Wt, act=B.TMA_ACT_NONE)
    for rows in ends:
        z = X[rows].float() @ Wt
        assert torch.equal(G[rows], z.bfloat16()) and torch.equal(U[rows], G[rows]) and torch.equal(H[rows], (z * z).bfloat16())
    del H, G, U
    dW, db, dX = B.tma_dense_residual_bwd(X, None, dY, Wt, R=R)
    for rows in ends:
        assert torch.equal(dX[rows], (dY[rows].float() @ Wt.t() + R[rows].float()).bfloat16())
    want, sums = torch.zeros((fi, fo), device="cuda"), torch.zeros(fo, device="cuda")
    for a in range(0, n, 30_000):          # (sums of whole numbers below 2^24: exact)
        part = dY[a:a + 30_000].float()
        want += X[a:a + 30_000].float().t() @ part
        sums += part.sum(0)
    assert torch.equal(dW, want) and torch.equal(db, sums)
    # rows where they lie, far apart
    far = W(n, 8_192)[:, 96:160]
    got, _ = B.tma_dense_residual_fwd(far, Wt[:, :40].contiguous())
    for rows in ends:
        assert torch.equal(got[rows], (far[rows].float() @ Wt[:, :40]).bfloat16())
