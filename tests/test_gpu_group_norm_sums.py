"""The sums of group norm over many rows: statistics, the two means of the input gradient, and the gradients of gamma, beta and slope, on data for which a row
that is missed or counted twice shows.  u = 2^-24, h = half a step of the storage type.

Whole numbers.  Squares and products of small whole numbers (and quarters of them) are added up exactly below 2^24 (2^22) in any order, so sums have to be the exact ones.
Means: a chunk of eight rows is added up exactly and joined to others, in a tile, over its tiles (at least eight lanes side by side) and over lanes: at most rows / 64 + 40
joins, each off by u of the mean (no more than X, the largest magnitude) and by 3 u of what it moves it by (in a chain 2 X / k at the k-th join, 42 u X in all for
a thousand; over lanes at most 12 times 2 X, 72 u X), with the chunk's own rounding less than (rows / 64 + 190) u X.

Any numbers.  The upstream gradient has a mean and a part along the normalised input, so that both means of the input gradient are of order one.  With stats
given, xh is off by 4 u |xh| from the definition at those stats; a row by itself has sums of at most 24 roundings, 30 u mean|x| rstd + 24 u |xh|.  y is off by |gamma| times that
and 3 u (|gamma xh| + |beta|).  SiLU's slope changes by at most half of it and is itself off by 8 u (1 + |y|), in bf16 storage (fast exponential, whose argument carries u |y|,
and reciprocal) by 2 u (1 + |y|) (2 |y| + 8); the other slopes are exact where y is not near zero (there the upstream gradient is zero).  Sums of A terms after each other are
off by A u of the sum of magnitudes: a lane's of a tile and its tiles' (1,024 + rows / 64; a row by itself 32), over all rows 512 + n / 8 at most.  The rest is the rounding of
the formula as it is written.  That the bounds are narrow enough is asserted: input gradients without their means, and gradients of zero, are ten bounds off."""
import pytest

from test_gpu_group_norm import ACTS, B, act_of, apply_act, close, laid_out, per_cell, segment_of, u

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
EDGES = {"one": [0, 16_003], "long": [0, 5, 15_005, 15_006, 16_000, 16_003], "ragged": [0, 1, 1, 40, 41, 300, 300, 300, 771, 780, 1200], "outside": [17, 60, 61, 444]}


def of_and_rows(edges, n):
    of = segment_of(n, edges)
    return of, torch.tensor([b - a for a, b in zip(edges[:-1], edges[1:])], dtype=torch.float64)


# ---- whole numbers ---------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("G,cg", [(4, 8), (3, 6), (2, 64), (1, 700)])
@pytest.mark.parametrize("name", list(EDGES))
def test_statistics_count_every_row_once(B, name, G, cg, dtype):
    edges = EDGES[name]
    n = edges[-1] + 4
    g = torch.Generator().manual_seed(G)
    of, rows = of_and_rows(edges, n)
    held = rows > 0
    ones, zeros = torch.ones(G * cg, device="cuda"), torch.zeros(G * cg, device="cuda")
    segments = torch.tensor(edges, dtype=torch.int32, device="cuda")
    # -a and a beside each other, a = 1 or 3 in each row and group: the mean is zero, the squares' sum exact
    a = 1 + 2 * torch.randint(0, 2, (n, G), generator=g)
    x = (a[:, :, None] * (1 - 2 * (torch.arange(cg) % 2))).reshape(n, G * cg)
    _, stats = B.tma_groupnorm_act_fwd(laid_out(B, x.to(dtype), "padded"), G, ones, zeros, segments=segments, eps=0.0)
    var = per_cell(x.double().square(), of, len(rows), G)
    assert not stats[:, :, 0].any() and not stats.cpu()[~held].any()
    want = var[held].rsqrt()
    close(stats.cpu()[held][:, :, 1], want, 4 * u * want, "rstd")          # a quotient, a root and a quotient
    # rows of -4 or 4: the mean
    x = (8 * torch.randint(0, 2, (n, G), generator=g) - 4)[:, :, None].expand(n, G, cg).reshape(n, G * cg)
    _, stats = B.tma_groupnorm_act_fwd(laid_out(B, x.to(dtype), "padded"), G, ones, zeros, segments=segments)
    tol = ((rows / 64 + 190) * u * 4)[:, None].expand(-1, G)
    assert (tol[held] < 4 / rows[held][:, None]).all()                     # (one row's share)
    close(stats.cpu()[held][:, :, 0], per_cell(x.double(), of, len(rows), G)[held], tol[held], "mean")


def whole_gradients(x, dy, gamma, beta, act, slope):
    y = gamma * x + beta
    dz = dy * torch.where(y > 0, 1.0, {"none": 1.0, "relu": 0.0, "prelu": slope}[act])
    return y, dz


@pytest.mark.parametrize("act", ["none", "relu", "prelu"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("G,cg", [(4, 8), (3, 5), (2, 64), (1, 70)])
@pytest.mark.parametrize("name", list(EDGES))
def test_backward_sums_over_segments_are_exact(B, name, G, cg, dtype, act):
    """Mean 0 and rstd 1 are given, so xh is x."""
    edges, F = EDGES[name], G * cg
    n = edges[-1] + 4
    g = torch.Generator().manual_seed(F)
    of, rows = of_and_rows(edges, n)
    S, inside = len(rows), of >= 0
    x = torch.randint(-3, 4, (n, F), generator=g).double()
    dy = torch.randint(0, 3, (n, F), generator=g).double() + (x > 0)
    gamma, beta = 1.0 + torch.randint(0, 2, (F,), generator=g), torch.randint(-1, 2, (F,), generator=g).double()
    slope = torch.tensor([0.25], device="cuda") if act == "prelu" else None
    stats = torch.tensor([0.0, 1.0]).expand(S, G, 2).contiguous().cuda()
    dX = torch.full((n, F), 7.0, dtype=dtype, device="cuda")
    _, dga, dbe, dsl = B.tma_groupnorm_act_bwd(laid_out(B, x.to(dtype), "padded"), laid_out(B, dy.to(dtype), "padded"), G, gamma.float().cuda(), beta.float().cuda(),
                                               act_of(B, act), slope=slope, segments=torch.tensor(edges, dtype=torch.int32, device="cuda"), stats=stats, dX_out=dX)
    y, dz = whole_gradients(x, dy * inside[:, None], gamma, beta, act, 0.25)
    assert (dz * x).abs().sum(0).max() < 2 ** 22 and (dy * y).abs().sum() < 2 ** 24
    assert torch.equal(dga.cpu().double(), (dz * x).sum(0)) and torch.equal(dbe.cpu().double(), dz.sum(0))
    if slope is not None:
        assert dsl.item() == (dy * y * (y <= 0) * inside[:, None]).sum().item()
    wide = lambda t: t[of.clamp(min=0)].repeat_interleave(cg, 1)
    dxh = dz * gamma
    size = (rows * cg).clamp(min=1)[:, None]
    assert (per_cell((dxh * x).abs(), of, S, G) * size).max() < (2 ** 22 if act == "prelu" else 2 ** 24)      # (in quarters: below 2^24 of them)
    m1, m2 = wide(per_cell(dxh, of, S, G)), wide(per_cell(dxh * x, of, S, G))
    want = dxh - m1 - x * m2
    tol = 5 * u * (dxh.abs() + m1.abs() + (x * m2).abs())
    tol = tol + torch.finfo(dtype).eps / 2 * (want.abs() + tol)
    close(dX.cpu()[inside], want[inside], tol[inside], "dX")
    assert (dX.cpu()[~inside] == 7).all()


@pytest.mark.parametrize("act", ["none", "relu", "prelu"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,G,cg", [(1, 4, 8), (5_003, 4, 8), (3_001, 1, 64), (70_001, 8, 4), (1_500, 2, 512), (40_000, 1, 2)])
def test_backward_sums_over_rows_by_themselves_are_exact(B, n, G, cg, dtype, act):
    """As many 1.5 as -1.5 in each group and eps = 1.75: the mean is 0, rstd 1 / 2, xh 3 / 4 of a sign, all exact."""
    g = torch.Generator().manual_seed(n)
    F = G * cg
    sign = torch.where(torch.rand((n, G, cg), generator=g).argsort(2) < cg // 2, -1.0, 1.0).reshape(n, F).double()
    xh = 0.75 * sign
    dy = torch.randint(0, 3, (n, F), generator=g).double() + (sign > 0)
    gamma, beta = 1.0 + torch.randint(0, 2, (F,), generator=g), torch.randint(-1, 2, (F,), generator=g).double()
    slope = torch.tensor([0.25], device="cuda") if act == "prelu" else None
    dX, dga, dbe, dsl = B.tma_groupnorm_act_bwd(laid_out(B, (1.5 * sign).to(dtype), "padded"), laid_out(B, dy.to(dtype), "padded"), G, gamma.float().cuda(),
                                                beta.float().cuda(), act_of(B, act), slope=slope, eps=1.75)
    y, dz = whole_gradients(xh, dy, gamma, beta, act, 0.25)
    assert (dz * xh).abs().sum(0).max() < 2 ** 20 and (dy * y).abs().sum() < 2 ** 22
    assert torch.equal(dga.cpu().double(), (dz * xh).sum(0)) and torch.equal(dbe.cpu().double(), dz.sum(0))
    if slope is not None:
        assert dsl.item() == (dy * y * (y <= 0)).sum().item()
    dxh = dz * gamma
    mean = lambda t: t.view(n, G, cg).mean(2).repeat_interleave(cg, 1)
    m1, m2 = mean(dxh), mean(dxh * xh)
    want = (dxh - m1 - xh * m2) / 2
    tol = 5 * u * (dxh.abs() + m1.abs() + (xh * m2).abs())
    close(dX.cpu(), want, tol + torch.finfo(dtype).eps / 2 * (want.abs() + tol), "dX")


# ---- any numbers ---------------------------------------------------------------
class Gradients:
    """Inputs, the gradients in 64 bits and how far the kernels' may be off; edges None: rows by themselves."""

    def __init__(self, n, G, cg, edges, dtype, act, seed):
        g = torch.Generator().manual_seed(seed)
        F, h = G * cg, torch.finfo(dtype).eps / 2
        self.G, self.act, self.slope, self.dtype = G, act, 0.25, dtype
        single = edges is None
        edges = list(range(n + 1)) if single else edges
        of, rows = of_and_rows(edges, n)
        S = len(rows)
        self.inside = inside = of >= 0
        wide = lambda t: t[of.clamp(min=0)].repeat_interleave(cg, 1) * inside[:, None]
        cell = lambda t: wide(per_cell(t, of, S, G))
        self.x = (torch.randn((n, F), generator=g) + 0.3).to(dtype)
        X = self.x.double()
        self.gamma, self.beta = 1 + 0.2 * torch.rand(F, generator=g), 0.2 * torch.randn(F, generator=g)
        mean = per_cell(X, of, S, G)
        rstd = (per_cell((X - wide(mean)).square(), of, S, G) + 1e-5).rsqrt() * (rows > 0)[:, None]
        mean = mean * (rows > 0)[:, None]
        if not single:                 # what is given, as it is held
            self.stats = torch.stack([mean, rstd], 2).float()
            mean, rstd = self.stats.double().unbind(2)
        rs = wide(rstd)
        xh = (X - wide(mean)) * rs
        dy = (1 + 0.7 * xh + 0.5 * torch.randn((n, F), generator=g)).to(dtype)
        ga, be = self.gamma.double(), self.beta.double()
        y = ga * xh + be
        d_xh = (30 * cell(X.abs()) * rs + 24 * xh.abs() if single else 4 * xh.abs()) * u
        d_y = ga.abs() * d_xh + 3 * u * ((ga * xh).abs() + be.abs())
        if act in ("relu", "prelu"):
            dy = torch.where(y.abs() <= 2 * d_y, torch.zeros((), dtype=dtype), dy)
        self.dy = dy
        dy = dy.double() * inside[:, None]
        if act == "silu":
            t = 1 / (1 + torch.exp(-y))
            dz = dy * t * (1 + y * (1 - t))
            d_dz = dy.abs() * (d_y / 2 + (8 * u * (1 + y.abs()) if dtype == torch.float32 else 2 * u * (1 + y.abs()) * (2 * y.abs() + 8)))
        else:
            dz = dy * torch.where(y > 0, 1.0, {"none": 1.0, "relu": 0.0, "prelu": self.slope}[act])
            d_dz = u * dz.abs()
        dxh = dz * ga
        d_dxh = ga.abs() * d_dz + u * dxh.abs()
        terms = wide((32 if single else 1024 + rows / 64)[:, None].expand(S, G)) if not single else 32.0
        m1, m2 = cell(dxh), cell(dxh * xh)
        d_m1 = terms * u * cell(dxh.abs()) + cell(d_dxh)
        d_m2 = (terms + 2) * u * cell((dxh * xh).abs()) + cell(d_dxh * xh.abs() + dxh.abs() * d_xh)
        self.dx = (dxh - m1 - xh * m2) * rs
        tol = (d_dxh + d_m1 + xh.abs() * d_m2 + m2.abs() * d_xh + 5 * u * (dxh.abs() + m1.abs() + (xh * m2).abs())) * rs + (24 * u if single else u) * self.dx.abs()
        self.dx_tol = tol + h * (self.dx.abs() + tol)
        P = (512 + n / 8) * u
        self.sums = [((dz * xh).sum(0), P * (dz * xh).abs().sum(0) + (d_dz * xh.abs() + dz.abs() * d_xh).sum(0)), (dz.sum(0), P * dz.abs().sum(0) + d_dz.sum(0))]
        low = dy * y * (y <= 0)
        self.sums.append((low.sum(), P * low.abs().sum() + (dy.abs() * (d_y + u * y.abs()) * (y <= 0)).sum()))
        # what the bounds would let pass
        several = inside if single else wide((rows > 1)[:, None].expand(S, G).double())[:, 0] > 0
        for without in (m1, xh * m2):
            assert ((without * rs).abs() / self.dx_tol.clamp(min=1e-300))[several].max() > 10
        for want, t in self.sums[:3 if act == "prelu" else 2]:
            assert (want.abs() / t).max() > 10, (want.abs() / t).max()


def check(B, c, layout, edges):
    how = dict(slope=torch.tensor([c.slope], device="cuda") if c.act == "prelu" else None, eps=1e-5)
    if edges is not None:
        how.update(segments=torch.tensor(edges, dtype=torch.int32, device="cuda"), stats=c.stats.cuda())
    dx = laid_out(B, torch.full_like(c.x, 7.0), layout)
    got = B.tma_groupnorm_act_bwd(laid_out(B, c.x, layout), laid_out(B, c.dy, layout), c.G, c.gamma.cuda(), c.beta.cuda(), act_of(B, c.act), dX_out=dx, **how)
    close(dx.cpu()[c.inside], c.dx[c.inside], c.dx_tol[c.inside], "dX")
    assert (dx.cpu()[~c.inside] == 7).all()
    for what, g, (want, tol) in zip(("dgamma", "dbeta", "dslope"), got[1:], c.sums):
        if g is not None:
            close(g.cpu().reshape(want.shape), want, tol, what)


SHAPES = [(1, 3), (3, 5), (32, 8), (1, 256), (5, 70), (2, 700)]


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("G,cg", SHAPES)
def test_gradients_of_rows_by_themselves(B, G, cg, dtype, act):
    for n, layout in [(37, "odd"), (1003, "padded")]:
        check(B, Gradients(n, G, cg, None, dtype, act, n + G), layout, None)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("G,cg", SHAPES)
@pytest.mark.parametrize("edges", [[0, 900], EDGES["ragged"], EDGES["outside"]], ids=["one", "ragged", "outside"])
def test_gradients_over_segments(B, edges, G, cg, dtype, act):
    check(B, Gradients(edges[-1] + 3, G, cg, edges, dtype, act, 5 + G), "odd" if cg == 70 else "padded", edges)


@pytest.mark.parametrize("act", ["prelu", "silu"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("edges", [[0, 5, 50_005, 50_006, 53_000, 60_000], [0, 60_000]], ids=["ragged", "one"])
def test_gradients_over_many_tiles(B, edges, dtype, act):
    check(B, Gradients(60_000, 4, 8, edges, dtype, act, 1), "padded", edges)


def test_gradients_against_differences(B):
    """L = sum(G (.) Y) along the gradient's own signs, a central difference of the fp32 forward pass.  Its truncation is what the same difference has in 64 bits; the rounding of a
    pass is at most sum|G| times an element's bound, 4 (160 + 44 / 8) u (|gamma| (|xh| + mean|x| rstd) + |beta|) and u |y| more, here below 800 u times 8 (the factor is 5.5)."""
    edges, G, cg, step = [0, 20, 64], 4, 8, 2.0 ** -5
    c = Gradients(64, G, cg, edges, torch.float32, "silu", 7)
    of, _ = of_and_rows(edges, 64)
    wide = lambda t: t[of].repeat_interleave(cg, 1)
    dy, segments = c.dy.double(), torch.tensor(edges, dtype=torch.int32, device="cuda")

    def plain(x, gamma, beta):
        v = x - wide(per_cell(x, of, 2, G))
        return (apply_act(gamma * v * wide((per_cell(v * v, of, 2, G) + 1e-5).rsqrt()) + beta, "silu", 0) * dy).sum().item()

    def kernel(x, gamma, beta):
        y = B.tma_groupnorm_act_fwd(x.float().cuda(), G, gamma.float().cuda(), beta.float().cuda(), B.TMA_ACT_SILU, segments=segments)[0]
        return (y.cpu().double() * dy).sum().item()

    at = [c.x.double(), c.gamma.double(), c.beta.double()]
    _, stats = B.tma_groupnorm_act_fwd(c.x.cuda(), G, c.gamma.cuda(), c.beta.cuda(), B.TMA_ACT_SILU, segments=segments)
    grads = B.tma_groupnorm_act_bwd(c.x.cuda(), c.dy.cuda(), G, c.gamma.cuda(), c.beta.cuda(), B.TMA_ACT_SILU, segments=segments, stats=stats)[:3]
    leaves = [t.clone().requires_grad_(True) for t in at]
    x, gamma, beta = leaves
    v = x - wide(per_cell(x, of, 2, G))
    exact = torch.autograd.grad((apply_act(gamma * v * wide((per_cell(v * v, of, 2, G) + 1e-5).rsqrt()) + beta, "silu", 0) * dy).sum(), leaves)
    rounding = 2 * dy.abs().sum().item() * 800 * u * 8 / (2 * step)
    for k, (mine, true) in enumerate(zip(grads, exact)):
        d = torch.sign(true) * (0.5 if k == 0 else 1.0)
        hi, lo = list(at), list(at)
        hi[k], lo[k] = (at[k] + step * d).float().double(), (at[k] - step * d).float().double()
        along = (true * (hi[k] - lo[k])).sum().item() / (2 * step)
        truncation = abs((plain(*hi) - plain(*lo)) / (2 * step) - along)
        assert along > 10 * (truncation + rounding), (along, truncation, rounding)
        slope = (kernel(*hi) - kernel(*lo)) / (2 * step)
        mine = (mine.cpu().double() * (hi[k] - lo[k])).sum().item() / (2 * step)
        assert abs(slope - mine) <= truncation + rounding
