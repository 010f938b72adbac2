"""Group norm with an activation against the definition in 64 bits.

Tolerances, element by element.  u = 2^-24, h = half a step of the storage type.  A mean over a group is a tree of sums of at most
D = 160 + rows / 8 roundings from a value to the result (128 elements of a lane, six exchanges between lanes, a join per tile of at
least eight rows and a few operations each), so it is off by D u mean|x|, and rstd, from squares about that mean, by 2 D u of
itself (the mean's own error counts squared).  An element of the result is then off by at most
    4 D u (|gamma| (|xh| + mean|x| rstd) + |beta|)      (the activations' slopes are below 1.1)
and one rounding, h |y|.  The gradient's terms dxh = gamma dz carry 4 D u (1 + |gamma| (|xh| + mean|x| rstd) + |beta|) of |gamma dy| (SiLU's
slope changes by at most one half per unit); m1 and m2 are means of them: with A the largest |gamma dy| of the group and c the
largest of these factors, dX is off by 8 D u c A rstd (2 + |xh| max|xh|) + h |dX|, dgamma and dbeta by 8 D u c sums of |dy| max(1, |xh|)
and the roundings of a sum over n rows, n u of the same.
Where y is nearer to zero than its tolerance ReLU's and PReLU's slope may be either: there the upstream gradient is zero."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
u = 2.0 ** -24
EPS = 1e-5
ACTS = ["none", "relu", "prelu", "silu"]


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2305_09887_amd import binding
    binding.lib()
    return binding


def act_of(B, name):
    return {"none": B.TMA_ACT_NONE, "relu": B.TMA_ACT_RELU, "prelu": B.TMA_ACT_PRELU, "silu": B.TMA_ACT_SILU}[name]


def apply_act(y, name, slope):
    if name == "silu":
        return y / (1 + torch.exp(-y))
    return torch.where(y > 0, y, {"none": 1.0, "relu": 0.0, "prelu": slope}[name] * y)


def laid_out(B, x, layout):
    n, F = x.shape
    if layout == "padded":
        d = B._padded(n, F, x.dtype, "cuda")
    elif layout == "dense":
        d = torch.empty((n, F), dtype=x.dtype, device="cuda")
    else:
        d = torch.empty((n * (F + 3) + 1,), dtype=x.dtype, device="cuda")[1:].view(n, F + 3)[:, :F]
    d.copy_(x)
    return d


def segment_of(n, edges):
    """each row's segment (-1: none)"""
    of = torch.full((n,), -1, dtype=torch.long)
    for s, (a, b) in enumerate(zip(edges[:-1], edges[1:])):
        of[a:b] = s
    return of


def per_cell(x, of, S, G, how="mean"):
    """mean or largest value of every (segment, group) of x"""
    v = x.view(x.shape[0], G, -1)[of >= 0]
    at = of[of >= 0]
    if how == "max":
        return torch.zeros((S, G), dtype=torch.float64).scatter_reduce_(0, at[:, None].expand(-1, G), v.amax(2), "amax")
    size = torch.bincount(at, minlength=S).clamp(min=1)[:, None] * v.shape[2]
    return torch.zeros((S, G), dtype=torch.float64).index_add_(0, at, v.sum(2)) / size


class Case:
    def __init__(self, n, G, cg, edges, dtype, act, seed, shift=0.3):
        g = torch.Generator().manual_seed(seed)
        F = G * cg
        self.x = (torch.randn((n, F), generator=g) + shift).to(dtype)
        self.dy = torch.randn((n, F), generator=g).to(dtype)
        self.gamma, self.beta = 1 + 0.3 * torch.randn(F, generator=g), 0.3 * torch.randn(F, generator=g)
        self.G, self.edges, self.act, self.slope, self.dtype = G, edges, act, 0.25, dtype
        X = self.x.double()
        S = len(edges) - 1
        self.of = segment_of(n, edges)
        self.inside = self.of >= 0
        self.wide = wide = lambda t: t[self.of.clamp(min=0)].repeat_interleave(cg, 1) * self.inside[:, None]
        self.mean = per_cell(X, self.of, S, G)
        self.var = per_cell((X - wide(self.mean)).square(), self.of, S, G)
        mag = per_cell(X.abs(), self.of, S, G)
        rows = max([b - a for a, b in zip(edges[:-1], edges[1:])] + [1])
        self.D = D = 160 + rows / 8
        self.rstd = 1 / (self.var + EPS).sqrt()
        self.rs = wide(self.rstd)
        self.xh = (X - wide(self.mean)) * self.rs
        self.y = self.gamma.double() * self.xh + self.beta.double()
        spread = self.gamma.double().abs() * (self.xh.abs() + wide(mag) * self.rs) + self.beta.double().abs()
        self.near = 4 * D * u * spread
        self.c = 1 + spread
        self.out = apply_act(self.y, act, self.slope)
        self.tol = 1.1 * self.near + torch.finfo(dtype).eps / 2 * (self.out.abs() + 1.1 * self.near)
        if act in ("relu", "prelu"):
            self.dy = torch.where(self.y.abs() <= self.near, torch.zeros((), dtype=dtype), self.dy)
    def backward(self):
        n, G, S, h = self.x.shape[0], self.G, len(self.edges) - 1, torch.finfo(self.dtype).eps / 2
        y = self.y.clone().requires_grad_(True)
        dy, xh = self.dy.double() * self.inside[:, None], self.xh
        dz = torch.autograd.grad(apply_act(y, self.act, self.slope), y, dy)[0]
        dslope = dy * self.y * (self.y <= 0)
        dxh = dz * self.gamma.double()
        cell = lambda t, how="mean": self.wide(per_cell(t, self.of, S, G, how))
        dx = (dxh - cell(dxh) - xh * cell(dxh * xh)) * self.rs
        off = 8 * self.D * u * cell(self.c, "max") * cell((self.gamma.double() * dy).abs() * 1.1, "max") * self.rs * (2 + xh.abs() * cell(xh.abs(), "max"))
        mass = 1.1 * dy.abs()
        share = 8 * self.D * u * self.c.max() + n * u
        sums = ((dz * xh).sum(0), dz.sum(0))
        tols = (share * (mass * xh.abs().clamp(min=1)).sum(0), share * mass.sum(0))
        return dx, off + h * (dx.abs() + off), sums, tols, dslope.sum(), share * (mass * (1 + self.y.abs())).sum()


def close(got, want, tol, what):
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {((got.double() - want).abs() / tol.clamp(min=1e-300)).max():.3g} tolerances"


def check(B, c, layout, segments=None, rows_per_segment=1):
    n, F = c.x.shape
    x, dy = laid_out(B, c.x, layout), laid_out(B, c.dy, layout)
    gamma, beta = c.gamma.cuda(), c.beta.cuda()
    slope = torch.tensor([c.slope], device="cuda") if c.act == "prelu" else None
    how = dict(slope=slope, segments=segments, rows_per_segment=rows_per_segment, eps=EPS)
    out = laid_out(B, torch.full_like(c.x, 7.0), layout)
    got, stats = B.tma_groupnorm_act_fwd(x, c.G, gamma, beta, act_of(B, c.act), out=out, **how)
    assert got is out
    close(out.cpu()[c.inside], c.out[c.inside], c.tol[c.inside], "Y")
    assert (out.cpu()[~c.inside] == 7).all()
    if stats is not None:
        held = torch.tensor([b > a for a, b in zip(c.edges[:-1], c.edges[1:])])
        assert not stats.cpu()[~held].any()
        close(stats.cpu()[held][:, :, 0], c.mean[held], (c.D * u * (c.mean.abs() + (c.var + EPS).sqrt()) * 4)[held], "mean")
        close(stats.cpu()[held][:, :, 1], c.rstd[held], (8 * c.D * u * c.rstd * (1 + c.mean.abs() * c.rstd))[held], "rstd")
        plain, none = B.tma_groupnorm_act_fwd(x, c.G, gamma, beta, act_of(B, c.act), need_stats=False, **how)
        assert none is None and torch.equal(plain[c.inside.cuda()], out[c.inside.cuda()])
    dx = laid_out(B, torch.full_like(c.x, 7.0), layout)
    res = B.tma_groupnorm_act_bwd(x, dy, c.G, gamma, beta, act_of(B, c.act), stats=stats, dX_out=dx, **how)
    want, tol, sums, tols, dslope, slope_tol = c.backward()
    close(dx.cpu()[c.inside], want[c.inside], tol[c.inside], "dX")
    assert (dx.cpu()[~c.inside] == 7).all()
    close(res[1].cpu(), sums[0], tols[0], "dgamma")
    close(res[2].cpu(), sums[1], tols[1], "dbeta")
    if slope is None:
        assert res[3] is None
    else:
        close(res[3].cpu()[0], dslope, slope_tol, "dslope")
    again = B.tma_groupnorm_act_bwd(x, dy, c.G, gamma, beta, act_of(B, c.act), stats=stats, dX_out=dy, **how)      # in place, the same bits
    assert torch.equal(again[0][c.inside.cuda()], dx[c.inside.cuda()])
    assert all(torch.equal(a, b) for a, b in zip(again[1:3], res[1:3]))


SHAPES = [(1, 3), (3, 5), (2, 2), (32, 8), (8, 16), (4, 25), (1, 256), (7, 12), (5, 70), (40, 24), (2, 700)]


@pytest.mark.parametrize("act", ["prelu", "silu"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("G,cg", SHAPES)
def test_rows_by_themselves(B, G, cg, dtype, act):
    for n, layout in [(1, "padded"), (37, "odd"), (1003, "dense"), (2500, "padded")]:
        if n * G * cg > 700_000:
            n = 301
        check(B, Case(n, G, cg, list(range(n + 1)), dtype, act, n + G), layout)


@pytest.mark.parametrize("act", ["relu", "silu"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("G,cg", SHAPES)
def test_runs_of_rows(B, G, cg, dtype, act):
    for S, R, layout in [(1, 1500, "padded"), (30, 7, "odd"), (3, 64, "dense"), (100, 2, "padded")]:
        n = S * R
        check(B, Case(n, G, cg, list(range(0, n + 1, R)), dtype, act, S + G), layout, rows_per_segment=R)


EDGES = {"one": [0, 900], "ragged": [0, 1, 1, 40, 41, 300, 300, 300, 771, 780, 1200], "empty_ends": [0, 0, 0, 500, 500], "outside": [17, 60, 61, 444],
         "none": [50, 50, 50], "single": [3, 4], "rows": list(range(200))}


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("G,cg", [(1, 3), (32, 8), (2, 700)])
@pytest.mark.parametrize("name", list(EDGES))
def test_ragged_segments(B, name, G, cg, dtype, act):
    edges = EDGES[name]
    n = edges[-1] + (9 if name in ("outside", "none", "single") else 0)
    c = Case(n, G, cg, edges, dtype, act, 5 + G)
    for layout in ("padded", "odd"):
        check(B, c, layout, segments=torch.tensor(edges, dtype=torch.int32, device="cuda"))


def test_long_segments_and_many_tiles(B):
    """Segments over many tiles beside short ones: 60,000 rows, one of 50,000."""
    edges = [0, 5, 50_005, 50_006, 53_000, 60_000]
    check(B, Case(60_000, 4, 8, edges, torch.float32, "silu", 1), "padded", segments=torch.tensor(edges, dtype=torch.int32, device="cuda"))
    check(B, Case(60_000, 2, 16, [0, 60_000], torch.bfloat16, "prelu", 2), "padded", rows_per_segment=60_000)


def test_variance_far_from_zero(B):
    """A mean of 1000 standard deviations: sums of squares of raw values would leave nothing of the variance (1e6 u = 0.06)."""
    for how, edges in [(dict(), list(range(401))), (dict(rows_per_segment=400), [0, 400])]:
        c = Case(400, 2, 32, edges, torch.float32, "none", 3, shift=1000.0)
        y, _ = B.tma_groupnorm_act_fwd(c.x.cuda(), 2, c.gamma.cuda(), c.beta.cuda(), eps=EPS, **how)
        close(y.cpu(), c.out, c.tol, "far")
        assert (y.cpu().double() - c.out).abs().max() < 0.01


def test_one_group_and_single_rows_are_layer_normalisation(B):
    x = torch.randn((900, 128), generator=torch.Generator().manual_seed(1)).cuda()
    gamma, beta, slope = torch.rand(128, device="cuda"), torch.rand(128, device="cuda"), torch.tensor([0.25], device="cuda")
    want = B.tma_layernorm_prelu_fwd(x, gamma, beta, slope)
    got, _ = B.tma_groupnorm_act_fwd(x, 1, gamma, beta, B.TMA_ACT_PRELU, slope=slope)
    assert (got - want).abs().max() <= 64 * u * want.abs().max()


def test_nan_and_infinity_stay_in_their_segment_and_group(B):
    edges = [0, 100, 230]
    c = Case(240, 4, 8, edges, torch.float32, "silu", 4)
    x = c.x.clone()
    x[30, 9] = float("nan")
    x[235] = float("inf")            # outside the segments
    seg = torch.tensor(edges, dtype=torch.int32, device="cuda")
    y = B.tma_groupnorm_act_fwd(x.cuda(), 4, c.gamma.cuda(), c.beta.cuda(), B.TMA_ACT_SILU, segments=seg)[0].cpu()
    bad = torch.zeros((240, 32), dtype=torch.bool)
    bad[:100, 8:16] = True
    assert torch.isnan(y[bad]).all()
    good = ~bad & c.inside[:, None]
    close(y[good], c.out[good], c.tol[good], "others")


@pytest.mark.parametrize("kind", ["row", "ragged"])
def test_stream_and_graph(B, kind):
    n, G, F = 3001, 4, 48
    g = torch.Generator().manual_seed(6)
    x, dy = torch.randn((n, F), generator=g).cuda(), torch.randn((n, F), generator=g).cuda()
    gamma, beta = torch.rand(F, device="cuda"), torch.rand(F, device="cuda")
    seg = torch.tensor([0, 10, 1000, 1000, 3000], dtype=torch.int32, device="cuda") if kind == "ragged" else None
    S = 4 if seg is not None else 1
    ws = torch.empty(max(B.tma_groupnorm_act_fwd_workspace_bytes(n, F, G, S, 0), B.tma_groupnorm_act_bwd_workspace_bytes(n, F, G, S, 0)),
                     dtype=torch.uint8, device="cuda")
    y, dx, dg, db = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(gamma), torch.zeros_like(beta)
    st = torch.zeros((4, G, 2), device="cuda") if seg is not None else None

    def passes(stream=None):
        B.tma_groupnorm_act_fwd(x, G, gamma, beta, B.TMA_ACT_SILU, segments=seg, out=y, stats_out=st, ws=ws, stream=stream)
        B.tma_groupnorm_act_bwd(x, dy, G, gamma, beta, B.TMA_ACT_SILU, segments=seg, stats=st, dX_out=dx, dgamma=dg, dbeta=db, ws=ws, stream=stream)

    outs = (y, dx, dg, db)
    passes()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    s = torch.cuda.Stream()
    for t in outs:
        t.zero_()
    s.wait_stream(torch.cuda.current_stream())
    passes(s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        passes()
    for k in range(4):
        x.copy_(torch.randn((n, F), generator=g))
        if seg is not None:
            seg.copy_(torch.tensor([[0, 0, 1, 2999, 3001], [5, 900, 901, 2000, 2500], [0, 3001, 3001, 3001, 3001], [1, 2, 3, 4, 5]][k]).int())
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in outs]
        ws.random_(0, 255)
        for t in outs:
            t.zero_()
        passes()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, replayed)), k


def test_gradient_against_differences(B):
    """L = sum(G (.) Y) along a random direction, central difference with step 2^-6 of a smooth layer in fp32: the quotient's own error is
    step^2 / 6 of the third derivative (below 30 |d|^3 per element here: 4e-5 x 30 of sum|G|) and the rounding of two passes."""
    c = Case(64, 4, 8, [0, 20, 64], torch.float32, "silu", 7)
    seg = torch.tensor(c.edges, dtype=torch.int32, device="cuda")
    x, dy, gamma, beta = c.x.cuda(), c.dy.cuda(), c.gamma.cuda(), c.beta.cuda()
    f = lambda x_, g_, b_: (B.tma_groupnorm_act_fwd(x_, 4, g_, b_, B.TMA_ACT_SILU, segments=seg)[0].double() * dy.double()).sum().item()
    _, st = B.tma_groupnorm_act_fwd(x, 4, gamma, beta, B.TMA_ACT_SILU, segments=seg)
    dx, dg, db, _ = B.tma_groupnorm_act_bwd(x, dy, 4, gamma, beta, B.TMA_ACT_SILU, segments=seg, stats=st)
    step, mass, g = 2.0 ** -6, dy.double().abs().sum().item(), torch.Generator().manual_seed(2)
    for at, (t, grad) in enumerate([(x, dx), (gamma, dg), (beta, db)]):
        d = (torch.rand(t.shape, generator=g) * 2 - 1).cuda()
        hi, lo = [x, gamma, beta], [x, gamma, beta]
        hi[at], lo[at] = t + step * d, t - step * d
        slope = (f(*hi) - f(*lo)) / (2 * step)
        assert abs(slope - (grad.double() * d.double()).sum().item()) <= (step * step / 6 * 30 + 4 * c.D * u * 4 / step) * mass


def test_rows_beyond_two_to_the_31_elements(B):
    n, F, G = 8_500_000, 256, 32
    x = torch.zeros((n, F), dtype=torch.bfloat16, device="cuda")
    c = Case(1000, G, F // G, list(range(1001)), torch.bfloat16, "prelu", 9)
    x[-1000:] = c.x.cuda()
    slope = torch.tensor([0.25], device="cuda")
    y, _ = B.tma_groupnorm_act_fwd(x, G, c.gamma.cuda(), c.beta.cuda(), B.TMA_ACT_PRELU, slope=slope, eps=EPS)
    close(y[-1000:].cpu(), c.out, c.tol, "far rows")
    edges = [0, n - 1000, n]
    s = Case(1000, G, F // G, [0, 1000], torch.bfloat16, "prelu", 9)
    y, st = B.tma_groupnorm_act_fwd(x, G, c.gamma.cuda(), c.beta.cuda(), B.TMA_ACT_PRELU, slope=slope, eps=EPS,
                                    segments=torch.tensor(edges, dtype=torch.int32, device="cuda"))
    close(y[-1000:].cpu(), s.out, s.tol, "far segment")
    assert not st[0, :, 0].any()


def test_no_rows(B):
    gamma, beta = torch.ones(8, device="cuda"), torch.ones(8, device="cuda")
    x = torch.empty((0, 8), device="cuda")
    for how in (dict(), dict(rows_per_segment=5), dict(segments=torch.zeros(3, dtype=torch.int32, device="cuda"))):
        y, st = B.tma_groupnorm_act_fwd(x, 2, gamma, beta, **how)
        assert y.shape == (0, 8)
        dx, dg, db, _ = B.tma_groupnorm_act_bwd(x, x, 2, gamma, beta, stats=st, **how)
        assert not dg.any() and not db.any() and dx.shape == (0, 8)
