"""Dense layers with weights per group of rows, against the formulas in 64 bits.

Tolerances, element by element.  u = 2^-24, half a step of fp32; h = half a step of the storage type (2^-24, bf16 2^-8).  A sum
of K products in fp32, in whatever order, is off by at most (K + 2) u sum|a b| (K - 1 additions, a rounded product each, and
three exact parts of a value leave at most u of it); with bf16 storage the weights are rounded once, h sum|a b| more; the result
is rounded once, h of what it is."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
u = 2.0 ** -24


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2305_09887_amd import binding
    binding.lib()
    return binding


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def matrix(B, n, F, dtype, g, layout, scale=1.0):
    x = (torch.randn((n, F), generator=g) * scale).to(dtype)
    if layout == "padded":
        d = B._padded(n, F, dtype, "cuda")
    elif layout == "dense":
        d = torch.empty((n, F), dtype=dtype, device="cuda")
    else:       # an odd pitch, from the second element on
        d = torch.empty((n * (F + 3) + 1,), dtype=dtype, device="cuda")[1:].view(n, F + 3)[:, :F]
    d.copy_(x)
    return x.double(), d


class Case:
    def __init__(self, B, sizes, F_in, F_out, dtype, layout="padded", listed=True, loose=0, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.sizes = dtype, sizes
        m = sum(sizes)
        self.n = n = m + loose
        self.E = E = len(sizes)
        perm = torch.randperm(n, generator=g) if listed else torch.arange(n)
        self.rows = perm[:m].split(list(sizes))
        self.offsets = torch.tensor([0] + list(np.cumsum(sizes)), dtype=torch.int32, device="cuda")
        self.order = perm.int().cuda() if listed else None
        self.X, self.dX = matrix(B, n, F_in, dtype, g, layout)
        self.G, self.dG = matrix(B, n, F_out, dtype, g, layout, 0.5)
        self.H, self.dH = matrix(B, n, F_out, dtype, g, layout)
        self.W = torch.randn((E, F_in, F_out), generator=g) * 0.3
        self.b = torch.randn((E, F_out), generator=g)
        self.free = perm[m:]
        self.narrowed = 0.0 if dtype == torch.float32 else half_step(dtype)

    def forward(self, relu, bias=True):
        """{row: ...} as (rows, values, tolerance) per group"""
        h, K = half_step(self.dtype), self.X.shape[1]
        for e, r in enumerate(self.rows):
            w, b = self.W[e].double(), self.b[e].double() if bias else torch.zeros(self.W.shape[2], dtype=torch.float64)
            z = self.X[r] @ w + b
            mass = self.X[r].abs() @ w.abs() + b.abs()
            tol = ((K + 3) * u + self.narrowed) * mass
            yield r, (z.clamp(min=0) if relu else z), tol + h * (z.abs() + tol)


def close(got, want, tol, what):
    bad = (got.double() - want).abs() > tol
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {((got.double() - want).abs() / tol.clamp(min=1e-300)).max():.3g} tolerances"


SIZES = {"one": [1], "few": [3, 0, 1, 7, 2], "empty_ends": [0, 0, 40, 0, 65, 0], "single_rows": [1] * 37, "uneven": [130, 1, 0, 700, 64, 63],
         "large": [5000, 0, 1, 9000, 129], "all_empty": [0, 0, 0], "one_group": [2300]}
WIDTHS = [(1, 1), (5, 3), (16, 16), (47, 100), (64, 33), (100, 260), (150, 41), (128, 256), (300, 129), (530, 8)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("F_in,F_out", WIDTHS)
@pytest.mark.parametrize("name", list(SIZES))
def test_forward(B, name, F_in, F_out, dtype):
    for k, (layout, listed, relu, bias) in enumerate([("padded", True, True, True), ("dense", False, False, False), ("odd", True, False, True)]):
        c = Case(B, SIZES[name], F_in, F_out, dtype, layout, listed, loose=5 if listed else 0, seed=k)
        out = B._padded(c.n, F_out, dtype, "cuda").fill_(7.0)
        B.tma_grouped_dense_fwd(c.dX, c.W.cuda(), c.b.cuda() if bias else None, c.offsets, int(relu), order=c.order, Y_out=out)
        got = out.cpu()
        for r, want, tol in c.forward(relu, bias):
            close(got[r], want, tol, f"{name} {layout}")
        assert (got[c.free] == 7).all()          # rows of no group


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("F_in,F_out", WIDTHS)
@pytest.mark.parametrize("name", list(SIZES))
def test_backward(B, name, F_in, F_out, dtype):
    h = half_step(dtype)
    for k, (layout, listed, relu) in enumerate([("padded", True, True), ("dense", False, False), ("odd", True, True)]):
        c = Case(B, SIZES[name], F_in, F_out, dtype, layout, listed, loose=4 if listed else 0, seed=10 + k)
        dX = B._padded(c.n, F_in, dtype, "cuda").fill_(7.0)
        dW, db, _ = B.tma_grouped_dense_bwd(c.dX, c.dH if relu else None, c.dG, c.W.cuda(), c.offsets, int(relu), order=c.order, dX_out=dX)
        dW, db, dX = dW.cpu(), db.cpu(), dX.cpu()
        for e, r in enumerate(c.rows):
            z = c.G[r] * (c.H[r] > 0) if relu else c.G[r]
            x, w, m = c.X[r], c.W[e].double(), len(r)
            close(dW[e], x.T @ z, (m + 2) * u * (x.abs().T @ z.abs()), f"dW {name} {layout}")
            close(db[e], z.sum(0), (m + 2) * u * z.abs().sum(0), f"db {name} {layout}")
            want = z @ w.T
            tol = ((F_out + 3) * u + c.narrowed) * (z.abs() @ w.abs().T)
            close(dX[r], want, tol + h * (want.abs() + tol), f"dX {name} {layout}")
        assert (dX[c.free] == 7).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_optional_results_and_repeatability(B, dtype):
    c = Case(B, SIZES["uneven"], 70, 90, dtype, loose=3, seed=5)
    args = (c.dX, c.dH, c.dG, c.W.cuda(), c.offsets, B.TMA_ACT_RELU)
    full = B.tma_grouped_dense_bwd(*args, order=c.order)
    assert B.tma_grouped_dense_bwd(*args, order=c.order, need_dbias=False, need_dX=False)[1:] == (None, None)
    for _ in range(2):
        again = B.tma_grouped_dense_bwd(*args, order=c.order)
        assert torch.equal(full[0], again[0]) and torch.equal(full[1], again[1])
        listed = torch.cat(c.rows).cuda()
        assert torch.equal(full[2][listed], again[2][listed])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes", [[9, 4], [900, 0, 300]])
def test_infinities_and_nan_stay_in_their_rows(B, dtype, sizes):
    c = Case(B, sizes, 40, 24, dtype, loose=2, seed=6)
    x = c.dX
    bad = int(c.rows[0][3])
    x[bad, 7] = float("inf")
    nan = int(c.rows[0][1])
    x[nan, 0] = float("nan")
    x[c.free.cuda()] = float("nan")              # rows of no group
    Y = B.tma_grouped_dense_fwd(x, c.W.cuda(), c.b.cuda(), c.offsets, B.TMA_ACT_NONE, order=c.order).cpu()
    assert torch.isnan(Y[nan]).all()
    w = c.W[0][7]
    assert torch.equal(Y[bad].double(), torch.where(w > 0, float("inf"), float("-inf")).double())
    for r, want, tol in c.forward(False):
        keep = (r != bad) & (r != nan)
        close(Y[r][keep], want[keep], tol[keep], "other rows")
    # a gradient that a ReLU masks counts for nothing, whatever it is
    c.dG[bad] = float("nan")
    c.dH[bad] = -1.0
    x[bad], x[nan] = 0.0, 0.0
    dW, db, dX = B.tma_grouped_dense_bwd(x, c.dH, c.dG, c.W.cuda(), c.offsets, B.TMA_ACT_RELU, order=c.order)
    assert torch.isfinite(dW).all() and torch.isfinite(db).all() and not dX[bad].any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_values_at_both_ends_of_the_range(B, dtype):
    """The bounds are relative to the sums of magnitudes, so they hold for gradients of 1e-30 and activations of 1e30 alike."""
    h = half_step(dtype)
    for scale in (2.0 ** -96, 2.0 ** 96):
        c = Case(B, [300, 0, 77], 65, 72, dtype, seed=8)
        c.dX.mul_(scale)
        Y = B.tma_grouped_dense_fwd(c.dX, c.W.cuda(), None, c.offsets, B.TMA_ACT_NONE, order=c.order).cpu()
        for r, want, tol in c.forward(False, bias=False):
            close(Y[r].double() / scale, want, tol, f"scale {scale}")
        dW, _, _ = B.tma_grouped_dense_bwd(c.dX, None, c.dG, c.W.cuda(), c.offsets, B.TMA_ACT_NONE, order=c.order)
        for e, r in enumerate(c.rows):
            close(dW[e].cpu().double() / scale, c.X[r].T @ c.G[r], (len(r) + 2) * u * (c.X[r].abs().T @ c.G[r].abs()), f"dW scale {scale}")


@pytest.mark.parametrize("sizes", [[3, 1, 0, 6], [2000, 0, 900, 64]])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_on_a_stream_of_its_own_and_replayed_in_a_graph(B, dtype, sizes):
    c = Case(B, sizes, 96, 80, dtype, loose=3, seed=9)
    W, b, F = c.W.cuda(), c.b.cuda(), B._feat_dtype(c.dX)
    ws = torch.empty(max(B.tma_grouped_dense_fwd_workspace_bytes(c.n, c.E, 96, 80, F), B.tma_grouped_dense_bwd_workspace_bytes(c.n, c.E, 96, 80, F)),
                     dtype=torch.uint8, device="cuda")
    Y, dX = torch.zeros_like(c.dG), torch.zeros_like(c.dX)
    dW, db = torch.zeros_like(W), torch.zeros_like(b)

    def passes(stream=None):
        B.tma_grouped_dense_fwd(c.dX, W, b, c.offsets, B.TMA_ACT_RELU, order=c.order, Y_out=Y, ws=ws, stream=stream)
        B.tma_grouped_dense_bwd(c.dX, Y, c.dG, W, c.offsets, B.TMA_ACT_RELU, order=c.order, dW=dW, dbias=db, dX_out=dX, ws=ws, stream=stream)

    passes()
    torch.cuda.synchronize()
    want = [t.clone() for t in (Y, dW, db, dX)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for t in (Y, dW, db, dX):
        t.zero_()
    s.wait_stream(torch.cuda.current_stream())
    passes(s)
    s.synchronize()
    assert all(torch.equal(a, b_) for a, b_ in zip((Y, dW, db, dX), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        passes()
    # other sizes of the groups at every replay: they live on the device
    m, held = sum(sizes), c.offsets.clone()
    for k in range(4):
        cut = torch.sort(torch.randint(0, m + 1, (c.E - 1,), generator=torch.Generator().manual_seed(k))).values
        c.offsets.copy_(held if k == 3 else torch.cat([torch.tensor([0]), cut, torch.tensor([m])]).int())
        for t in (Y, dW, db, dX):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in (Y, dW, db, dX)]
        for t in (Y, dW, db, dX):
            t.zero_()
        passes()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b_) for a, b_ in zip((Y, dW, db, dX), replayed)), k
        ws.random_(0, 255)                        # nothing in the workspace outlives a call
    assert all(torch.equal(a, b_) for a, b_ in zip(replayed, want))


def test_rows_beyond_two_to_the_31_elements(B):
    n, F = 8_500_000, 256
    X = torch.zeros((n, F), dtype=torch.bfloat16, device="cuda")
    far = torch.arange(n - 500, n, device="cuda")
    g = torch.Generator().manual_seed(1)
    x = torch.randn((500, F), generator=g).bfloat16()
    X[far] = x.cuda()
    order = torch.zeros(n, dtype=torch.int32, device="cuda")
    order[:500] = far.int()
    offsets = torch.tensor([0, 200, 500], dtype=torch.int32, device="cuda")
    W = torch.randn((2, F, 16), generator=g) * 0.1
    Y = torch.zeros((n, 16), dtype=torch.bfloat16, device="cuda")
    B.tma_grouped_dense_fwd(X, W.cuda(), None, offsets, B.TMA_ACT_NONE, order=order, Y_out=Y)
    for e, (a, b) in enumerate([(0, 200), (200, 500)]):
        want, mass = x[a:b].double() @ W[e].double(), x[a:b].double().abs() @ W[e].double().abs()
        tol = ((F + 3) * u + 2.0 ** -8) * mass
        close(Y[far[a:b]].cpu(), want, tol + 2.0 ** -8 * (want.abs() + tol), "far rows")
    assert not Y[:n - 500].any()
    dY = torch.zeros_like(Y)
    dY[far] = 1.0
    del Y
    dX = torch.zeros_like(X)
    dW, db, _ = B.tma_grouped_dense_bwd(X, None, dY, W.cuda(), offsets, B.TMA_ACT_NONE, order=order, dX_out=dX)
    assert torch.equal(db.cpu(), torch.tensor([[200.0] * 16, [300.0] * 16]))
    want = torch.ones((200, 16), dtype=torch.float64) @ W[0].double().T
    tol = (19 * u + 2.0 ** -8) * (torch.ones((200, 16), dtype=torch.float64) @ W[0].double().abs().T)
    close(dX[far[:200]].cpu(), want, tol + 2.0 ** -8 * (want.abs() + tol), "far gradients")
    assert not dX[:n - 500].any()


def test_gradients_against_differences(B):
    """L = sum(G (.) Y): the gradient along a random direction against a central difference of the fp32 forward pass.  The layer is
    linear in each operand (no ReLU), so the quotient has no error of its own, only the rounding of two passes: at most
    2 (K + 4) u sum|G| |X| |W| / step."""
    c = Case(B, [200, 0, 333], 30, 20, torch.float32, seed=12)
    W, b = c.W.cuda(), c.b.cuda()
    dW, db, dX = B.tma_grouped_dense_bwd(c.dX, None, c.dG, W, c.offsets, B.TMA_ACT_NONE, order=c.order)
    f = lambda X, W_, b_: (B.tma_grouped_dense_fwd(X, W_, b_, c.offsets, B.TMA_ACT_NONE, order=c.order).double() * c.dG.double()).sum().item()
    mass = (c.dG.double().abs() * B.tma_grouped_dense_fwd(c.dX.abs(), W.abs(), b.abs(), c.offsets, B.TMA_ACT_NONE, order=c.order).double()).sum().item()
    g = torch.Generator().manual_seed(3)
    step = 1.0
    for t, grad, at in [(c.dX, dX, 0), (W, dW, 1), (b, db, 2)]:
        d = torch.randn(t.shape, generator=g).cuda()
        args = [c.dX, W, b]
        hi, lo = list(args), list(args)
        hi[at], lo[at] = t + step * d, t - step * d
        slope = (f(*hi) - f(*lo)) / (2 * step)
        assert abs(slope - (grad.double() * d.double()).sum().item()) <= 8 * 34 * u * mass * 4


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_offsets_that_descend_touch_nothing_else(B, dtype):
    """Not a list that tma_group_rows writes, so the results are anything: but they stay in the outputs, and the call ends."""
    n, E, F_in, F_out = 3000, 64, 40, 24
    g = torch.Generator().manual_seed(5)
    W = torch.randn(E, F_in, F_out, generator=g).cuda()
    offsets = torch.tensor([0, n] * (E // 2) + [0], dtype=torch.int32, device="cuda")
    whole = {F: torch.full((n + 64, 48), 3.0, dtype=dtype, device="cuda") for F in (F_in, F_out)}
    X = torch.ones(n, F_in, dtype=dtype, device="cuda")
    dY = torch.ones(n, 48, dtype=dtype, device="cuda")[:, :F_out]
    Y, dX = whole[F_out][32:32 + n, :F_out], whole[F_in][32:32 + n, :F_in]
    B.tma_grouped_dense_fwd(X, W, None, offsets, B.TMA_ACT_RELU, Y_out=Y)
    B.tma_grouped_dense_bwd(X, Y, dY, W, offsets, B.TMA_ACT_RELU, dX_out=dX)
    torch.cuda.synchronize()
    for F, t in whole.items():
        assert (t[:32] == 3).all() and (t[32 + n:] == 3).all() and (t[:, F:] == 3).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("F_in,F_out", [(40, 24), (260, 130)])
def test_weight_gradients_of_infinities_and_of_values_near_the_range_end(B, dtype, F_in, F_out):
    c = Case(B, [900, 0, 300], F_in, F_out, dtype, seed=9)
    bad, large = int(c.rows[0][5]), int(c.rows[2][7])
    c.dX[bad, 7], c.dX[large, 3] = float("inf"), 2.0 ** 120
    c.X[large, 3] = 2.0 ** 120
    c.X[bad, 7] = 0.0                            # (not looked at)
    dW, db, _ = B.tma_grouped_dense_bwd(c.dX, None, c.dG, c.W.cuda(), c.offsets, B.TMA_ACT_NONE, order=c.order)
    g = c.G[bad]
    want = torch.where(g > 0, float("inf"), torch.where(g < 0, float("-inf"), float("nan")))
    assert torch.equal(dW[0, 7].cpu().double().nan_to_num(nan=0.5, posinf=1.0, neginf=-1.0), want.nan_to_num(nan=0.5, posinf=1.0, neginf=-1.0))
    for e, r in enumerate(c.rows):
        keep = torch.ones(F_in, dtype=torch.bool)
        if e == 0:
            keep[7] = False
        tol = (len(r) + 2) * u * (c.X[r].abs().T @ c.G[r].abs())
        close(dW[e].cpu()[keep], (c.X[r].T @ c.G[r])[keep], tol[keep], f"dW of group {e}")
        close(db[e].cpu(), c.G[r].sum(0), (len(r) + 2) * u * c.G[r].abs().sum(0), "db")


LONG = [([90_000, 0, 1, 120_000, 333], 33, 50), ([200_003], 128, 64), ([17_000, 40, 0, 9_000], 20, 2_100), ([30_000, 5, 25_000], 300, 510),
        ([30_000, 5, 25_000], 510, 250), ([900, 3, 700], 1_300, 70), ([900, 3, 700], 70, 1_300)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes,F_in,F_out", LONG)
def test_long_lists_and_wide_products(B, sizes, F_in, F_out, dtype):
    """Lists that are long, or products that are wide, enough for weights in LDS, and some too wide for that: results, masked and plain gradients, infinities."""
    h = half_step(dtype)
    for k, (layout, relu) in enumerate([("padded", True), ("odd", False)]):
        c = Case(B, sizes, F_in, F_out, dtype, layout, loose=3, seed=30 + k)
        look = [r[torch.cat([torch.arange(min(len(r), 300)), torch.arange(max(len(r) - 300, 0), len(r))])] for r in c.rows]      # of each group
        out = B._padded(c.n, F_out, dtype, "cuda").fill_(7.0)
        B.tma_grouped_dense_fwd(c.dX, c.W.cuda(), c.b.cuda(), c.offsets, int(relu), order=c.order, Y_out=out)
        dX = B._padded(c.n, F_in, dtype, "cuda").fill_(7.0)
        B.tma_grouped_dense_bwd(c.dX, c.dH if relu else None, c.dG, c.W.cuda(), c.offsets, int(relu), order=c.order, dX_out=dX)
        for e, r in enumerate(look):
            x, w, z = c.X[r], c.W[e].double(), c.G[r] * (c.H[r] > 0) if relu else c.G[r]
            want, mass = x @ w + c.b[e].double(), x.abs() @ w.abs() + c.b[e].double().abs()
            tol = ((F_in + 3) * u + c.narrowed) * mass
            want = want.clamp(min=0) if relu else want
            close(out[r.cuda()].cpu(), want, tol + h * (want.abs() + tol), f"Y {layout}")
            want = z @ w.T
            tol = ((F_out + 3) * u + c.narrowed) * (z.abs() @ w.abs().T)
            close(dX[r.cuda()].cpu(), want, tol + h * (want.abs() + tol), f"dX {layout}")
        assert (out[c.free.cuda()] == 7).all() and (dX[c.free.cuda()] == 7).all()
        bad = int(c.rows[0][77])
        c.dX[bad, F_in - 1] = float("inf")
        again = B._padded(c.n, F_out, dtype, "cuda").fill_(7.0)
        B.tma_grouped_dense_fwd(c.dX, c.W.cuda(), None, c.offsets, 0, order=c.order, Y_out=again)
        w = c.W[0, -1]
        assert torch.equal(again[bad].cpu().double(), torch.where(w > 0, float("inf"), float("-inf")).double())
        finite = torch.isfinite(again.float()).all(1)
        assert int((~finite).sum()) == 1 and not finite[bad]
