"""Wide layers whose widths and rows end anywhere in a group of eight units: small whole numbers, which are exact in every step, with workspaces full of NaN, so that a
misplaced unit or one that was never written shows."""
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


def whole(g, *shape, top=2):
    return torch.randint(-top, top + 1, shape, generator=g, device="cuda").double()


def room(nbytes):
    return torch.full((nbytes // 4,), math.nan, device="cuda")


# small tiles; large tiles (bf16: rows enough for three quarters of the chip) forward, along rows and of weights; ranges of k
SHAPES = [(300, 8, 8), (999, 40, 100), (5000, 32, 288), (5000, 288, 32), (2100, 260, 500), (700, 736, 1000), (3100, 33, 257), (8100, 544, 2016), (8100, 2016, 544),
          (16_300, 2016, 1056), (90, 4096, 300), (129, 3000, 290)]


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("n,fi,fo", SHAPES)
def test_gated(B, n, fi, fo, dtype):
    g = torch.Generator(device="cuda").manual_seed(n + fi)
    code = B._feat_dtype(torch.empty(0, dtype=dtype, device="cuda"))
    X, Wg, Wu = whole(g, n, fi), whole(g, fi, fo, top=1), whole(g, fi, fo, top=1)
    x, wg, wu = X.to(dtype), Wg.float(), Wu.float()
    ws = room(B.tma_gated_dense_fwd_workspace_bytes(n, fi, fo, code))
    h, G, U = B.tma_gated_dense_fwd(x, wg, wu, None, None, B.TMA_ACT_RELU, ws=ws)
    for got, want in ((G, X @ Wg), (U, X @ Wu), (h, (X @ Wg).clamp(min=0) * (X @ Wu))):
        assert torch.equal(got, want.float().to(dtype))
    del h
    G, U, dH = whole(g, n, fo, top=1), whole(g, n, fo, top=1), whole(g, n, fo, top=1)
    ws = room(B.tma_gated_dense_bwd_workspace_bytes(n, fi, fo, code, True))
    got = B.tma_gated_dense_bwd(x, G.to(dtype), U.to(dtype), dH.to(dtype), wg, wu, B.TMA_ACT_RELU, R=x, ws=ws)
    dG, dU = dH * U * (G > 0), dH * G.clamp(min=0)
    for t, want in zip(got[:4], (X.t() @ dG, X.t() @ dU, dG.sum(0), dU.sum(0))):
        assert torch.equal(t.double(), want)
    assert torch.equal(got[4], (dG @ Wg.t() + dU @ Wu.t() + X).float().to(dtype))


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("n,fi,fo", SHAPES)
def test_residual(B, n, fi, fo, dtype):
    g = torch.Generator(device="cuda").manual_seed(n + fo)
    code = B._feat_dtype(torch.empty(0, dtype=dtype, device="cuda"))
    X, W, R = whole(g, n, fi), whole(g, fi, fo, top=1), whole(g, n, fo)
    x, w, r = X.to(dtype), W.float(), R.to(dtype)
    ws = room(B.tma_dense_residual_fwd_workspace_bytes(n, fi, fo, code))
    y, z = B.tma_dense_residual_fwd(x, w, None, B.TMA_ACT_RELU, R=r, save=True, ws=ws)
    assert torch.equal(z, (X @ W).float().to(dtype)) and torch.equal(y, ((X @ W).clamp(min=0) + R).float().to(dtype))
    for act, Z in ((B.TMA_ACT_RELU, whole(g, n, fo)), (B.TMA_ACT_NONE, None)):
        dY = whole(g, n, fo)
        ws = room(B.tma_dense_residual_bwd_workspace_bytes(n, fi, fo, act, code, True))
        dW, db, dX = B.tma_dense_residual_bwd(x, None if Z is None else Z.to(dtype), dY.to(dtype), w, act, R=x, ws=ws)
        dZ = dY if Z is None else dY * (Z > 0)
        assert torch.equal(dW.double(), X.t() @ dZ) and torch.equal(db.double(), dZ.sum(0))
        assert torch.equal(dX, (dZ @ W.t() + X).float().to(dtype))
