"""What the calls for wide layers may be given twice: results over the gradients that come in, a layer's own rows as what goes past it.  Small whole numbers, exact."""
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


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("n,F", [(1, 16), (40, 33), (64, 200), (65, 200), (130, 2048), (3000, 96), (8200, 1024)])
def test_one_buffer_in_two_places(B, n, F, dtype):
    g = torch.Generator(device="cuda").manual_seed(n)
    X, W, Wu, dY, Z, U = whole(g, n, F), whole(g, F, F, top=1), whole(g, F, F, top=1), whole(g, n, F, top=1), whole(g, n, F, top=1), whole(g, n, F, top=1)
    x, w, wu, z, u = X.to(dtype), W.float(), Wu.float(), Z.to(dtype), U.to(dtype)
    # what goes past the layer is its input
    y, _ = B.tma_dense_residual_fwd(x, w, None, B.TMA_ACT_RELU, R=x)
    assert torch.equal(y, ((X @ W).clamp(min=0) + X).float().to(dtype)) and torch.equal(x.double(), X)
    # the input's gradient over the output's, which went past the layer too
    for act, dZ in ((B.TMA_ACT_NONE, dY), (B.TMA_ACT_RELU, dY * (Z > 0))):
        dy = dY.to(dtype)
        dW, db, dX = B.tma_dense_residual_bwd(x, z, dy, w, act, R=dy, dX_out=dy)
        assert dX is dy and torch.equal(dX, (dZ @ W.t() + dY).float().to(dtype))
        assert torch.equal(dW.double(), X.t() @ dZ) and torch.equal(db.double(), dZ.sum(0))
    # gated: the gradient that comes in is also added; rows, gate and gradient are one
    dh = dY.to(dtype)
    dG, dU = dY * U * (Z > 0), dY * Z.clamp(min=0)
    got = B.tma_gated_dense_bwd(x, z, u, dh, w, wu, B.TMA_ACT_RELU, R=dh)
    assert torch.equal(got[4], (dG @ W.t() + dU @ Wu.t() + dY).float().to(dtype)) and torch.equal(dh.double(), dY)
    got = B.tma_gated_dense_bwd(z, z, z, z, w, w, B.TMA_ACT_NONE, R=z)
    assert torch.equal(got[0].double(), Z.t() @ (Z * Z)) and torch.equal(got[1], got[0])
    assert torch.equal(got[4], (2 * ((Z * Z) @ W.t()) + Z).float().to(dtype))
