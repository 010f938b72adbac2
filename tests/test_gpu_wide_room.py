"""Forward calls of wide layers allocate what they use: rows that are read where they lie take no room."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2305_09887_amd import binding
    binding.lib()
    return binding


def _peak(call):
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    out = call()
    torch.cuda.synchronize()
    return out, torch.cuda.max_memory_allocated() - before


@pytest.mark.parametrize("layer", ["gated", "residual"])
def test_what_a_call_allocates(B, layer):
    n, f = 200_000, 256
    g = torch.Generator(device="cuda").manual_seed(1)
    flat = torch.randint(-2, 3, (n * f + 8,), generator=g, device="cuda").bfloat16()
    W, Wu = (torch.randint(-1, 2, (f, f), generator=g, device="cuda").float() for _ in range(2))
    results = {}
    for off in (0, 1):                   # at 16 bytes, and not
        X = flat[off:off + n * f].view(n, f)
        if layer == "gated":
            call = lambda: B.tma_gated_dense_fwd(X, W, Wu, None, None, B.TMA_ACT_RELU, save=False)[0]
        else:
            call = lambda: B.tma_dense_residual_fwd(X, W, None, B.TMA_ACT_RELU, R=X)[0]
        results[off], peak = _peak(call)
        x = X.double()
        z = x @ W.double()
        want = z.clamp(min=0) * (x @ Wu.double()) if layer == "gated" else z.clamp(min=0) + x
        assert torch.equal(results[off], want.float().bfloat16())
        size = n * f * 2
        assert peak <= size + (8 << 20) if off == 0 else 2 * size <= peak <= 2 * size + (8 << 20)
