"""Dropout: mask and values against the written rule in unsigned 64-bit integers, bit for bit (one product in fp32, one
rounding to storage, as the plain form's)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
U = np.uint64


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2305_09887_amd import binding
    binding.lib()
    return binding


def mix(seed, unit):
    with np.errstate(over="ignore"):
        z = U(seed & (2**64 - 1)) + (unit.astype(U) + U(1)) * U(0x9E3779B97F4A7C15)
        z = (z ^ (z >> U(30))) * U(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> U(27))) * U(0x94D049BB133111EB)
        return z ^ (z >> U(31))


def plain(x, p, seed, step=None, first_row=0):
    n, F = x.shape
    if step is not None:
        seed = int(mix(seed, np.array([step & (2**64 - 1)], dtype=U))[0])
    units = (F + 3) // 4
    rows = (np.arange(n, dtype=U) + U(first_row))[:, None] * U(units)
    z = mix(seed, rows + np.arange(units, dtype=U)[None, :])
    field = np.stack([(z >> U(16 * k)) & U(0xFFFF) for k in range(4)], 2).reshape(n, 4 * units)[:, :F]
    limit = int(np.floor(p * 65536 + 0.5))
    scale = np.float32(65536 / (65536 - limit)) if limit < 65536 else np.float32(0)
    keep = torch.from_numpy(field >= limit)
    return torch.where(keep, x.float() * torch.tensor(scale), torch.zeros(())).to(x.dtype)


def rows(B, n, F, dtype, seed, layout):
    x = torch.randn((n, F), generator=torch.Generator().manual_seed(seed)).to(dtype)
    if layout == "padded":
        d = B._padded(n, F, dtype, "cuda")
    elif layout == "dense":
        d = torch.empty((n, F), dtype=dtype, device="cuda")
    else:       # an odd pitch, from the second element on
        d = torch.empty((n * (F + 3) + 1,), dtype=dtype, device="cuda")[1:].view(n, F + 3)[:, :F]
    d.copy_(x)
    return x, d


@pytest.mark.parametrize("layout", ["padded", "dense", "odd"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,F", [(1, 1), (3, 5), (1000, 47), (130, 64), (257, 150), (33, 1030), (5, 2500), (40001, 16)])
def test_values_are_the_rules(B, n, F, dtype, layout):
    x, d = rows(B, n, F, dtype, n + F, layout)
    for p, seed, step, first in [(0.5, 1, None, 0), (0.1, 2**64 - 5, 77, 0), (0.83, 12345, 2**40, 10**10), (0.0, 3, None, 0), (1.0, 4, 0, 2)]:
        t = torch.tensor([step], dtype=torch.int64, device="cuda") if step is not None else None
        want = plain(x, p, seed, step, first)
        got = B.tma_dropout_fwd(d, p, seed, step=t, first_row=first)
        assert torch.equal(got.cpu(), want), (p, seed)
        assert torch.equal(B.tma_dropout_bwd(d, p, seed, step=t, first_row=first).cpu(), want)      # one mask for both directions


def test_in_place_leaves_padding_and_other_rows(B):
    held = torch.full((70, 48), 9.0, device="cuda")
    view = held[3:60, :47]
    x = torch.randn((57, 47), generator=torch.Generator().manual_seed(1))
    view.copy_(x)
    assert B.tma_dropout_fwd(view, 0.4, 11, out=view) is view
    assert torch.equal(view.cpu(), plain(x, 0.4, 11))
    assert (held[:3] == 9).all() and (held[60:] == 9).all() and (held[:, 47] == 9).all()


def test_dropped_infinities_are_zero_and_kept_ones_stay(B):
    x = torch.full((64, 64), float("inf"))
    x[::2] = float("nan")
    got = B.tma_dropout_fwd(x.cuda(), 0.5, 5).cpu()
    mask = plain(torch.ones(64, 64), 0.5, 5) != 0
    assert (got[~mask] == 0).all()
    assert torch.isnan(got[::2][mask[::2]]).all() and torch.isinf(got[1::2][mask[1::2]]).all()


def test_share_of_dropped_elements_and_independence_of_steps(B):
    """Counts of n Bernoulli draws lie within six standard deviations; two steps' masks agree as independent ones do."""
    n, p = 2_000_000, 0.3
    x = torch.ones((n // 16, 16), device="cuda")
    masks = [B.tma_dropout_fwd(x, p, 9, step=torch.tensor([k], device="cuda")) == 0 for k in (1, 2)]
    for m in masks:
        assert abs(m.sum().item() - n * p) < 6 * (n * p * (1 - p)) ** 0.5
    both = (masks[0] & masks[1]).sum().item()
    assert abs(both - n * p * p) < 6 * (n * p * p * (1 - p * p)) ** 0.5


def test_blocks_of_rows_draw_what_the_whole_does(B):
    x, d = rows(B, 300, 30, torch.float32, 2, "padded")
    whole = B.tma_dropout_fwd(d, 0.5, 8).cpu()
    for a, b in [(0, 100), (100, 101), (101, 300)]:
        assert torch.equal(B.tma_dropout_fwd(d[a:b], 0.5, 8, first_row=a).cpu(), whole[a:b])


def test_a_replayed_graph_draws_anew_where_the_step_advances(B):
    x, d = rows(B, 501, 33, torch.bfloat16, 4, "padded")
    step, out = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.empty_like(d)
    B.tma_dropout_fwd(d, 0.25, 6, step=step, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.tma_dropout_fwd(d, 0.25, 6, step=step, out=out)
        step.add_(1)
    for k in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert int(step) == k + 1
        assert torch.equal(out.cpu(), plain(x, 0.25, 6, k))


def test_rows_beyond_two_to_the_31_elements(B):
    n, F = 8_500_000, 256            # 2.2e9 elements: byte offsets pass 2^32
    d = torch.zeros((n, F), dtype=torch.bfloat16, device="cuda")
    d[-1000:] = 1.0
    B.tma_dropout_fwd(d, 0.5, 3, out=d)
    want = plain(torch.ones((1000, F), dtype=torch.bfloat16), 0.5, 3, first_row=n - 1000)
    assert torch.equal(d[-1000:].cpu(), want) and not d[:1000].any()


def test_no_rows(B):
    assert B.tma_dropout_fwd(torch.empty((0, 8), device="cuda"), 0.5, 1).shape == (0, 8)
