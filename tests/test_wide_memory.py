"""What the calls for wide layers ask of memory: laid-out operands take their own size in bf16 parts, rounded up to units of 32 by 16, however narrow the layer.
In host code: nothing here touches a device."""
import pytest

from test_layer_refusals import lib  # noqa: F401

SIZES = [(250_000, 8, 8), (2_400_000, 32, 32), (12_500_000, 32, 32), (1_000_003, 300, 40), (1_000_000, 33, 257), (700_000, 288, 96), (100_000, 1, 1), (300_000, 513, 8)]


def up(x, m):
    return (x + m - 1) // m * m


def small(n, F_in, F_out, sides):
    """Everything but rows laid out: weights, sums of columns, at most 512 ranges' shares of the weights' gradients."""
    weights = 3 * 2 * up(F_in, 32) * (sides * up(F_out, 32) + 32)
    sums = (4096 + 64) * sides * up(F_out, 32) * 4
    shares = 512 * sides * F_in * F_out * 4
    planes = 9 * 65536          # of three operands, each rounded up to 64 KB
    return weights + sums + shares + planes + 8 * 256


@pytest.mark.parametrize("n,F_in,F_out", SIZES)
@pytest.mark.parametrize("dtype", [0, 1], ids=["f32", "bf16"])
def test_backward(lib, n, F_in, F_out, dtype):
    rows, parts = up(n, 32), 1 if dtype else 3
    for sides, query in ((1, lambda dx: lib.tma_dense_residual_bwd_workspace_bytes(n, F_in, F_out, 3, dtype, dx)),
                         (2, lambda dx: lib.tma_gated_dense_bwd_workspace_bytes(n, F_in, F_out, dtype, dx))):
        laid_out = 2 * rows * (parts * up(F_in, 32) + (2 if dtype else 3) * sides * up(F_out, 32))
        for dx in (0, 1):
            assert laid_out <= query(dx) <= laid_out + small(n, F_in, F_out, sides), (sides, dx, query(dx), laid_out)


@pytest.mark.parametrize("n,F_in,F_out", SIZES)
@pytest.mark.parametrize("dtype", [0, 1], ids=["f32", "bf16"])
def test_forward(lib, n, F_in, F_out, dtype):
    for sides, query in ((1, lib.tma_dense_residual_fwd_workspace_bytes), (2, lib.tma_gated_dense_fwd_workspace_bytes)):
        laid_out = 2 * up(n, 32) * (1 if dtype else 3) * up(F_in, 32)
        assert query(n, F_in, F_out, dtype) <= laid_out + small(n, F_in, F_out, sides)


def test_a_wide_layer_of_one_unit_more_than_eight(lib):
    """288 columns are nine units, not sixteen."""
    n = 1_000_000
    grows = [lib.tma_dense_residual_bwd_workspace_bytes(n, F, 32, 3, 0, 1) for F in (256, 288, 320)]
    for a, b in zip(grows, grows[1:]):
        assert b - a <= 3 * 2 * up(n, 32) * 32 + (1 << 20)
