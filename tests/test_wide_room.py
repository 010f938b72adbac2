"""Forward products of wide layers that read bf16 rows where they lie ask for no room to lay those rows out: in host code, nothing here touches a device."""
import pytest

from test_layer_refusals import lib, refused  # noqa: F401
from test_wide_refusals import A, P, gated_fwd, res_fwd

CALLS = [(gated_fwd, "tma_gated_dense_fwd", "H", 2), (res_fwd, "tma_dense_residual_fwd", "Y", 1)]
N, F_IN, F_OUT = 1_000_003, 256, 256


def queries(lib, name, *sizes):
    return getattr(lib, name + "_workspace_bytes")(*sizes), getattr(lib, name + "_workspace_bytes_at16")(*sizes)


@pytest.mark.parametrize("call,name,out,sides", CALLS)
def test_rows_at_16_bytes(lib, call, name, out, sides):
    whole, at16 = queries(lib, name, N, F_IN, F_OUT, 1)
    assert whole >= 2 * N * F_IN and at16 <= 2 * F_IN * sides * F_OUT + 4096 and at16 % 256 == 0
    sizes = dict(n=N, F_in=F_IN, F_out=F_OUT, dtype=1, ldx=F_IN, ws_bytes=at16, **{k: F_OUT for k in (("ldg", "ldh") if out == "H" else ("ldr", "ldz", "ldy"))})
    # past the workspace's check, to the next one
    refused(lib, call(lib, **sizes, **{out: None}), -1, b"NULL")
    refused(lib, call(lib, **{**sizes, "ldx": F_IN + 8}, **{out: None}), -1, b"NULL")
    refused(lib, call(lib, **{**sizes, "ws_bytes": at16 - 256}), -3, b"workspace")
    for other in (dict(X=P(4096 + 2)), dict(ldx=F_IN + 1), dict(ldx=(1 << 22) + 8)):
        refused(lib, call(lib, **{**sizes, **other}), -3, b"workspace")
        refused(lib, call(lib, **{**sizes, **other, "ws_bytes": whole}, **{out: None}), -1, b"NULL")


@pytest.mark.parametrize("call,name,out,sides", CALLS)
def test_where_rows_are_laid_out_in_any_case(lib, call, name, out, sides):
    for sizes in ((N, 256, 256, 0), (N, 250, 256, 1), (1000, 64, 65536, 1)):      # fp32; a width that is no multiple of 32; many columns
        whole, at16 = queries(lib, name, *sizes)
        assert whole == at16 > 2 * sizes[0] * sizes[1]
    for sizes in ((1, 4096, 1024, 0), (64, 300, 20000, 1), (0, 256, 256, 1)):      # few rows: nothing is laid out
        whole, at16 = queries(lib, name, *sizes)
        assert whole == at16
    for sizes in ((-1, 8, 8, 1), (1 << 31, 8, 8, 1), (100, 0, 8, 1), (100, 8, 65537, 1)):
        assert queries(lib, name, *sizes) == (0, 0)
