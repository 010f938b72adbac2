"""Sizes at and past the ends of what the calls for layers of several kinds of rows take, in host code: a size, or a refusal, and never the end of the process."""
import ctypes
import itertools
import os

import pytest

i64, i32, sz = ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t
FAKE, OTHER = ctypes.c_void_p(4096), ctypes.c_void_p(8192)      # never dereferenced
NS = [-1, 0, 1, 100, 10**6, 2**31 - 1, 2**31, 2**63 - 1]
ES = [-1, 0, 1, 50, 1024, 1025, 2**31 - 1]
FS = [-1, 0, 1, 65, 4096, 65536, 65537, 2**24, 2**30, 2**31 - 1]


@pytest.fixture(scope="module")
def lib():
    from paper_2305_09887_amd import binding, build
    if not os.path.exists(build.LIB):
        build.build(verbose=False)
    return binding.lib()


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("n", NS)
def test_workspaces_of_grouped_dense(lib, n, dtype):
    for E, fi, fo in itertools.product(ES, FS, FS):
        taken = 0 <= n < 2**31 and 1 <= E <= 1024 and 1 <= fi <= 65536 and 1 <= fo <= 65536
        need = [lib.tma_grouped_dense_fwd_workspace_bytes(i64(n), i32(E), i32(fi), i32(fo), i32(dtype))]
        need += [lib.tma_grouped_dense_bwd_workspace_bytes(i64(n), i32(E), i32(fi), i32(fo), i32(dtype), i32(k)) for k in (0, 1)]
        for b in need:
            assert b % 256 == 0 and (b >= 256 if taken else b == 0), (n, E, fi, fo, need)


@pytest.mark.parametrize("F_in,F_out", [(2**31 - 1, 8), (8, 2**31 - 1), (65537, 8), (8, 65537)])
@pytest.mark.parametrize("dtype", [0, 1])
def test_grouped_dense_refuses_such_widths(lib, dtype, F_in, F_out):
    ld = i64(2**31)
    fwd = lib.tma_grouped_dense_fwd(i64(100), i32(1), FAKE, None, FAKE, ld, i32(F_in), FAKE, None, i32(F_out), i32(0), i32(dtype), OTHER, ld, FAKE, sz(1 << 50), None)
    assert fwd == -2 and b"F_in=%d F_out=%d" % (F_in, F_out) in lib.tma_last_error()
    bwd = lib.tma_grouped_dense_bwd(i64(100), i32(1), FAKE, None, FAKE, ld, None, FAKE, ld, FAKE, i32(F_in), i32(F_out), i32(0), i32(dtype), FAKE, None, OTHER, ld,
                                    FAKE, sz(1 << 50), None)
    assert bwd == -2 and b"F_in=%d F_out=%d" % (F_in, F_out) in lib.tma_last_error()


@pytest.mark.parametrize("dtype", [0, 1])
def test_workspaces_of_group_norm_and_rows(lib, dtype):
    for n, F, G, S in itertools.product(NS, FS, [-1, 0, 1, 65, 2**31 - 1], [-1, 0, 1, 1000, 2**31 - 1, 2**31]):
        taken = 0 <= n < 2**31 and 1 <= F <= 2**20 and G >= 1 and F % G == 0 and 1 <= S < 2**31
        for name in ("tma_groupnorm_act_fwd_workspace_bytes", "tma_groupnorm_act_bwd_workspace_bytes"):
            b = getattr(lib, name)(i64(n), i32(F), i32(G), i64(S), i32(dtype))
            assert b % 256 == 0 and (b > 0 if taken else b == 0), (name, n, F, G, S)
    for n, E in itertools.product(NS, ES):
        b = lib.tma_group_rows_workspace_bytes(i64(n), i32(E))
        assert b % 256 == 0 and (b > 0) == (0 <= n < 2**31 and 1 <= E <= 1024)
