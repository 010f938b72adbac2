"""What the calls for layers of several kinds of rows refuse, in host code: nothing here touches a device."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
i64, i32, u64, sz, dbl, flt = (ctypes.c_int64, ctypes.c_int32, ctypes.c_uint64, ctypes.c_size_t, ctypes.c_double, ctypes.c_float)
FAKE, OTHER, ODD = ctypes.c_void_p(4096), ctypes.c_void_p(8192), ctypes.c_void_p(4100)      # never dereferenced
BIG = sz(1 << 50)


@pytest.fixture(scope="module")
def lib():
    from paper_2305_09887_amd import binding, build
    if not os.path.exists(build.LIB):
        build.build(verbose=False)
    return binding.lib()


def refused(lib, rc, code, text):
    assert rc == code, (rc, lib.tma_last_error())
    assert text in lib.tma_last_error(), lib.tma_last_error()


def test_group_rows(lib):
    def call(n=10, E=4, group=FAKE, offsets=FAKE, order=FAKE, ws=FAKE, ws_bytes=BIG):
        return lib.tma_group_rows(i64(n), group, i32(E), offsets, order, ws, ws_bytes, None)

    refused(lib, call(n=-1), -1, b"n outside")
    refused(lib, call(n=1 << 31), -1, b"n outside")
    refused(lib, call(E=0), -2, b"E=0")
    refused(lib, call(E=1025), -2, b"E=1025")
    for k in ("group", "offsets", "order"):
        refused(lib, call(**{k: None}), -1, b"NULL")
    refused(lib, call(ws=None), -1, b"workspace")
    refused(lib, call(ws=ODD), -1, b"256-byte")
    refused(lib, call(n=10**6, ws_bytes=sz(1000)), -3, b"workspace")
    assert lib.tma_group_rows_workspace_bytes(i64(-1), i32(4)) == 0 and lib.tma_group_rows_workspace_bytes(i64(5), i32(0)) == 0
    assert lib.tma_group_rows_workspace_bytes(i64(10**6), i32(7)) % 256 == 0


def test_grouped_dense(lib):
    def fwd(n=10, E=2, offsets=FAKE, order=None, X=FAKE, ldx=8, F_in=8, W=FAKE, bias=None, F_out=8, act=0, dtype=0, Y=OTHER, ldy=8, ws=FAKE, ws_bytes=BIG):
        return lib.tma_grouped_dense_fwd(i64(n), i32(E), offsets, order, X, i64(ldx), i32(F_in), W, bias, i32(F_out), i32(act), i32(dtype), Y, i64(ldy), ws,
                                         ws_bytes, None)

    def bwd(n=10, E=2, offsets=FAKE, X=FAKE, ldx=8, Y=FAKE, dY=FAKE, ldy=8, W=FAKE, F_in=8, F_out=8, act=1, dtype=0, dW=FAKE, dX=OTHER, ld_dx=8, ws=FAKE,
            ws_bytes=BIG):
        return lib.tma_grouped_dense_bwd(i64(n), i32(E), offsets, None, X, i64(ldx), Y, dY, i64(ldy), W, i32(F_in), i32(F_out), i32(act), i32(dtype), dW, None,
                                         dX, i64(ld_dx), ws, ws_bytes, None)

    for call in (fwd, bwd):
        refused(lib, call(n=-1), -1, b"n outside")
        refused(lib, call(n=1 << 31), -1, b"n outside")
        refused(lib, call(E=0), -2, b"E=0")
        refused(lib, call(E=1025), -2, b"E=1025")
        refused(lib, call(F_in=0), -2, b"F_in=0")
        refused(lib, call(F_out=65537), -2, b"F_out=65537")
        for act in (-1, 2, 3):
            refused(lib, call(act=act), -1, b"act")
        refused(lib, call(dtype=2), -4, b"dtype")
        refused(lib, call(offsets=None), -1, b"offsets")
        refused(lib, call(ws=None), -1, b"workspace")
        refused(lib, call(ws=ODD), -1, b"256-byte")
        refused(lib, call(ws_bytes=sz(16)), -3, b"workspace")
        refused(lib, call(X=None), -1, b"NULL")
        refused(lib, call(W=None), -1, b"NULL")
        refused(lib, call(ldx=7), -2, b"ldx" if call is fwd else b"leading")
    refused(lib, fwd(Y=FAKE), -1, b"one")
    refused(lib, fwd(ldy=7), -2, b"ldy")
    refused(lib, bwd(dW=None), -1, b"dW")
    refused(lib, bwd(Y=None), -1, b"Y is required")
    refused(lib, bwd(dX=FAKE), -1, b"one of the inputs")
    refused(lib, bwd(ld_dx=7), -2, b"leading")


def test_group_norm(lib):
    def fwd(n=12, F=8, G=2, S=3, seg=None, R=4, X=FAKE, ldx=8, gamma=FAKE, beta=FAKE, slope=None, eps=1e-5, act=0, dtype=0, Y=OTHER, ldy=8, stats=FAKE,
            ws=FAKE, ws_bytes=BIG):
        return lib.tma_groupnorm_act_fwd(i64(n), i32(F), i32(G), i64(S), seg, i64(R), X, i64(ldx), gamma, beta, slope, flt(eps), i32(act), i32(dtype), Y,
                                         i64(ldy), stats, ws, ws_bytes, None)

    def bwd(n=12, F=8, G=2, S=3, seg=None, R=4, X=FAKE, ldx=8, dY=FAKE, ldd=8, gamma=FAKE, beta=FAKE, slope=None, eps=1e-5, act=0, dtype=0, stats=FAKE,
            dX=OTHER, ldo=8, dgamma=FAKE, dbeta=FAKE, dslope=None, ws=FAKE, ws_bytes=BIG):
        return lib.tma_groupnorm_act_bwd(i64(n), i32(F), i32(G), i64(S), seg, i64(R), X, i64(ldx), dY, i64(ldd), gamma, beta, slope, flt(eps), i32(act),
                                         i32(dtype), stats, dX, i64(ldo), dgamma, dbeta, dslope, ws, ws_bytes, None)

    for call in (fwd, bwd):
        refused(lib, call(n=-4), -1, b"n outside")
        refused(lib, call(G=3), -2, b"G=3")
        refused(lib, call(G=0), -2, b"G=0")
        refused(lib, call(F=2050, G=2, ldx=2050), -2, b"1025")
        refused(lib, call(dtype=7), -4, b"dtype")
        for act in (-1, 4):
            refused(lib, call(act=act), -1, b"act")
        refused(lib, call(eps=-1.0), -1, b"eps")
        refused(lib, call(eps=float("nan")), -1, b"eps")
        refused(lib, call(gamma=None), -1, b"gamma")
        refused(lib, call(act=2), -1, b"slope")
        refused(lib, call(R=5), -2, b"runs")
        refused(lib, call(R=0), -2, b"runs")
        refused(lib, call(seg=FAKE, S=0), -1, b"n_segments")
        refused(lib, call(X=None), -1, b"NULL")
        refused(lib, call(ldx=7), -2, b"leading")
        refused(lib, call(ws=None), -1, b"workspace")
        refused(lib, call(ws=ODD), -1, b"256-byte")
        refused(lib, call(ws_bytes=sz(16)), -3, b"workspace")
    refused(lib, fwd(Y=FAKE), -1, b"one")
    refused(lib, fwd(stats=ODD), -1, b"8-byte")
    refused(lib, bwd(dX=FAKE), -1, b"dX_out")
    refused(lib, bwd(stats=None), -1, b"stats")
    refused(lib, bwd(act=2, slope=FAKE), -1, b"gradient output")
    refused(lib, bwd(dgamma=None), -1, b"gradient output")
    refused(lib, bwd(dY=OTHER, ldo=9), -2, b"in place")


def test_dropout(lib):
    for name in ("tma_dropout_fwd", "tma_dropout_bwd"):
        def call(n=10, F=8, X=FAKE, ldx=8, p=0.5, step=None, first=0, dtype=0, Y=OTHER, ldy=8):
            return getattr(lib, name)(i64(n), i32(F), X, i64(ldx), dbl(p), u64(1), step, i64(first), i32(dtype), Y, i64(ldy), None)

        refused(lib, call(n=-1), -1, b"n outside")
        refused(lib, call(F=0), -2, b"F=0")
        for p in (-0.01, 1.01, float("nan")):
            refused(lib, call(p=p), -1, b"p outside")
        refused(lib, call(first=-1), -1, b"first_row")
        refused(lib, call(dtype=3), -4, b"dtype")
        refused(lib, call(step=ODD), -1, b"8-byte")
        refused(lib, call(X=None), -1, b"NULL")
        refused(lib, call(Y=None), -1, b"NULL")
        refused(lib, call(ldx=7), -2, b"leading")
        refused(lib, call(Y=FAKE, ldy=9), -2, b"in place")


def test_the_binding_refuses_host_tensors_and_wrong_shapes(lib):
    import torch
    from paper_2305_09887_amd import binding as B
    x = torch.zeros((4, 8))
    for call in (lambda: B.tma_dropout_fwd(x, 0.5, 1), lambda: B.tma_group_rows(torch.zeros(4, dtype=torch.int32), 2),
                 lambda: B.tma_groupnorm_act_fwd(x, 2, torch.zeros(8), torch.zeros(8)),
                 lambda: B.tma_grouped_dense_fwd(x, torch.zeros((2, 8, 3)), None, torch.zeros(3, dtype=torch.int32), 0)):
        with pytest.raises(B.TmaError, match="one CUDA/HIP device"):
            call()
