"""What the calls for wide layers, the gradients' norm and clipping refuse, in host code: nothing here touches a device."""
import ctypes
import os

import pytest

from test_layer_refusals import BIG, FAKE, ODD, OTHER, lib, refused  # noqa: F401

torch = pytest.importorskip("torch")
P = ctypes.c_void_p
A = [P(4096 * (k + 1)) for k in range(16)]      # never dereferenced


def gated_fwd(lib, n=100, X=A[0], ldx=8, F_in=8, Wg=A[1], Wu=A[2], F_out=8, act=3, dtype=0, G=A[3], U=A[4], ldg=8, H=A[5], ldh=8, ws=A[6], ws_bytes=1 << 50):
    return lib.tma_gated_dense_fwd(n, X, ldx, F_in, Wg, Wu, None, None, F_out, act, dtype, G, U, ldg, H, ldh, ws, ws_bytes, None)


def gated_bwd(lib, n=100, X=A[0], ldx=8, G=A[3], U=A[4], ldg=8, dH=A[5], ldh=8, Wg=A[1], Wu=A[2], F_in=8, F_out=8, act=3, dtype=0, dWg=A[7], dWu=A[8], dbg=None,
              dbu=None, dX=A[9], ld_dx=8, R=None, ldr=8, ws=A[6], ws_bytes=1 << 50):
    return lib.tma_gated_dense_bwd(n, X, ldx, G, U, ldg, dH, ldh, Wg, Wu, F_in, F_out, act, dtype, dWg, dWu, dbg, dbu, dX, ld_dx, R, ldr, ws, ws_bytes, None)


def res_fwd(lib, n=100, X=A[0], ldx=8, F_in=8, W=A[1], F_out=8, act=0, dtype=0, R=A[2], ldr=8, Z=A[3], ldz=8, Y=A[4], ldy=8, ws=A[6], ws_bytes=1 << 50):
    return lib.tma_dense_residual_fwd(n, X, ldx, F_in, W, None, F_out, act, dtype, R, ldr, Z, ldz, Y, ldy, ws, ws_bytes, None)


def res_bwd(lib, n=100, X=A[0], ldx=8, Z=A[3], ldz=8, dY=A[4], ldy=8, W=A[1], F_in=8, F_out=8, act=3, dtype=0, dW=A[7], dX=A[9], ld_dx=8, R=None, ldr=8, ws=A[6],
            ws_bytes=1 << 50):
    return lib.tma_dense_residual_bwd(n, X, ldx, Z, ldz, dY, ldy, W, F_in, F_out, act, dtype, dW, None, dX, ld_dx, R, ldr, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [gated_fwd, gated_bwd, res_fwd, res_bwd])
def test_sizes_types_and_workspaces(lib, call):
    refused(lib, call(lib, n=-1), -1, b"n outside")
    refused(lib, call(lib, n=1 << 31), -1, b"n outside")
    refused(lib, call(lib, F_in=0), -2, b"F_in=0")
    refused(lib, call(lib, F_out=65537), -2, b"F_out=65537")
    for act in (-1, 2, 5):
        refused(lib, call(lib, act=act), -1, b"act")
    for dtype in (-1, 2):
        refused(lib, call(lib, dtype=dtype), -4, b"dtype")
    refused(lib, call(lib, ws=None), -1, b"workspace")
    refused(lib, call(lib, ws=P(4100)), -1, b"256-byte")
    refused(lib, call(lib, ws_bytes=100), -3, b"workspace")
    refused(lib, call(lib, ldx=7), -2, b"leading dimension")
    refused(lib, call(lib, X=None), -1, b"NULL")


def test_gated(lib):
    for k in ("Wg", "Wu", "H"):
        refused(lib, gated_fwd(lib, **{k: None}), -1, b"NULL")
    for k in ("G", "U"):
        refused(lib, gated_fwd(lib, **{k: None}), -1, b"go together")
    refused(lib, gated_fwd(lib, ldg=7), -2, b"leading dimension")
    refused(lib, gated_fwd(lib, ldh=7), -2, b"leading dimension")
    for k in (dict(H=A[0]), dict(G=A[0]), dict(U=A[0]), dict(G=A[5]), dict(U=A[5]), dict(U=A[3])):
        refused(lib, gated_fwd(lib, **k), -1, b"are one")
    for k in ("G", "U", "dH", "Wg", "Wu"):
        refused(lib, gated_bwd(lib, **{k: None}), -1, b"NULL")
    for k in (dict(dWg=None), dict(dWu=None), dict(dWu=A[7])):
        refused(lib, gated_bwd(lib, **k), -1, b"dW_gate")
    for k in (dict(dbg=A[10]), dict(dbu=A[10]), dict(dbg=A[10], dbu=A[10])):
        refused(lib, gated_bwd(lib, **k), -1, b"go together")
    for k in ("ldg", "ldh", "ld_dx"):
        refused(lib, gated_bwd(lib, **{k: 7}), -2, b"leading dimension")
    refused(lib, gated_bwd(lib, R=A[11], ldr=7), -2, b"leading dimension")
    for k in (A[0], A[3], A[4], A[5]):
        refused(lib, gated_bwd(lib, dX=k), -1, b"dX_out is one of")
    for k in ("Wg", "Wu"):
        refused(lib, gated_bwd(lib, **{k: A[7]}), -1, b"a weight is its gradient")
        refused(lib, gated_bwd(lib, **{k: A[8]}), -1, b"a weight is its gradient")
    refused(lib, gated_bwd(lib, R=A[9], ldr=9), -2, b"in place")


def test_residual(lib):
    for k in ("W", "Y"):
        refused(lib, res_fwd(lib, **{k: None}), -1, b"NULL")
    for k in ("ldz", "ldy", "ldr"):
        refused(lib, res_fwd(lib, **{k: 7}), -2, b"leading dimension")
    for k in (dict(Y=A[0]), dict(Z=A[0]), dict(Z=A[4]), dict(Z=A[2])):
        refused(lib, res_fwd(lib, **k), -1, b"Z_out is one")
    refused(lib, res_fwd(lib, R=A[4], ldr=9), -2, b"in place")
    refused(lib, res_bwd(lib, dW=None), -1, b"dW is NULL")
    refused(lib, res_bwd(lib, dW=A[1]), -1, b"dW is NULL, or W")
    for k in ("dY", "W"):
        refused(lib, res_bwd(lib, **{k: None}), -1, b"NULL")
    refused(lib, res_bwd(lib, Z=None), -1, b"Z is required")
    for k in ("ldz", "ldy", "ld_dx"):
        refused(lib, res_bwd(lib, **{k: 7}), -2, b"leading dimension")
    for k in (A[0], A[3], A[4]):
        refused(lib, res_bwd(lib, dX=k), -1, b"dX_out is one of")
    refused(lib, res_bwd(lib, R=A[9], ldr=9), -2, b"in place")


def test_workspace_sizes(lib):
    for query in (lib.tma_gated_dense_fwd_workspace_bytes, lib.tma_dense_residual_fwd_workspace_bytes):
        assert query(1, 64, 64, 1) == 0 and query(64, 32, 32, 0) == 0 and query(1, 8192, 1024, 1) >= 2 * 1024 * 4 and query(65, 64, 64, 1) > 0
        for n, fi, fo in ((-1, 8, 8), (1 << 31, 8, 8), (100, 0, 8), (100, 8, 0), (100, 65537, 8), (100, 8, 65537), (100, -5, 8)):
            assert query(n, fi, fo, 0) == 0
        assert query(1000, 300, 77, 0) % 256 == 0
    for query, more in ((lib.tma_gated_dense_bwd_workspace_bytes, ()), (lib.tma_dense_residual_bwd_workspace_bytes, (3,))):
        assert query(-1, 8, 8, *more, 0, 1) == 0 and query(5, 8, 0, *more, 0, 1) == 0
        assert query(1000, 300, 77, *more, 0, 1) % 256 == 0
        assert query(1000, 300, 77, *more, 0, 1) > query(1000, 300, 77, *more, 0, 0) > query(1000, 300, 77, *more, 1, 0) > 0
    # the widest layers on the largest part that a card holds the rows of
    assert lib.tma_gated_dense_fwd_workspace_bytes(1 << 20, 65536, 65536, 1) > (1 << 20) * 65536 * 2
    assert lib.tma_grad_norm_workspace_bytes(-1) == 0 and lib.tma_grad_norm_workspace_bytes((1 << 17) + 1) == 0
    assert lib.tma_grad_norm_workspace_bytes(0) >= 2048 * 8 and lib.tma_grad_norm_workspace_bytes(1 << 17) % 256 == 0


def test_lists_of_gradients(lib):
    ptrs, sizes = (ctypes.c_void_p * 2)(4096, 8192), (ctypes.c_int64 * 2)(10, 20)

    def norm(n=2, p=ptrs, s=sizes, dtype=0, out=A[0], ws=A[1], ws_bytes=1 << 30):
        return lib.tma_grad_norm(n, p, s, dtype, out, ws, ws_bytes, None)

    def clip(n=2, p=ptrs, s=sizes, dtype=0, out=A[0], ws=A[1], ws_bytes=1 << 30, outs=None, bound=1.0):
        return lib.tma_grad_clip(n, p, outs, s, dtype, bound, out, ws, ws_bytes, None)

    for call in (norm, clip):
        refused(lib, call(n=-1), -1, b"n_tensors")
        refused(lib, call(n=(1 << 17) + 1), -1, b"n_tensors")
        refused(lib, call(dtype=2), -4, b"dtype")
        for k in ("p", "s", "out"):
            refused(lib, call(**{k: None}), -1, b"NULL")
        refused(lib, call(ws=None), -1, b"workspace")
        refused(lib, call(ws=P(4100)), -1, b"256-byte")
        refused(lib, call(ws_bytes=4096), -3, b"workspace")
        refused(lib, call(s=(ctypes.c_int64 * 2)(10, -1)), -2, b"size of tensor 1")
        refused(lib, call(p=(ctypes.c_void_p * 2)(4096, None)), -1, b"tensor 1 is NULL")
        refused(lib, call(p=(ctypes.c_void_p * 2)(4098, 4096)), -1, b"tensor 0 is NULL or not aligned")
        refused(lib, call(p=(ctypes.c_void_p * 2)(4097, 4096), dtype=1), -1, b"tensor 0 is NULL or not aligned")
    refused(lib, clip(outs=(ctypes.c_void_p * 2)(4096, None)), -1, b"tensor 1")
    for bound in (-1.0, float("nan")):
        refused(lib, clip(bound=bound), -1, b"max_norm")
    for p, s in (((4096, 4096), (10, 20)), ((8192, 4096), (10, 1025)), ((4096, 4100), (10, 20)), ((4096,) * 2 + tuple(range(8192, 8192 + 64 * 400, 64)), (1, 1) + (16,) * 400)):
        P_, S_ = (ctypes.c_void_p * len(p))(*p), (ctypes.c_int64 * len(s))(*s)
        refused(lib, clip(n=len(p), p=P_, s=S_), -1, b"overlap")
        apart = (ctypes.c_void_p * len(p))(*[(1 << 30) - (1 << 14) * i for i in range(len(p))])
        refused(lib, clip(n=len(p), p=apart, s=S_, outs=P_), -1, b"overlap")


def test_trainers_refuse_blocks_that_are_none():
    from paper_2305_09887_amd import binding as B
    from paper_2305_09887_amd.trainer import LocalTrainer
    X = torch.zeros((3, 8))
    for dims, more in (([8, 8, 4], dict(encoder="sage", block_width=8)), ([8, 6, 4], dict(encoder="mlp", block_width=8)), ([8, 8], dict(encoder="mlp", block_width=8)),
                       ([8, 8, 4], dict(encoder="mlp", block_width=-1)), ([8, 8, 4], dict(encoder="mlp", block_width=8, norm_act=True))):
        with pytest.raises(B.TmaError, match="block_width"):
            LocalTrainer(None, None, None, X, None, dims, **more)
    for c in (-1.0, float("nan"), float("inf")):
        with pytest.raises(B.TmaError, match="clip_norm"):
            LocalTrainer(None, None, None, X, None, [8, 4], clip_norm=c)


def test_the_reader_of_lists_of_tensors():
    """On host tensors (device -1): what it takes, what it refuses and where."""
    from paper_2305_09887_amd import binding as B
    from paper_2305_09887_amd import build
    if not os.path.exists(build.LISTS):
        build.build_lists()

    def read(tensors, dtype=0, index=-1, lengths=None):
        n = len(tensors)
        a, s = (ctypes.c_uint64 * max(n, 1))(), (ctypes.c_int64 * max(n, 1))(*(lengths or [0] * n))
        B._read("here", tensors, dtype, index, ctypes.addressof(a), ctypes.addressof(s), 1 if lengths else 0, "tensor")
        return list(a)[:n], list(s)[:n]

    flat = torch.arange(40.0)
    ts = [flat[:7], flat[7:8], torch.empty(0), flat[8:].view(4, 8), torch.nn.Parameter(torch.ones(3, 5)), torch.tensor(2.0)]
    for tensors in (ts, tuple(ts)):
        a, s = read(tensors)
        assert s == [7, 1, 0, 32, 15, 1] and a == [t.data_ptr() for t in ts]
        assert read(tensors, lengths=s) == (a, s)
    assert read([t.detach().bfloat16() for t in ts], dtype=1)[1] == [7, 1, 0, 32, 15, 1]
    assert read([]) == ([], [])
    for bad in (flat.double(), flat.half(), flat.bfloat16(), flat.view(5, 8).t(), flat[::2], flat.expand(2, 40), torch.ones(3).to_sparse(), 3.0, None, torch.empty(3, device="meta")):
        with pytest.raises(B.TmaError, match="here: tensor 1:"):
            read([flat, bad, flat])
    with pytest.raises(B.TmaError, match="here: tensor 0:"):
        read([flat], index=0)
    with pytest.raises(B.TmaError, match="differs from its gradient in size"):
        read([flat, flat[:3]], lengths=[40, 4])
