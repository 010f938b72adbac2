"""Residual blocks with gated layers, their products' gradients and clipping together, as a trainer runs them: loss and every gradient against automatic
differentiation of the same model in 64 bits (the trainers' own bound: 1e-4 of a tensor's norm, 2e-2 in bf16 storage); captured steps; several streams."""
import pytest

from test_gpu_typed_layers import B, graph  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def make(B, n, dims, F, dtype, clip=0.0, dropout=0.0, optimizer="sgd", stream=None, seed=0, scale=1.0):
    from paper_2305_09887_amd.trainer import LocalTrainer
    g = torch.Generator().manual_seed(seed)
    rowptr, colidx, inv, _ = graph(max(n, 2), 4, seed)
    X = torch.randn((n, dims[0]), generator=g).to(dtype)
    y = torch.randint(0, dims[-1], (n,), generator=g).int()
    params = []
    for l, (fi, fo) in enumerate(zip(dims[:-1], dims[1:])):
        shapes = [(fi, F), (fi, F), (F,), (F,), (F, fi), (fi,)] if fi == fo and l < len(dims) - 2 else [(fi, fo), (fo,)]
        params.append(tuple(torch.randn(s, generator=g) * (scale / s[0] ** 0.5 if len(s) == 2 else 0.1) for s in shapes))
    d = lambda t: t.cuda()
    tr = LocalTrainer(d(torch.from_numpy(rowptr[:n + 1])), d(torch.from_numpy(colidx)), d(torch.from_numpy(inv.astype("float32")[:n])), d(X), d(y), dims, params=params,
                      encoder="mlp", block_width=F, clip_norm=clip, dropout=dropout, dropout_seed=5, optimizer=optimizer, stream=stream)
    return tr, X, y, params


def model(X, y, params):
    leaves = [tuple(t.double().requires_grad_() for t in layer) for layer in params]
    h = X.double()
    for l, layer in enumerate(leaves):
        if len(layer) == 6:
            Wg, Wu, bg, bu, Wd, bd = layer
            gate = h @ Wg + bg
            h = h + (gate * torch.sigmoid(gate) * (h @ Wu + bu)) @ Wd + bd
        else:
            h = h @ layer[0] + layer[1]
            if l < len(leaves) - 1:
                h = h.clamp(min=0)
    loss = torch.nn.functional.cross_entropy(h, y.long())
    return loss, leaves, torch.autograd.grad(loss, [t for layer in leaves for t in layer])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,dims,F", [(1, [16, 16, 4], 24), (40, [20, 20, 20, 7], 33), (700, [24, 24, 24, 24, 5], 64), (3_000, [64, 64, 64, 10], 200)])
def test_gradients(B, n, dims, F, dtype):
    tr, X, y, params = make(B, n, dims, F, dtype)
    loss, leaves, want = model(X, y, params)
    tr.forward()
    tr.backward()
    torch.cuda.synchronize()
    bound = 2e-2 if dtype == torch.bfloat16 else 1e-4
    loss = float(loss.detach())
    assert abs(float(tr.loss) - loss) <= bound * max(1.0, loss)
    got = [g for layer in tr.grads for g in layer]
    assert len(got) == len(want)
    for i, (g, w) in enumerate(zip(got, want)):
        err, norm = float((g.cpu().double() - w).norm()), float(w.norm())
        assert err <= bound * norm, (i, tuple(w.shape), err, norm)


def test_a_step_clips_and_adam_and_sgd_take_the_clipped_gradients(B):
    for optimizer in ("sgd", "adam"):
        tr, X, y, params = make(B, 300, [24, 24, 24, 5], 40, torch.float32, clip=0.05, optimizer=optimizer)
        free = make(B, 300, [24, 24, 24, 5], 40, torch.float32, optimizer=optimizer)[0]
        W0 = tr.W.clone()
        free.step(0.5)
        tr.step(0.5)
        norm = float(free.dW.double().norm())
        assert norm > 0.1 and abs(float(tr.grad_norm) - norm) <= 1e-6 * norm
        want = free.dW.double() * (0.05 / norm)
        assert bool(((tr.dW.double() - want).abs() <= want.abs() * 2.0 ** -22).all())
        if optimizer == "sgd":
            assert torch.equal(tr.W, W0 - 0.5 * tr.dW) or float((tr.W - (W0 - 0.5 * tr.dW)).abs().max()) <= 2.0 ** -24 * float(W0.abs().max()) * 2
        wide = make(B, 300, [24, 24, 24, 5], 40, torch.float32, clip=1e6, optimizer=optimizer)[0]
        wide.step(0.5)
        assert torch.equal(wide.W, free.W)


def test_a_captured_step_replays_as_the_eager_one(B):
    for dtype, dropout in ((torch.float32, 0.0), (torch.bfloat16, 0.3)):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            a, b = (make(B, 900, [64, 64, 64, 6], 96, dtype, clip=0.05, dropout=dropout, stream=s)[0] for _ in range(2))
            a.step(0.1), b.step(0.1)
            s.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                a.step(0.1)
            for k in range(5):
                junk = torch.randn(1 << 20, device="cuda").sum()
                graph.replay()
                b.step(0.1)
                s.synchronize()
                assert torch.equal(a.W, b.W) and torch.equal(a.dW, b.dW) and torch.equal(a.loss, b.loss) and torch.equal(a.grad_norm, b.grad_norm), k
                del junk


def test_trainers_on_streams_of_their_own_at_once(B):
    alone = []
    for k in range(3):
        tr = make(B, 2_000 + 100 * k, [64, 64, 64, 6], 96, torch.float32, clip=0.05, seed=k)[0]
        for _ in range(4):
            tr.step(0.1)
        alone.append(tr.W.clone())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    trs = []
    for k, s in enumerate(streams):
        with torch.cuda.stream(s):
            trs.append(make(B, 2_000 + 100 * k, [64, 64, 64, 6], 96, torch.float32, clip=0.05, seed=k, stream=s)[0])
    torch.cuda.synchronize()
    for _ in range(4):
        for tr in trs:
            tr.step(0.1)
    torch.cuda.synchronize()
    assert all(torch.equal(tr.W, w) for tr, w in zip(trs, alone))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_a_trainer_without_nodes(B, dtype):
    tr = make(B, 0, [16, 16, 4], 24, dtype, clip=1.0)[0]
    held = tr.W.clone()
    tr.dW.fill_(7.0)
    tr.step(0.1)
    assert not tr.dW.any() and torch.equal(tr.W, held) and float(tr.grad_norm) == 0


def test_the_sampled_trainer_clips(B):
    from paper_2305_09887_amd import synth
    from paper_2305_09887_amd.trainer import SampledLinkTrainer
    rowptr, colidx = synth.uniform_graph(500, 3_000, seed=1)
    X = synth.features(500, 16, seed=2)
    d = lambda a: torch.as_tensor(a).cuda()
    free, held = (SampledLinkTrainer(d(rowptr).int(), d(colidx).int(), len(colidx), d(X), [16, 24, 8], [8, 12, 1], [5, 5], 64, clip_norm=c,
                                     params=synth.sage_params([16, 24, 8], seed=3),
                                     decoder_params=[(torch.ones(8, 12) / 4, torch.tensor([0.25])), (torch.ones(12, 1) / 4,)]) for c in (0.0, 1e-3))
    free.step(0.1)
    held.step(0.1)
    norm = float(free.dW.double().norm())
    assert norm > 1e-2 and abs(float(held.grad_norm) - norm) <= 1e-6 * norm
    assert abs(float(held.dW.double().norm()) - 1e-3) <= 1e-8
