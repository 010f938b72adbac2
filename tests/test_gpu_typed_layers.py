"""Rows by kind, products per kind, group norm with PReLU and dropout together, as a trainer runs them: loss and every gradient against
automatic differentiation of the same model in 64 bits, with the masks of the written rule.  The bound is the trainers' own, 1e-4 of a
tensor's norm (2e-2 in bf16 storage)."""
import numpy as np
import pytest

from test_gpu_dropout import plain as dropped

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2305_09887_amd import binding
    binding.lib()
    return binding


def graph(n, degree, seed):
    """A symmetric graph's CSR and its row-normalised adjacency."""
    r = np.random.default_rng(seed)
    A = np.zeros((n, n), dtype=bool)
    A[r.integers(0, n, n * degree // 2), r.integers(0, n, n * degree // 2)] = True
    A |= A.T
    np.fill_diagonal(A, False)
    rowptr = np.concatenate([[0], A.sum(1).cumsum()]).astype(np.int32)
    colidx = np.nonzero(A)[1].astype(np.int32)
    deg = A.sum(1)
    inv = np.where(deg > 0, 1 / np.maximum(deg, 1), 0)
    return rowptr, colidx, inv, torch.from_numpy(A * inv[:, None])


def make(B, encoder, n, dims, norm_groups, p, kinds, dtype, seed=0, stream=None, optimizer="sgd"):
    from paper_2305_09887_amd.trainer import LocalTrainer
    g = torch.Generator().manual_seed(seed)
    rowptr, colidx, inv, A = graph(n, 6, seed)
    X = torch.randn((n, dims[0]), generator=g).to(dtype)
    y = torch.randint(0, dims[-1], (n,), generator=g).int()
    E = max(kinds, 1)
    params = []
    for l, (fi, fo) in enumerate(zip(dims[:-1], dims[1:])):
        shape = (E, fi, fo) if kinds else (fi, fo)
        lin = [torch.randn(shape, generator=g) * (2 / (fi + fo)) ** 0.5 for _ in range(2 if encoder == "sage" else 1)]
        lin.append(torch.randn((E, fo) if kinds else (fo,), generator=g) * 0.1)
        if norm_groups and l < len(dims) - 2:
            lin += [1 + 0.2 * torch.randn(fo, generator=g), 0.2 * torch.randn(fo, generator=g), torch.tensor([0.25])]
        params.append(tuple(lin))
    ids = torch.randint(0, kinds, (n,), generator=g).int() if kinds else None
    tr = LocalTrainer(torch.from_numpy(rowptr).cuda(), torch.from_numpy(colidx).cuda(), torch.from_numpy(inv.astype(np.float32)).cuda(), X.cuda(),
                      y.cuda(), dims, params=params, encoder=encoder, norm_act=norm_groups > 0, norm_groups=norm_groups, dropout=p, dropout_seed=77,
                      node_kinds=ids.cuda() if kinds else None, n_kinds=kinds, stream=stream, optimizer=optimizer)
    return tr, X, y, params, ids, A


def model(B, encoder, X, y, params, ids, A, norm_groups, p, step):
    """Loss, and the parameters as leaves."""
    leaves = [tuple(t.double().requires_grad_(True) for t in layer) for layer in params]
    h = X.double()
    for l, layer in enumerate(leaves):
        if ids is not None:
            z = torch.stack([h[v] @ layer[0][ids[v]] + layer[1][ids[v]] for v in range(h.shape[0])])
        elif encoder == "sage":
            z = h @ layer[0] + A @ h @ layer[1] + layer[2]
        else:
            z = h @ layer[0] + layer[1]
        h = z
        if l < len(leaves) - 1:
            if norm_groups:
                gamma, beta, slope = layer[-3:]
                v = z.view(z.shape[0], norm_groups, -1)
                xh = (v - v.mean(2, keepdim=True)) / (v.var(2, unbiased=False, keepdim=True) + 1e-5).sqrt()
                u = gamma * xh.reshape(z.shape) + beta
                h = torch.where(u > 0, u, slope * u)
            else:
                h = z.clamp(min=0)
            if p:
                h = h * dropped(torch.ones(h.shape), p, B.tma_mix64(77, l), step).double()
    return torch.nn.functional.cross_entropy(h, y.long()), leaves


def off(got, want):
    return ((got.double() - want).norm() / want.norm().clamp(min=1e-30)).item()


@pytest.mark.parametrize("encoder,kinds,norm_groups,p", [("mlp", 3, 4, 0.3), ("mlp", 5, 0, 0.5), ("mlp", 0, 8, 0.0), ("sage", 0, 4, 0.2), ("sage", 0, 0, 0.6),
                                                         ("mlp", 200, 2, 0.1)])
def test_gradients_of_a_training_pass(B, encoder, kinds, norm_groups, p):
    n, dims, lr = 301, [20, 48, 32, 7], 0.05
    tr, X, y, params, ids, A = make(B, encoder, n, dims, norm_groups, p, kinds, torch.float32)
    for step in range(2):
        loss = tr.step(lr).item()
        want, leaves = model(B, encoder, X, y, params, ids, A, norm_groups, p, step)
        assert abs(loss - want.item()) <= 1e-4 * abs(want.item())
        grads = torch.autograd.grad(want, [t for layer in leaves for t in layer])
        mine = [t for layer in tr.grads for t in layer]
        for k, (a, b) in enumerate(zip(mine, grads)):
            assert off(a.cpu().reshape(b.shape), b) <= 1e-4, (step, k, off(a.cpu().reshape(b.shape), b))
        params = [tuple(t.detach() for t in layer) for layer in leaves]
        flat = iter(grads)
        params = [tuple(t - lr * next(flat) for t in layer) for layer in params]
    assert int(tr.drop_step) == 2 if p else True


def test_evaluation_drops_nothing(B):
    tr, X, y, params, ids, A = make(B, "mlp", 150, [12, 32, 5], 4, 0.5, 3, torch.float32)
    tr.training = False
    logits = tr.forward().clone()
    assert torch.equal(logits, tr.forward())
    tr.backward()
    want, _ = model(B, "mlp", X, y, params, ids, A, 4, 0.0, 0)
    assert abs(tr.loss.item() - want.item()) <= 1e-4 * want.item()


def test_bf16_storage(B):
    tr, X, y, params, ids, A = make(B, "mlp", 400, [24, 64, 48, 6], 8, 0.25, 4, torch.bfloat16)
    loss = tr.step(0.05).item()
    want, leaves = model(B, "mlp", X, y, params, ids, A, 8, 0.25, 0)
    assert abs(loss - want.item()) <= 2e-2 * want.item()
    grad = torch.autograd.grad(want, leaves[-1][0])[0]
    assert off(tr.grads[-1][0].cpu(), grad) <= 2e-2


def test_captured_steps_are_the_eager_ones(B):
    """Four replays of a captured step against four eager steps of a twin: each draws its own mask, the same bits."""
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        a = make(B, "mlp", 260, [16, 32, 32, 5], 4, 0.4, 3, torch.float32, stream=s)[0]
        b = make(B, "mlp", 260, [16, 32, 32, 5], 4, 0.4, 3, torch.float32, stream=s)[0]
        a.step(0.1), b.step(0.1)
        s.synchronize()
        graph_ = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph_, stream=s):
            a.step(0.1)
        for k in range(4):
            graph_.replay()
            b.step(0.1)
            s.synchronize()
            assert torch.equal(a.W, b.W) and torch.equal(a.loss, b.loss), k
            torch.zeros(1000, device="cuda").add_(1).sum().item()
        assert int(a.drop_step) == int(b.drop_step) == 5


def test_kinds_that_are_none_are_refused(B):
    from paper_2305_09887_amd.trainer import LocalTrainer
    X, y = torch.zeros((4, 3), device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    rp, none, inv = torch.zeros(5, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(4, device="cuda")
    build = lambda **kw: LocalTrainer(rp, none, inv, X, y, [3, 4, 2], **{"encoder": "mlp", **kw})
    kinds = torch.tensor([0, 1, 2, 1], dtype=torch.int32, device="cuda")
    build(node_kinds=kinds, n_kinds=3)
    for kw, text in [(dict(node_kinds=kinds, n_kinds=2), "outside"), (dict(node_kinds=kinds), "come together"), (dict(n_kinds=2), "come together"),
                     (dict(node_kinds=kinds, n_kinds=3, encoder="sage"), "MLP"), (dict(norm_groups=2), "norm_act"),
                     (dict(norm_act=True, norm_groups=3), "multiples"), (dict(dropout=1.0), "dropout"), (dict(dropout=-0.1), "dropout")]:
        with pytest.raises(B.TmaError, match=text):
            build(**kw)


def test_two_streams_at_once(B):
    """The same chain of calls on two streams, workspaces the calls' own: what each would have given alone, bit for bit."""
    n, E, F = 40_000, 6, 96

    def inputs(seed):
        g = torch.Generator().manual_seed(seed)
        kinds = torch.randint(0, E, (n,), generator=g).int().cuda()
        X, dY = torch.randn(n, F, generator=g).cuda(), torch.randn(n, F, generator=g).cuda()
        W, b = (torch.randn(E, F, F, generator=g) * 0.1).cuda(), torch.randn(E, F, generator=g).cuda()
        cuts = torch.sort(torch.randint(0, n, (30,), generator=g)).values.int()
        segments = torch.cat([torch.zeros(1, dtype=torch.int32), cuts, torch.tensor([n], dtype=torch.int32)]).cuda()
        return kinds, X, dY, W, b, segments, torch.ones(F, device="cuda"), torch.zeros(F, device="cuda")

    def chain(x, stream):
        kinds, X, dY, W, b, segments, gamma, beta = x
        offsets, order = B.tma_group_rows(kinds, E, stream=stream)
        Y = B.tma_grouped_dense_fwd(X, W, b, offsets, B.TMA_ACT_RELU, order=order, stream=stream)
        H, stats = B.tma_groupnorm_act_fwd(Y, 8, gamma, beta, B.TMA_ACT_SILU, segments=segments, stream=stream)
        D = B.tma_dropout_fwd(H, 0.3, 5, stream=stream)
        dH = B.tma_dropout_bwd(dY, 0.3, 5, stream=stream)
        dN, dga, dbe, _ = B.tma_groupnorm_act_bwd(Y, dH, 8, gamma, beta, B.TMA_ACT_SILU, segments=segments, stats=stats, stream=stream)
        dW, db, dX = B.tma_grouped_dense_bwd(X, Y, dN, W, offsets, B.TMA_ACT_RELU, order=order, stream=stream)
        return offsets, order, Y, D, dga, dbe, dW, db, dX

    both = [inputs(1), inputs(2)]
    torch.cuda.synchronize()
    alone = []
    for x in both:
        alone.append(chain(x, None))
        torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        results = [chain(x, s) for x, s in zip(both, streams)]
        torch.cuda.synchronize()
        for got, want in zip(results, alone):
            for a, c in zip(got, want):
                assert torch.equal(a, c)
