"""What a trainer with residual blocks does with its gradients: Adam's moments and weights after clipped steps, and gradients through blocks whose outputs are dropped, against
automatic differentiation in 64 bits (the trainers' own bound: 1e-4 of a tensor's norm, 2e-2 in bf16 storage)."""
import pytest

from test_gpu_typed_layers import B  # noqa: F401
from test_gpu_wide_trainer import make

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_adam_takes_the_clipped_gradients(B):  # noqa: F811
    clip, lr = 0.05, 0.01
    tr = make(B, 300, [24, 24, 24, 5], 40, torch.float32, clip=clip, optimizer="adam")[0]
    m = v = torch.zeros_like(tr.W, dtype=torch.float64)
    for step in (1, 2, 3):
        W, m0, v0 = tr.W.double(), tr.adam_m.double(), tr.adam_v.double()
        tr.step(lr)
        g, norm = tr.dW.double(), float(tr.grad_norm)
        assert norm > 2 * clip and abs(float(g.norm()) - clip) <= clip * 2.0 ** -22       # (its values' roundings, and the bound's)
        m, v = 0.9 * m0 + 0.1 * g, 0.999 * v0 + 0.001 * g * g
        # three roundings each, of the coefficients, the products and the sum
        assert bool(((tr.adam_m.double() - m).abs() <= (0.9 * m0.abs() + 0.1 * g.abs()) * 2.0 ** -22 + 1e-44).all())
        assert bool(((tr.adam_v.double() - v).abs() <= v * 2.0 ** -21 + 1e-44).all())
        change = lr * (tr.adam_m.double() / (1 - 0.9 ** step)) / ((tr.adam_v.double() / (1 - 0.999 ** step)).sqrt() + 1e-8)
        assert bool(((tr.W.double() - (W - change)).abs() <= W.abs() * 2.0 ** -23 + change.abs() * 2.0 ** -20).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,dims,F", [(40, [20, 20, 20, 7], 33), (900, [24, 24, 24, 24, 5], 64), (700, [16, 24, 24, 5], 40)])
def test_gradients_through_dropped_blocks(B, n, dims, F, dtype):  # noqa: F811
    p = 0.3
    tr, X, y, params = make(B, n, dims, F, dtype, dropout=p)
    masks = [B.tma_dropout_fwd(torch.ones((n, f), device="cuda"), p, tr.drop_seeds[l], step=tr.drop_step).cpu().double() for l, f in enumerate(dims[1:-1])]
    for mask in masks:
        assert 0.5 < float((mask > 0).double().mean()) < 0.9
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
        if l < len(leaves) - 1:
            h = h * masks[l]
    loss = torch.nn.functional.cross_entropy(h, y.long())
    want = torch.autograd.grad(loss, [t for layer in leaves for t in layer])
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
