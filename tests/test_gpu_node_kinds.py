"""Other kinds for a trainer's nodes: the lists stay where captured steps read them, and a refused call changes nothing."""
import pytest

from test_gpu_typed_layers import B, make

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
N, DIMS, E = 260, [16, 32, 32, 5], 3


def trainer(B, stream=None):
    return make(B, "mlp", N, DIMS, 4, 0.4, E, torch.float32, stream=stream)[0]


def other_kinds(seed):
    return torch.randint(0, E, (N,), generator=torch.Generator().manual_seed(seed)).int().cuda()


def test_a_captured_step_runs_on_the_kinds_that_were_set_after_it(B):
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        a, b = trainer(B, s), trainer(B, s)
        a.step(0.1), b.step(0.1)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            a.step(0.1)
        where = a.kind_offsets.data_ptr(), a.kind_order.data_ptr()
        for k in range(4):
            kinds = other_kinds(k)
            a.set_kinds(kinds)
            b.set_kinds(kinds)
            assert where == (a.kind_offsets.data_ptr(), a.kind_order.data_ptr())
            junk = [torch.full((m,), 7, dtype=torch.int32, device="cuda") for m in (E + 1, N) for _ in range(20)]      # takes what was freed
            graph.replay()
            b.step(0.1)
            s.synchronize()
            assert torch.equal(a.W, b.W) and torch.equal(a.loss, b.loss), k
            del junk


def test_a_refused_call_leaves_the_kinds_as_they_were(B):
    a, b = trainer(B), trainer(B)
    kinds = other_kinds(7)
    a.set_kinds(kinds), b.set_kinds(kinds)
    held = a.kind_offsets.clone(), a.kind_order.clone()
    wrong = kinds.clone()
    wrong[100:] = E
    negative = kinds.clone()
    negative[3] = -1
    for given, text in [(wrong, "outside"), (negative, "outside"), (kinds[:-1], "one kind per node"), (kinds.cpu(), "device"), (kinds.long(), "int32")]:
        with pytest.raises(B.TmaError, match=text):
            a.set_kinds(given)
        assert torch.equal(a.kind_offsets, held[0]) and torch.equal(a.kind_order, held[1])
    a.step(0.1), b.step(0.1)
    assert torch.equal(a.W, b.W)
    assert int(a.kind_offsets[-1]) == N and torch.equal(a.kind_order.sort().values, torch.arange(N, dtype=torch.int32, device="cuda"))


def test_a_trainer_without_kinds_takes_none(B):
    with pytest.raises(B.TmaError, match="without kinds"):
        make(B, "mlp", 20, [4, 8, 3], 0, 0.0, 0, torch.float32)[0].set_kinds(torch.zeros(20, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_trainer_without_nodes(B, dtype):
    """No rows at all: every layer's gradients are zero, and the parameters stay."""
    from paper_2305_09887_amd.trainer import LocalTrainer
    i32 = lambda k: torch.zeros(k, dtype=torch.int32, device="cuda")
    tr = LocalTrainer(i32(1), i32(1), torch.zeros(0, device="cuda"), torch.zeros((0, 8), dtype=dtype, device="cuda"), i32(0), [8, 16, 12, 4], encoder="mlp", norm_act=True,
                      norm_groups=4, dropout=0.5, node_kinds=i32(0), n_kinds=3)
    tr.W.copy_(torch.randn(tr.W.shape, generator=torch.Generator().manual_seed(1)))
    tr.set_kinds(i32(0))
    held = tr.W.clone()
    tr.dW.fill_(7.0)
    assert tr.forward().shape == (0, 4)
    tr.step(0.1)
    assert not tr.dW.any() and torch.equal(tr.W, held)
