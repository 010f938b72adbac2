"""Dense layers with weights per group on small whole numbers: every product, sum and part of a value is exact in whatever order (all sums of magnitudes stay
below 2^24), so the results are the exact ones rounded once to the storage type, bit for bit.  A row that is missed, counted twice, or taken from the wrong place
shows in any of them.  Groups that are far longer than the mean, on the kernels for a few rows a group; runs of rows that are longer than the list of row
numbers held in LDS (1,024 rows in fp32, 2,048 in bf16), for their weight gradients; weights that bf16 holds exactly, for which bf16 storage rounds the result alone."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2305_09887_amd import binding
    binding.lib()
    return binding


def whole(shape, most, g, dtype=torch.float32):
    return torch.randint(-most, most + 1, shape, generator=g, device="cuda").to(dtype)


def check(B, sizes, F_in, F_out, dtype, relu, seed, few):
    g = torch.Generator(device="cuda").manual_seed(seed)
    m, E = sum(sizes), len(sizes)
    n = m
    order = torch.randperm(n, generator=g, device="cuda")
    X, G, H = B._padded(n, F_in, dtype, "cuda"), B._padded(n, F_out, dtype, "cuda"), B._padded(n, F_out, dtype, "cuda")
    X.copy_(whole((n, F_in), 3, g)), G.copy_(whole((n, F_out), 3, g)), H.copy_(whole((n, F_out), 3, g))
    W, b = whole((E, F_in, F_out), 3, g), whole((E, F_out), 9, g)
    assert 9 * max(F_in, F_out, max(sizes)) + 9 < 2 ** 24
    offsets = torch.tensor([0] + list(sizes), device="cuda").cumsum(0).int()
    act = B.TMA_ACT_RELU if relu else B.TMA_ACT_NONE
    Y, dX = torch.full_like(G, 7.0), torch.full_like(X, 7.0)
    B.tma_profile_begin(None)
    B.tma_grouped_dense_fwd(X, W, b, offsets, act, order=order.int(), Y_out=Y)
    dW, db, _ = B.tma_grouped_dense_bwd(X, H if relu else None, G, W, offsets, act, order=order.int(), dX_out=dX)
    ran = B.tma_profile_end()
    assert all(("few" in name) == few for name in ran if name.startswith("grouped")), (ran, few)
    at = 0
    for e, size in enumerate(sizes):
        r = order[at:at + size]
        at += size
        x, w, z = X[r].double(), W[e].double(), (G[r] * (H[r] > 0) if relu else G[r]).double()
        want = x @ w + b[e].double()
        want = (want.clamp(min=0) if relu else want).to(dtype)
        assert torch.equal(Y[r], want), f"Y of group {e}: {int((Y[r] != want).sum())} of {want.numel()} off"
        want = (z @ w.T).to(dtype)
        assert torch.equal(dX[r], want), f"dX of group {e}: {int((dX[r] != want).sum())} of {want.numel()} off"
        want = (x.T @ z).float()
        assert torch.equal(dW[e], want), f"dW of group {e}: {int((dW[e] != want).sum())} of {want.numel()} off"
        assert torch.equal(db[e], z.sum(0).float()), f"db of group {e}"


# at most two rows a group on average in bf16 (six in fp32), and groups of far more
SKEWED = {"seventeen": [17] + [0] * 9, "eight": [0, 8, 0, 0], "nine": [0, 0, 9, 0, 0], "mixed": [0] * 5 + [1] * 40 + [77] + [0] * 60 + [9], "one_of_many": [0] * 500 + [900] + [0] * 523}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("name,F_in,F_out", [(name, fi, fo) for name in SKEWED for fi, fo in
                                             [(1, 1), (33, 70), (256, 256), (530, 40), (40, 530), (1_100, 129), (129, 1_100)]
                                             if name != "one_of_many" or fi * fo < 10_000])
def test_few_rows_on_average_and_groups_of_many(B, name, F_in, F_out, dtype):
    for relu in (False, True):
        check(B, SKEWED[name], F_in, F_out, dtype, relu, F_in + relu, True)


@pytest.mark.parametrize("per", [6, 7])
def test_both_sides_of_the_line_in_fp32(B, per):
    check(B, [per * 4, 0, 0, 0], 100, 60, torch.float32, True, per, per == 6)


@pytest.mark.parametrize("per", [2, 3])
def test_both_sides_of_the_line_in_bf16(B, per):
    check(B, [0, per * 4, 0, 0], 100, 60, torch.bfloat16, True, per, per == 2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes,F_in,F_out", [([130, 0, 63, 1], 65, 101), ([900, 3, 0, 2_000], 128, 256), ([40] * 30, 47, 33), ([300_000, 5, 20_000], 128, 64),
                                              ([200_000], 43, 130), ([60_000, 61_000], 300, 131)])
def test_tiles_and_resident_weights(B, sizes, F_in, F_out, dtype):
    for relu in (False, True):
        check(B, sizes, F_in, F_out, dtype, relu, 3 + relu, False)


# rows over (runs in flight - groups): 1,300,000 / 509 and 120,013 / 26, each more than two lists of 1,024 and one (the second: two) of 2,048
@pytest.mark.parametrize("relu", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes,F_in,F_out", [([1_200_000, 0, 100_000], 9, 7), ([100_000, 13, 20_000], 700, 690)])
def test_weight_gradients_of_long_runs(B, sizes, F_in, F_out, dtype, relu):
    check(B, sizes, F_in, F_out, dtype, relu, 11, False)
