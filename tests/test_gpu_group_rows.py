"""Rows by group: the order and offsets of a stable sort by id, whole numbers, compared bit for bit."""
import numpy as np
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


def plain(ids, E):
    inside = (ids >= 0) & (ids < E)
    key = np.where(inside, ids, E)
    order = np.argsort(key, kind="stable")
    offsets = np.searchsorted(key[order], np.arange(E + 1))
    return offsets, order[:offsets[E]]


def draw(n, E, how, seed):
    r = np.random.default_rng(seed)
    if how == "one":
        return np.full(n, E - 1, np.int32)
    if how == "descending":
        return (E - 1 - np.arange(n) * E // max(n, 1)).astype(np.int32)
    ids = r.integers(0, E, n).astype(np.int32)
    if how == "skewed":
        ids = np.where(r.random(n) < 0.9, min(3, E - 1), ids).astype(np.int32)
    if how == "loose":      # ids that are none, the extreme ones among them
        bad = r.choice(np.array([-1, E, -2**31, 2**31 - 1, E + 63], dtype=np.int64), n).astype(np.int32)
        ids = np.where(r.random(n) < 0.4, bad, ids).astype(np.int32)
    return ids


@pytest.mark.parametrize("how", ["even", "skewed", "loose", "one", "descending"])
@pytest.mark.parametrize("n,E", [(0, 1), (0, 600), (1, 1), (1, 1024), (63, 2), (64, 7), (65, 64), (1000, 3), (4097, 512), (5000, 513),
                                 (16384, 16), (16385, 16), (70001, 1), (70001, 100), (70001, 1024), (1_000_003, 33)])
def test_order_and_offsets(B, n, E, how):
    ids = draw(n, E, how, n + E)
    want_offsets, want = plain(ids, E)
    order = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    for _ in range(2):
        offsets, got = B.tma_group_rows(torch.from_numpy(ids).cuda(), E, order_out=order)
        assert np.array_equal(offsets.cpu().numpy(), want_offsets)
        got = got.cpu().numpy()
        assert np.array_equal(got[:len(want)], want)
        assert (got[len(want):] == -7).all()        # behind the last group nothing is written


def test_an_offset_array_and_a_stream_of_its_own(B):
    ids = draw(20001, 9, "loose", 3)
    held = torch.from_numpy(np.concatenate([[5], ids]).astype(np.int32)).cuda()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    offsets, order = B.tma_group_rows(held[1:], 9, stream=s)
    s.synchronize()
    want_offsets, want = plain(ids, 9)
    assert np.array_equal(offsets.cpu().numpy(), want_offsets) and np.array_equal(order.cpu().numpy()[:len(want)], want)


@pytest.mark.parametrize("n", [900, 50_000])
def test_replayed_in_a_graph(B, n):
    E = 12
    ids = torch.from_numpy(draw(n, E, "loose", 1)).cuda()
    offsets, order = torch.zeros(E + 1, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    ws = torch.empty(max(B.tma_group_rows_workspace_bytes(n, E), 256), dtype=torch.uint8, device="cuda")
    B.tma_group_rows(ids, E, offsets_out=offsets, order_out=order, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.tma_group_rows(ids, E, offsets_out=offsets, order_out=order, ws=ws)
    for k in range(4):
        new = draw(n, E, "loose" if k % 2 else "skewed", 50 + k)
        ids.copy_(torch.from_numpy(new))
        order.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        want_offsets, want = plain(new, E)
        assert np.array_equal(offsets.cpu().numpy(), want_offsets)
        assert np.array_equal(order.cpu().numpy()[:len(want)], want) and (order[len(want):] == -7).all()
