"""Tokens to experts and back at calls and widths beside those of test_gpu_experts.py, whose tolerances these are."""
import numpy as np
import pytest
import torch

from paper_2601_10639_amd import stemlib as L
from tests.test_gpu_block_bind import count   # noqa: F401 (a fixture)
from tests import test_gpu_experts as E
from tests.test_gpu_experts import DEV, make_ctx

pytestmark = pytest.mark.gpu


def test_a_gradient_of_weights_needs_rows(count):
    """Without dys and ys it is refused, natively and from Python; with a ys of no rows every place is none, and the gradient zero."""
    ctx = make_ctx(4, "f32")
    dy, dw = torch.ones(4, 16, device=DEV), torch.full((4, 2), 9.0, device=DEV)
    place, none = torch.zeros(4, 2, dtype=torch.int32, device=DEV), torch.full((4, 2), -1, dtype=torch.int32, device=DEV)
    for _ in range(2):
        with pytest.raises(L.StemError) as err:
            L.stem_experts_combine_backward(ctx, dy, place, dweights=dw)
        assert err.value.status == L.STEM_ERR_INVALID_ARG
        torch.cuda.synchronize()
        assert (dw == 9).all()
        L.stem_sync_status(ctx)
        count.off()
    L.stem_experts_combine_backward(ctx, dy, none, ys=torch.empty(0, 16, device=DEV), dweights=dw)
    L.stem_sync_status(ctx)
    assert not dw.any()


@pytest.mark.parametrize("T,k,n", [(524288, 1, 512), (131073, 4, 63), (262145, 2, 64), (300001, 1, 1), (35001, 16, 255), (600000, 2, 65), (1 << 20, 16, 512)])
def test_sort_of_many_pairs(T, k, n):
    """Around the number of segments whose counts a kernel of its own adds up, to 16 million pairs."""
    rng = np.random.default_rng(T + n)
    e = np.minimum(rng.integers(0, n, (T, k), dtype=np.int16), rng.integers(-(n // 9) - 1, n, (T, k), dtype=np.int16))      # some are liked more, some none
    e[T // 3:T // 3 + 5000] = n - 1                                                                       # a segment of one kind
    flat = np.where(e < 0, n, e).reshape(-1).astype(np.int16)
    order, counts = np.argsort(flat, kind="stable").astype(np.int32), np.bincount(flat, minlength=n + 1)
    end = T * k - counts[n]
    place = np.full(T * k, -1, np.int32)
    place[order[:end]] = np.arange(end)
    order[end:] = -1
    ctx, experts = make_ctx(T), torch.from_numpy(e.astype(np.int32)).to(DEV)
    src, got, offsets = (torch.full(s, -7, dtype=torch.int32, device=DEV) for s in ((T * k,), (T, k), (n + 1,)))
    for _ in range(2):
        L.stem_experts_sort(ctx, experts, src, got, offsets)
        assert np.array_equal(src.cpu().numpy(), order) and np.array_equal(got.cpu().numpy().reshape(-1), place)
        assert np.array_equal(offsets.cpu().numpy(), np.concatenate([[0], np.cumsum(counts[:n])]))


def test_graph_of_a_sort_of_many_pairs():
    """Captured, replayed on other experts between eager sorts of another size, which use the same counts."""
    T, k, n = 300000, 2, 40
    ctx = make_ctx(T)
    draw = lambda seed, rows: torch.randint(-2, n, (rows, k), generator=torch.Generator().manual_seed(seed), dtype=torch.int32).to(DEV)
    outs = lambda rows: [torch.zeros(s, dtype=torch.int32, device=DEV) for s in ((rows * k,), (rows, k), (n + 1,))]
    e, a, b, few = draw(0, T), outs(T), outs(T), outs(9000)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        L.stem_experts_sort(ctx, e, *a)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        L.stem_experts_sort(ctx, e, *a)
    for seed in range(1, 4):
        e.copy_(draw(seed, T))
        L.stem_experts_sort(ctx, e, *b)
        L.stem_experts_sort(ctx, draw(9, 9000), *few)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(a, b))


# rows of more than one turn of a lane's pieces, with a last piece that lies over the one before it, and in place one element at a time
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,k,n,width", [(37, 2, 5, 2049), (30, 3, 4, 4099), (21, 2, 3, 8191), (19, 1, 3, 1025), (40, 4, 6, 2052), (3, 16, 9, 16387)])
def test_rows_of_more_than_one_turn(T, k, n, width, dtype):
    E.test_dispatch(T, k, n, width, dtype)
    for weights in (True, False):
        E.test_combine(T, k, n, width, weights, dtype)
    E.test_combine_backward(T, k, n, width, dtype)
