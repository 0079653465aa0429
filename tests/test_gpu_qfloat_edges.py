"""Products in 8-bit floating point at the edges of their kernels, in graphs, on other streams, and together with what brings tokens to experts and back.
Tolerances: test_gpu_qfloat.py's."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as B
from oracle import qfloat_oracle as Q
from paper_2601_10639_amd import stemlib as L
from tests.test_gpu_experts import draw_experts
from tests.test_gpu_qfloat import DEV, bf, bound, check_backward, check_ffn, check_linear, cut, dev, draw, f32, i32, make_ctx, num, offsets_of, wide

pytestmark = pytest.mark.gpu

# (T, N, K): what each is there for is held in test_qfloat_reach_cpu.py
TILES = {"ring": (4090, 4090, 4100), "pair": (3000, 1500, 300), "128x128": (2000, 1100, 520), "128x64": (300, 600, 700), "2 slices": (1300, 500, 4100),
         "3 slices": (300, 500, 4096), "4 slices": (300, 500, 5200)}
FEW = {"8 channels": (3, 1000, 1000), "16 channels": (5, 3001, 2000), "32 channels": (16, 5000, 4096), "depth 8": (2, 200, 8192), "turns": (2, 130, 9000),
       "form, depth 1": (17, 1001, 999), "form, depth 2": (40, 333, 1999), "form, depth 4": (100, 500, 4000), "form, depth 8": (33, 300, 8192), "form, turns": (33, 300, 17000),
       "form, 32 rows": (50, 5000, 2000), "form, 32 rows, 16 channels": (250, 1030, 1100)}
GATES = {"64x128": (100, 128, 320), "128x128": (1500, 192, 1600), "pair": (4400, 128, 2240), "few, inline": (8, 256, 1024), "few, by a kernel": (8, 128, 4160),
         "16, by a kernel": (16, 192, 2112)}
WEIGHT_SLICES = (3000, 300, 200)
WEIGHTS = [(9001, 100, 129, 1), (5000, 130, 260, 3), (3200, 2100, 2300, 1), (900, 1000, 3899, 4)]   # T, N, K, groups


def check_rows(ctx, T, N, K, rows):
    """Sampled rows of a large product."""
    x, W, res = draw(1, T, K), draw(2, N, K, std=0.05), draw(3, T, N)
    y = torch.empty(T, N, dtype=bf, device=DEV)
    L.stem_qfloat_linear(ctx, x, L.stem_qfloat_weights(ctx, W), y, residual=res)
    a, b = num(x[rows]), num(W)
    want, size = Q.linear(a, b[None])
    want = want + num(res[rows])
    assert (np.abs(num(y[rows]) - want) <= np.abs(want) * 2.0 ** -8 * (1 + 2 ** -7) + cut(a, b, size) + 2.0 ** -22 * np.abs(want)).all()
    again = torch.empty_like(y)
    L.stem_qfloat_linear(ctx, x, L.stem_qfloat_weights(ctx, W), again, residual=res)
    assert torch.equal(y, again)


@pytest.mark.parametrize("name", TILES)
def test_tiles(name):
    T, N, K = TILES[name]
    rows = np.unique(np.concatenate([np.arange(3), [T // 2, T - 2, T - 1], np.random.default_rng(1).integers(0, T, 200)]))
    check_rows(make_ctx(T, 64, wide(K)), T, N, K, rows)


@pytest.mark.parametrize("name", FEW)
def test_few_rows(name):
    T, N, K = FEW[name]
    ctx = make_ctx(T, 64, wide(K))
    y = check_linear(ctx, T, N, K, residual=True)
    check_linear(ctx, T, N, K, norm_kind=L.STEM_NORM_LAYER if K % 2 else L.STEM_NORM_RMS)
    # the same bits again
    x, W = draw(3, T, K) * draw(4, T, 1, std=0.5, mean=2.0), draw(5, 1, N, K, std=0.05)
    w = L.stem_qfloat_weights(ctx, W)
    again = torch.empty(T, N, dtype=bf, device=DEV)
    L.stem_qfloat_linear(ctx, x, w, again, residual=draw(6, T, N))
    assert torch.equal(again, y)


@pytest.mark.parametrize("name", GATES)
def test_gates(name):
    T, d, F = GATES[name]
    check_ffn(make_ctx(T, d, F), T, d, F)


def test_few_rows_of_groups():
    """Up to 8 rows, which every group's workgroups look for."""
    for T, groups, N, K in ((8, 3, 70, 200), (7, 512, 40, 130), (1, 5, 300, 1000), (8, 8, 1300, 2100)):
        ctx = make_ctx(T, 64, wide(K), groups=groups)
        check_linear(ctx, T, N, K, groups, offsets_of(T, T, groups), residual=True)
        check_linear(ctx, T, N, K, groups, np.array([0] + [T // 2] * (groups - 1) + [T], np.int32), norm_kind=L.STEM_NORM_RMS)


def test_one_group_with_offsets():
    """Rows in front of it and behind it are left as they were; the weight gradient is that of its rows."""
    T, N, K = WEIGHT_SLICES
    ctx = make_ctx(T, 64, 320, backward=True)
    for offsets in ([0, T], [7, T - 100], [5, 5], [T, T]):
        check_linear(ctx, T, N, K, 1, np.array(offsets, np.int32), residual=True)
        check_backward(ctx, T, N, K, 1, np.array(offsets, np.int32))


def test_weight_gradient_in_slices():
    T, N, K = WEIGHT_SLICES
    check_backward(make_ctx(T, 64, 320, backward=True), T, N, K)


@pytest.mark.parametrize("T,N,K,groups", WEIGHTS)
def test_weight_gradients_in_slices_and_pairs(T, N, K, groups):
    """Also of groups without rows, and of one that has nearly all, whose slices are those of the average."""
    ctx = make_ctx(T, 64, wide(K, N), groups=groups, backward=True)
    if groups == 1:
        check_backward(ctx, T, N, K)
    else:
        check_backward(ctx, T, N, K, groups, offsets_of(T, T, groups))
        check_backward(ctx, T, N, K, groups, np.array([3] * (groups - 1) + [T - 60, T], np.int32))


@pytest.mark.parametrize("T", [2, 40])
def test_output_over_the_input(T):
    N = K = 256
    ctx = make_ctx(T, 64, 256)
    x, w = draw(1, T, K), L.stem_qfloat_weights(ctx, draw(2, N, K, std=0.05))
    y = torch.empty(T, N, dtype=bf, device=DEV)
    L.stem_qfloat_linear(ctx, x, w, y)
    L.stem_qfloat_linear(ctx, x, w, x)
    assert torch.equal(x, y)


def test_outputs_beyond_32_bits():
    """More than 2^31 elements, and weight gradients of more than 2^32 bytes: the last rows and channels."""
    T, N, K = 33100, 65536, 64
    ctx = make_ctx(T, 64, 64)
    x, W = draw(1, T, K), draw(2, N, K, std=0.05)
    y = torch.empty(T, N, dtype=bf, device=DEV)
    L.stem_qfloat_linear(ctx, x, L.stem_qfloat_weights(ctx, W), y)
    rows, first = [0, T // 2, T - 129, T - 1], N - 512
    a, b = num(x[rows]), num(W[first:])
    want, size = Q.linear(a, b[None])
    assert (np.abs(num(y[rows][:, first:]) - want) <= np.abs(want) * 2.0 ** -8 * (1 + 2 ** -7) + cut(a, b, size)).all()
    del y
    T, N, K = 3, 33000, 33100
    ctx = make_ctx(T, 64, 33152, backward=True)
    dy, x = draw(3, T, N), draw(4, T, K)
    dW = torch.empty(N, K, device=DEV)
    W = L.StemQfloat(torch.empty(L.stem_qfloat_bytes(N, K), dtype=torch.uint8, device=DEV), None, 1, N, K)   # (only its shape is used here)
    L.stem_qfloat_linear_backward(ctx, dy, x, W, dW=dW)
    for n, k in ((0, 0), (N - 300, K - 300)):
        want = num(dy)[:, n:n + 300].T @ num(x)[:, k:k + 300]
        size = np.abs(num(dy)[:, n:n + 300]).T @ np.abs(num(x)[:, k:k + 300])
        assert (np.abs(num(dW[n:n + 300, k:k + 300]) - want) <= bound(T) * size).all()


def test_rows_beyond_32_bits():
    """Dispatch and combine of more than 2^31 elements."""
    T, k, width = 70000, 2, 16384
    ctx = L.stem_create(64, 64, 10, L.STEM_BF16, T)
    e = torch.randint(0, 4, (T, k), generator=torch.Generator().manual_seed(1)).to(i32).to(DEV)
    src, place, off = torch.empty(T * k, dtype=i32, device=DEV), torch.empty(T, k, dtype=i32, device=DEV), torch.empty(5, dtype=i32, device=DEV)
    L.stem_experts_sort(ctx, e, src, place, off)
    flat = e.reshape(-1).long()
    assert torch.equal(src.long(), torch.sort(flat, stable=True).indices)
    x = torch.empty(T, width, dtype=bf, device=DEV).normal_()
    xs, y = torch.empty(T * k, width, dtype=bf, device=DEV), torch.empty(T, width, dtype=bf, device=DEV)
    L.stem_experts_dispatch(ctx, x, src, xs, choices=k)
    at = torch.tensor([0, T, T * k - 2, T * k - 1], device=DEV)
    assert torch.equal(xs[at], x[src[at].long() // k])
    L.stem_experts_combine(ctx, xs, place, y)
    assert torch.equal(y, x + x)


def experts_layer(ctx, x, ids, e, w, gate, down, E, norm, bufs):
    """A mixture of layers: every token's choices go through their expert's layer, and come back weighted onto the residual stream."""
    src, place, off, xs, ids_s, ys, y = bufs
    L.stem_experts_sort(ctx, e, src, place, off)
    L.stem_experts_dispatch(ctx, x, src, xs, choices=e.shape[1], ids=ids, ids_out=ids_s)
    L.stem_qfloat_ffn_forward(ctx, xs, ids_s, gate, down, E, ys, norm=norm, offsets=off)
    L.stem_experts_combine(ctx, ys, place, y, weights=w, residual=x)
    return y


def experts_case(T, k, n, d, F, V=50, seed=1):
    rows = T * k
    ctx = make_ctx(rows, d, F, groups=n)
    x, E, g = draw(seed, T, d), draw(seed + 1, V, F), draw(seed + 2, d, std=0.2, mean=1.0)
    Wg, Wd = draw(seed + 3, n, F, d, std=0.05), draw(seed + 4, n, d, F, std=0.05)
    ids = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(seed)).to(i32).to(DEV)
    e = torch.from_numpy(draw_experts(seed, T, k, n)).to(DEV)
    w = torch.softmax(torch.randn(T, k, generator=torch.Generator().manual_seed(seed)), 1).to(DEV)
    bufs = (torch.empty(rows, dtype=i32, device=DEV), torch.empty(T, k, dtype=i32, device=DEV), torch.empty(n + 1, dtype=i32, device=DEV),
            torch.empty(rows, d, dtype=bf, device=DEV), torch.empty(rows, dtype=i32, device=DEV), torch.empty(rows, d, dtype=bf, device=DEV),
            torch.empty(T, d, dtype=bf, device=DEV))
    gate, down = L.stem_qfloat_weights(ctx, Wg), L.stem_qfloat_weights(ctx, Wd)
    return ctx, (x, ids, e, w, gate, down, E, L.stem_norm(L.STEM_NORM_RMS, 1e-5, g), bufs), (Wg, Wd, g)


@pytest.mark.parametrize("T,k,n,d,F", [(1, 2, 4, 64, 128), (3, 2, 8, 128, 320), (50, 2, 5, 128, 320), (400, 3, 7, 192, 256)])
def test_mixture_of_layers(T, k, n, d, F):
    ctx, args, (Wg, Wd, g) = experts_case(T, k, n, d, F)
    x, ids, e, w, _, _, E, _, _ = args
    y = experts_layer(ctx, *args)
    normed = B.norm(x.float().cpu().numpy(), "rms", 1e-5)[0] * num(g)
    want, size = num(x).copy(), np.zeros(T)
    for j in range(k):
        for t in range(T):
            m = int(e[t, j])
            if m >= 0:
                out = Q.ffn(normed[t:t + 1], ids[t:t + 1].cpu().numpy(), num(Wg[m:m + 1]), num(Wd[m:m + 1]), num(E))[0]
                want[t] += float(w[t, j]) * out
                size[t] += float(w[t, j]) * np.linalg.norm(out)
    # the layers' outputs are rounded to bf16 on their way, and differ by neighbours; then the sum
    off = np.linalg.norm(num(y) - want, axis=1)
    assert (off <= 2.0 ** -8 * np.linalg.norm(want, axis=1) + (2.0 ** -8 + 5000 ** -0.5) * size).all()


def test_training_through_experts():
    """The gradients of sum(dy * combine(linear(dispatch(x)))) for x, the weights and the router's weights, as the formulas give them."""
    T, k, n, K, N = 150, 2, 5, 136, 72
    rows = T * k
    ctx = make_ctx(rows, 64, 192, groups=n, backward=True)
    x, W, dy = draw(1, T, K), draw(2, n, N, K, std=0.05), draw(3, T, N)
    e_host = draw_experts(4, T, k, n)
    e, w = torch.from_numpy(e_host).to(DEV), torch.rand(T, k, generator=torch.Generator().manual_seed(5)).to(DEV)
    src, place, off = torch.empty(rows, dtype=i32, device=DEV), torch.empty(T, k, dtype=i32, device=DEV), torch.empty(n + 1, dtype=i32, device=DEV)
    xs, ys, dys, dxs = (torch.zeros(rows, m, dtype=bf, device=DEV) for m in (K, N, N, K))
    y, dx, dW, dw = torch.empty(T, N, dtype=bf, device=DEV), torch.empty(T, K, dtype=bf, device=DEV), torch.empty(n, N, K, device=DEV), torch.empty(T, k, device=DEV)
    q = L.stem_qfloat_weights(ctx, W, backward=True)
    L.stem_experts_sort(ctx, e, src, place, off)
    L.stem_experts_dispatch(ctx, x, src, xs, choices=k)
    L.stem_qfloat_linear(ctx, xs, q, ys, offsets=off)
    L.stem_experts_combine(ctx, ys, place, y, weights=w)
    L.stem_experts_combine_backward(ctx, dy, place, dys, ys=ys, weights=w, dweights=dw)
    L.stem_qfloat_linear_backward(ctx, dys, xs, q, dxs, dW, offsets=off)
    L.stem_experts_combine(ctx, dxs, place, dx)
    qW = [Q.squares(num(W[m])) for m in range(n)]
    qx = Q.blocks(num(x), 1)
    want_dx, want_dW, size_dx = np.zeros((T, K)), np.zeros((n, N, K)), np.zeros(T)
    for t in range(T):
        for j in range(k):
            m = e_host[t, j]
            if m < 0:
                assert dw[t, j] == 0
                continue
            out = qx[t] @ qW[m].T
            rounded = num(torch.from_numpy(out).to(bf))
            # (an output next to the middle between two values may be either)
            assert abs(float(dw[t, j]) - num(dy)[t] @ rounded) <= (2.0 ** -7 + 2.0 ** -18 * N) * np.abs(num(dy)[t]) @ np.abs(out)
            grad = num((w[t, j] * dy[t].float()).to(bf))
            part = Q.blocks(grad[None], 1)[0] @ qW[m]
            want_dx[t] += part
            size_dx[t] += np.linalg.norm(part)
            want_dW[m] += np.outer(grad, num(x)[t])
    assert (np.linalg.norm(num(dx) - want_dx, axis=1) <= 2.0 ** -8 * (np.linalg.norm(want_dx, axis=1) + size_dx) + 1e-4 * size_dx).all()
    assert np.abs(num(dW) - want_dW).max() <= bound(rows) * rows * np.abs(num(dy)).max() * np.abs(num(x)).max()


def test_graph_of_a_mixture():
    """Captured once, replayed on other tokens and other experts, with eager calls and synchronisations between; every replay against the eager result."""
    ctx, args, _ = experts_case(70, 2, 6, 128, 320)
    x, ids, e, w, gate, down, E, norm, bufs = args
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        experts_layer(ctx, *args)                           # (once outside, as graphs want it)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        experts_layer(ctx, *args)
    for seed in range(4):
        x.copy_(draw(100 + seed, *x.shape))
        e.copy_(torch.from_numpy(draw_experts(200 + seed, *e.shape, 6)).to(DEV))
        ids.copy_(torch.randint(0, 50, ids.shape, generator=torch.Generator().manual_seed(seed)).to(i32).to(DEV))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        replayed = bufs[-1].clone()
        bufs[-1].zero_()
        assert torch.equal(replayed, experts_layer(ctx, *args))
        torch.cuda.synchronize()


def test_graph_of_gradients():
    T, N, K = 700, 300, 200
    for groups, offsets in ((1, None), (3, offsets_of(1, T, 3))):
        ctx = make_ctx(T, 64, 320, groups=groups, backward=True)
        dy, x, w = draw(1, T, N), draw(2, T, K), L.stem_qfloat_weights(ctx, draw(3, groups, N, K, std=0.05), backward=True)
        dx, dW, o = torch.zeros(T, K, dtype=bf, device=DEV), torch.zeros(groups, N, K, device=DEV), dev(offsets)
        call = lambda accumulate: L.stem_qfloat_linear_backward(ctx, dy, x, w, dx, dW, offsets=o, accumulate=accumulate)
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            call(False)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call(True)
        for seed in range(3):
            dy.copy_(draw(50 + seed, T, N))
            torch.cuda.synchronize()
            call(False)
            once, first = dW.clone(), dx.clone()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(dW, once + once) and torch.equal(dx, first)


def test_streams():
    """A call on a stream that is given, and on the current one, waits for nothing else and is waited for by nothing else."""
    T, N, K = 200, 256, 256
    a, b = make_ctx(T, 64, 256), make_ctx(T, 64, 256)
    x, w = draw(1, T, K), L.stem_qfloat_weights(a, draw(2, N, K, std=0.05))
    want = torch.empty(T, N, dtype=bf, device=DEV)
    L.stem_qfloat_linear(a, x, w, want)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    y1, y2 = torch.empty_like(want), torch.empty_like(want)
    for _ in range(20):                                      # two contexts at once
        L.stem_qfloat_linear(a, x, w, y1, stream=s1)
        with torch.cuda.stream(s2):
            L.stem_qfloat_linear(b, x, w, y2)
    torch.cuda.synchronize()
    assert torch.equal(y1, want) and torch.equal(y2, want)


def test_two_graphs_of_one_context():
    """Products in slices, whose room and counters both graphs share, replayed in turn with eager calls between."""
    T, N, K = WEIGHT_SLICES
    ctx = make_ctx(T, 64, 4160, backward=True)
    dy, x, w = draw(1, T, N), draw(2, T, K), L.stem_qfloat_weights(ctx, draw(3, N, K, std=0.05), backward=True)
    dx, dW = torch.zeros(T, K, dtype=bf, device=DEV), torch.zeros(N, K, device=DEV)
    T2, N2, K2 = TILES["2 slices"]
    x2, w2, res = draw(4, T2, K2), L.stem_qfloat_weights(ctx, draw(5, N2, K2, std=0.05)), draw(6, T2, N2)
    y2 = torch.zeros(T2, N2, dtype=bf, device=DEV)
    calls = [lambda: L.stem_qfloat_linear_backward(ctx, dy, x, w, dx, dW), lambda: L.stem_qfloat_linear(ctx, x2, w2, y2, residual=res)]
    side, graphs = torch.cuda.Stream(), []
    for call in calls:
        with torch.cuda.stream(side):
            call()
        side.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            call()
    for seed in range(3):
        dy.copy_(draw(50 + seed, T, N))
        x2.copy_(draw(60 + seed, T2, K2))
        for call in calls:
            call()
        want = dx.clone(), dW.clone(), y2.clone()
        for _ in range(2):
            for t in (dx, dW, y2):
                t.zero_()
            for g in graphs:
                g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip((dx, dW, y2), want))


@pytest.mark.parametrize("T,N", [(5, 333), (300, 1001), (3000, 1503), (4090, 4090)])
def test_input_residual_and_output_are_one(T, N):
    ctx = make_ctx(T, 64, wide(N))
    x, w, y = draw(1, T, N), L.stem_qfloat_weights(ctx, draw(2, N, N, std=0.05)), torch.empty(T, N, dtype=bf, device=DEV)
    L.stem_qfloat_linear(ctx, x, w, y, residual=x)
    L.stem_qfloat_linear(ctx, x, w, x, residual=x)
    assert torch.equal(x, y)


@pytest.mark.parametrize("T", [1, 7])
def test_few_tokens_of_a_wide_layer(T):
    """Rows too long to be made to operands in place: the gate product's tiles, then few rows of their form."""
    check_ffn(make_ctx(T, 8256, 128), T, 8256, 128)


@pytest.mark.parametrize("T,K", [(9000, 700), (9000, 1024), (2500, 2999), (2500, 4096), (1500, 5001), (130, 8000), (40, 9001)])
def test_rows_behind_a_norm(T, K):
    """Each number of lanes a row, chunk and row tails, by groups too."""
    ctx = make_ctx(T, 64, wide(K), groups=3)
    check_linear(ctx, T, 40, K, norm_kind=L.STEM_NORM_RMS)
    check_linear(ctx, T, 40, K, 3, offsets_of(T, T, 3), norm_kind=L.STEM_NORM_LAYER)
