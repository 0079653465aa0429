"""Products in 8-bit integers on the GPU, against the oracle.

Tolerances.  Without a norm the integers and scales of a bf16 row are the oracle's bit for bit and the sum is exact, so an output is off by the
rounding to bf16, 2^-8 of itself, and three fp32 roundings.  With a norm, whose values are off by some 4e-7, an integer may be its neighbour:
of 2048 values with up to 127 steps that is one in ten rows, so up to three in a row are allowed, each of which moves an output by
s_t |w|.  The layer: a neighbouring integer in x moves hidden values of that token by about a thousandth, and with them as many of their
integers; 1e-2 of the whole output's norm."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as B
from paper_2601_10639_amd import stemlib as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
bf = torch.bfloat16


def make_ctx(T, d, F=None, V=100):
    return L.stem_create(d, F or d, V, L.STEM_BF16, T, reserve=L.STEM_RESERVE_QUANT)


def draw(seed, *shape, std=1.0, mean=0.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * std + mean).to(bf).to(DEV)


def num(t):
    return t.double().cpu().numpy()


def integers(w):
    """The [N, K] integers of a StemQuant, out of the blocks they lie in."""
    G, P = -(-w.N // 32), -(-w.K // 128) * 128
    return w.q.cpu().numpy().reshape(G, P // 32, 2, 32, 16).transpose(0, 3, 1, 2, 4).reshape(G * 32, P)


@pytest.mark.parametrize("N,K", [(1, 1), (3, 17), (32, 128), (33, 129), (100, 1999), (64, 4096), (31, 4104), (5, 8192), (40, 8193), (7, 20000)])
def test_weights(N, K):
    ctx = make_ctx(1, 64)
    W = draw(1, N, K, std=0.02)
    W[0] = 0
    if N > 2:
        W[2, K // 2] = float("inf")
    w = L.stem_quant_weights(ctx, W)
    q, s = B.quantise(W.float().cpu().numpy())
    got = integers(w)
    assert (got[:N, :K] == q).all() and (got[:, K:] == 0).all() and (got[N:] == 0).all()
    assert np.array_equal(w.scale.cpu().numpy(), s[:, 0], equal_nan=True)


def check_linear(ctx, T, N, K, norm_kind=None, residual=False, seed=3):
    x, W = draw(seed, T, K) * draw(seed + 1, T, 1, std=0.5, mean=2.0), draw(seed + 2, N, K, std=0.05)
    res = draw(seed + 3, T, N) if residual else None
    w = L.stem_quant_weights(ctx, W)
    y = torch.full((T, N), float("nan"), dtype=bf, device=DEV)
    v, norm, slack = x.float().cpu().numpy(), None, 0.0
    if norm_kind:
        g = draw(seed + 4, K, std=0.2, mean=1.0)
        norm = L.stem_norm(norm_kind, 1e-5, g)
        v = B.norm(v, {1: "rms", 2: "layer"}[norm_kind], 1e-5)[0] * num(g)
        slack = 3 * B.quantise(v)[1].astype(np.float64) * np.abs(num(W)).max(1)[None, :]
    L.stem_quant_linear(ctx, x, w, y, residual=res, norm=norm)
    want = B.quant_product(v, W.float().cpu().numpy()) + (num(res) if residual else 0.0)
    off = np.abs(num(y) - want)
    assert (off <= np.abs(want) * 2.0 ** -8 + slack + 1e-6 * np.abs(want).max()).all(), off.max()
    if residual:   # in place
        L.stem_quant_linear(ctx, x, w, res, residual=res, norm=norm)
        assert torch.equal(res, y)


# from one token and one channel on; sides that fill neither a block of 32 nor one of 128; token counts around every tile's edge
LINEAR = [(1, 1, 1), (1, 1, 64), (1, 64, 17), (2, 33, 100), (5, 4096, 1024), (16, 130, 700), (31, 64, 128), (33, 1000, 2047), (64, 512, 512), (65, 513, 640),
          (127, 300, 1999), (128, 256, 256), (129, 260, 1024), (200, 2048, 640), (255, 255, 255), (257, 257, 384), (300, 999, 2048), (513, 1024, 300),
          (700, 1001, 1999), (1024, 1024, 1024), (1111, 36, 65), (2049, 768, 1111), (4100, 520, 130)]


@pytest.mark.parametrize("T,N,K", LINEAR)
def test_linear(T, N, K):
    check_linear(make_ctx(T, 2048), T, N, K)
    check_linear(make_ctx(T, 2048), T, N, K, residual=True, seed=30)


@pytest.mark.parametrize("T,N,K,kind", [(1, 96, 64, 1), (3, 4096, 2048, 1), (32, 100, 1999, 2), (40, 512, 1024, 2), (300, 640, 2000, 1), (9, 64, 5000, 2), (3, 40, 9000, 1)])
def test_linear_behind_a_norm(T, N, K, kind):
    check_linear(make_ctx(T, 9024), T, N, K, kind, residual=T % 2 == 1)


def test_long_rows():
    check_linear(make_ctx(40, 64, 40000), 40, 96, 40000)


def test_rows_with_nan_and_zeros_stay_by_themselves():
    T, N, K = 70, 200, 512
    ctx = make_ctx(T, 512)
    x, W = draw(1, T, K), draw(2, N, K, std=0.05)
    w = L.stem_quant_weights(ctx, W)
    y, z = torch.empty(T, N, dtype=bf, device=DEV), torch.empty(T, N, dtype=bf, device=DEV)
    L.stem_quant_linear(ctx, x, w, y)
    x[3], x[40, 5], x[69, 511] = 0, float("nan"), float("-inf")
    L.stem_quant_linear(ctx, x, w, z)
    rest = [t for t in range(T) if t not in (3, 40, 69)]
    assert torch.equal(y[rest], z[rest]) and (z[3] == 0).all()
    assert torch.isnan(z[40]).all() and torch.isnan(z[69]).all()


FFN = [(1, 64, 64), (1, 1024, 4096), (3, 128, 320), (17, 448, 1472), (32, 256, 1024), (33, 256, 1024), (64, 512, 1536), (100, 896, 2624), (200, 64, 192),
       (256, 512, 2048), (300, 320, 1088), (700, 512, 1408), (4200, 128, 384)]


@pytest.mark.parametrize("T,d,F", FFN)
@pytest.mark.parametrize("norm_kind", [None, 1])
def test_ffn(T, d, F, norm_kind):
    V = 50
    ctx = make_ctx(T, d, F, V)
    x, Wg, Wd, E = draw(1, T, d), draw(2, F, d, std=1.5 * d ** -0.5), draw(3, d, F, std=F ** -0.5), draw(4, V, F)
    ids = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(5), dtype=torch.int32).to(DEV)
    g, d8 = L.stem_quant_weights(ctx, Wg), L.stem_quant_weights(ctx, Wd)
    w = draw(6, d, std=0.2, mean=1.0)
    norm = L.stem_norm(norm_kind, 1e-5, w) if norm_kind else None
    y = torch.full((T, d), float("nan"), dtype=bf, device=DEV)
    L.stem_quant_ffn_forward(ctx, x, ids, g, d8, E, y, norm=norm)
    L.stem_sync_status(ctx)
    n = B.norm(num(x), "rms", 1e-5)[0] * num(w) if norm_kind else num(x)
    want = B.quant_ffn(n, Wg.float().cpu().numpy(), Wd.float().cpu().numpy(), num(E)[ids.cpu().numpy()])
    assert np.linalg.norm(num(y) - want) <= 1e-2 * np.linalg.norm(want)
    assert np.abs(num(y) - want).max() <= 0.1 * np.abs(want).max()
    # the residual stream in place
    plain = y.clone()
    r = x.clone()
    L.stem_quant_ffn_forward(ctx, r, ids, g, d8, E, r, residual=r, norm=norm)
    assert np.linalg.norm(num(r) - num(x) - want) <= 1e-2 * np.linalg.norm(want) + 2.0 ** -8 * np.linalg.norm(num(r))
    # the same bits again
    L.stem_quant_ffn_forward(ctx, x, ids, g, d8, E, y, norm=norm)
    assert torch.equal(y, plain)


def test_ffn_is_the_layer():
    """Against the bf16 layer of the same weights: what 8 bits cost."""
    T, d, F, V = 300, 512, 2048, 100
    ctx = make_ctx(T, d, F, V)
    x, Wg, Wd, E = draw(1, T, d), draw(2, F, d, std=d ** -0.5), draw(3, d, F, std=F ** -0.5), draw(4, V, F)
    ids = torch.randint(0, V, (T,), dtype=torch.int32).to(DEV)
    y, z = torch.empty_like(x), torch.empty_like(x)
    L.stem_ffn_forward(ctx, x, ids, Wg, Wd, E, y)
    L.stem_quant_ffn_forward(ctx, x, ids, L.stem_quant_weights(ctx, Wg), L.stem_quant_weights(ctx, Wd), E, z)
    # rms of a rounding: 0.29 of a step of max / 127, max 3 to 10 times the rms: 0.7 to 2.3 % in each of four operands
    assert np.linalg.norm(num(y) - num(z)) <= 0.06 * np.linalg.norm(num(y))


def test_ids_outside_the_table_are_reported():
    T, d, F, V = 40, 64, 128, 10
    ctx = make_ctx(T, d, F, V)
    x, E = draw(1, T, d), draw(4, V, F)
    g, d8 = L.stem_quant_weights(ctx, draw(2, F, d)), L.stem_quant_weights(ctx, draw(3, d, F))
    ids = torch.zeros(T, dtype=torch.int32, device=DEV)
    y, z = torch.empty_like(x), torch.empty_like(x)
    L.stem_quant_ffn_forward(ctx, x, ids, g, d8, E, y)
    L.stem_sync_status(ctx)
    ids[7], ids[39] = V, -1
    L.stem_quant_ffn_forward(ctx, x, ids, g, d8, E, z)
    with pytest.raises(L.StemError) as e:
        L.stem_sync_status(ctx)
    assert e.value.status == L.STEM_ERR_ID_RANGE
    rest = [t for t in range(T) if t != 7]
    assert torch.equal(y[rest], z[rest])      # -1 is clamped to row 0, which all others name


def test_graph_replays_and_another_stream():
    T, d, F, V = 20, 256, 512, 64
    ctx = make_ctx(T, d, F, V)
    x, E = draw(1, T, d), draw(4, V, F)
    g, d8 = L.stem_quant_weights(ctx, draw(2, F, d, std=0.06)), L.stem_quant_weights(ctx, draw(3, d, F, std=0.04))
    ids = torch.arange(T, dtype=torch.int32, device=DEV)
    y, lin = torch.empty_like(x), torch.empty(T, F, dtype=bf, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        L.stem_quant_ffn_forward(ctx, x, ids, g, d8, E, y)
        L.stem_quant_linear(ctx, x, g, lin)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        L.stem_quant_ffn_forward(ctx, x, ids, g, d8, E, y)
        L.stem_quant_linear(ctx, x, g, lin)
    for k in range(4):
        x.copy_(draw(10 + k, T, d))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got, gl = y.clone(), lin.clone()
        L.stem_quant_ffn_forward(ctx, x, ids, g, d8, E, y)
        L.stem_quant_linear(ctx, x, g, lin)
        torch.cuda.synchronize()
        assert torch.equal(got, y) and torch.equal(gl, lin)


@pytest.mark.parametrize("T,N,K", [(1, 512, 512), (5, 700, 700), (40, 96, 96), (100, 256, 256)])
def test_linear_over_its_own_input(T, N, K):
    ctx = make_ctx(T, 704)
    x, w = draw(1, T, K), L.stem_quant_weights(ctx, draw(2, N, K, std=0.05))
    y = torch.empty(T, N, dtype=bf, device=DEV)
    L.stem_quant_linear(ctx, x, w, y)
    L.stem_quant_linear(ctx, x, w, x)
    assert torch.equal(x, y)


@pytest.mark.parametrize("T,F", [(5, 192), (300, 320), (700, 4096)])
def test_ids_outside_the_table_at_other_sizes(T, F):
    d, V = 64, 10
    ctx = make_ctx(T, d, F, V)
    x, E = draw(1, T, d), draw(4, V, F)
    g, d8 = L.stem_quant_weights(ctx, draw(2, F, d)), L.stem_quant_weights(ctx, draw(3, d, F))
    ids = torch.zeros(T, dtype=torch.int32, device=DEV)
    y, z = torch.empty_like(x), torch.empty_like(x)
    L.stem_quant_ffn_forward(ctx, x, ids, g, d8, E, y)
    ids[T - 2] = -7
    L.stem_quant_ffn_forward(ctx, x, ids, g, d8, E, z)
    with pytest.raises(L.StemError) as e:
        L.stem_sync_status(ctx)
    assert e.value.status == L.STEM_ERR_ID_RANGE
    assert torch.equal(y, z)


def test_a_table_row_that_is_no_number_spoils_its_tokens_only():
    T, d, F, V = 200, 128, 320, 20
    ctx = make_ctx(T, d, F, V)
    x, E = draw(1, T, d), draw(4, V, F)
    E[3, 0], E[5, F - 1], E[7, 100] = float("inf"), float("nan"), float("-inf")
    g, d8 = L.stem_quant_weights(ctx, draw(2, F, d, std=0.09)), L.stem_quant_weights(ctx, draw(3, d, F, std=0.05))
    ids = (torch.arange(T, dtype=torch.int32) % V).to(DEV)
    for t in (T, 30, 4):
        y = torch.empty_like(x)
        L.stem_quant_ffn_forward(ctx, x[:t], ids[:t], g, d8, E, y[:t])
        bad = torch.isnan(y[:t]).all(1)
        assert torch.equal(bad, (ids[:t] == 3) | (ids[:t] == 5) | (ids[:t] == 7))
        assert torch.isfinite(y[:t][~bad]).all()


def test_cut_products_give_the_same_bits_whatever_else_the_context_does():
    """K slices exchange through the context's tickets, which other kernels of the context use too."""
    T, d, F, V = 200, 512, 8192, 20
    ctx = make_ctx(T, d, F, V)
    x, h, E = draw(1, T, d), draw(2, T, F), draw(4, V, F)
    w = L.stem_quant_weights(ctx, draw(3, d, F, std=0.05))
    Wg, Wd = draw(5, F, d, std=0.05), draw(6, d, F, std=0.05)
    ids = torch.zeros(T, dtype=torch.int32, device=DEV)
    y, z, o = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    L.stem_quant_linear(ctx, h, w, y)
    for t in (16, 1, T):
        L.stem_ffn_forward(ctx, x[:t], ids[:t], Wg, Wd, E, o[:t])
        L.stem_quant_linear(ctx, h, w, z)
        assert torch.equal(y, z)


def test_refusals():
    T, d, F = 8, 64, 128
    ctx = make_ctx(T, d, F, 10)
    x, y, E = draw(1, T, d), draw(2, T, d), draw(4, 10, F)
    g, d8 = L.stem_quant_weights(ctx, draw(2, F, d)), L.stem_quant_weights(ctx, draw(3, d, F))
    ids = torch.zeros(T, dtype=torch.int32, device=DEV)

    def status(call, *a, **k):
        with pytest.raises(L.StemError) as e:
            call(*a, **k)
        return e.value.status

    bare = L.stem_create(d, F, 10, L.STEM_BF16, T)
    assert status(L.stem_quant_ffn_forward, bare, x, ids, g, d8, E, y) == L.STEM_ERR_WORKSPACE
    assert status(L.stem_quant_linear, bare, x, g, torch.empty(T, F, dtype=bf, device=DEV)) == L.STEM_ERR_WORKSPACE
    f32 = L.stem_create(d, F, 10, L.STEM_F32, T)
    assert status(L.stem_reserve, f32, L.STEM_RESERVE_QUANT) == L.STEM_ERR_UNSUPPORTED
    assert status(L.stem_quant_weights, f32, torch.zeros(F, d, device=DEV)) == L.STEM_ERR_UNSUPPORTED
    assert status(L.stem_quant_weights, ctx, torch.zeros(1, 131073, dtype=bf, device=DEV)) == L.STEM_ERR_SHAPE
    wide = L.stem_quant_weights(ctx, draw(1, 4, 129))
    assert status(L.stem_quant_linear, ctx, draw(1, T, 129), wide, torch.empty(T, 4, dtype=bf, device=DEV)) == L.STEM_ERR_SHAPE
    assert status(L.stem_quant_ffn_forward, ctx, x, ids, g, d8, E, None) == L.STEM_ERR_INVALID_ARG
    assert status(L.stem_quant_ffn_forward, ctx, x, ids, g, d8, E, y, norm=L.stem_norm(5)) == L.STEM_ERR_INVALID_ARG
    both = torch.empty(T * d + 64, dtype=bf, device=DEV)
    assert status(L.stem_quant_ffn_forward, ctx, both[:T * d].view(T, d), ids, g, d8, E, both[64:].view(T, d)) == L.STEM_ERR_INVALID_ARG
    for call in (lambda: L.stem_quant_ffn_forward(ctx, x, ids, d8, g, E, y), lambda: L.stem_quant_ffn_forward(ctx, x.float(), ids, g, d8, E, y),
                 lambda: L.stem_quant_linear(ctx, x, d8, y), lambda: L.stem_quant_linear(ctx, x, g, y)):
        with pytest.raises((TypeError, ValueError)):
            call()
    none = draw(1, 0, d)
    L.stem_quant_ffn_forward(ctx, none, ids[:0], g, d8, E, none)
