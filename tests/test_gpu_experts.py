"""Tokens to experts and back on the GPU, against plain loops in 64 bits.

Tolerances.  The sort and the dispatched rows are the oracle's exactly.  A combined row is one fp32 sum of k products and the residual, each step rounded to
half a unit, and one rounding to the type: (k + 1) 2^-24 of the sum of magnitudes, and eps / 2 of the value.  A weight's gradient is an fp32 sum of width
products: each lane adds width / 64 (rounded up to its vectors of at most 8) of them in turn and six steps join the lanes, so (width / 64 + 8 + 6) 2^-24
of the sum of magnitudes.  A row's gradient is one product: eps / 2, and half of 2^-24 in front of it."""
import numpy as np
import pytest
import torch

from paper_2601_10639_amd import stemlib as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": (L.STEM_BF16, torch.bfloat16), "f32": (L.STEM_F32, torch.float32)}


def make_ctx(T, dtype="bf16"):
    return L.stem_create(64, 64, 100, TYPES[dtype][0], max(T, 1))


def draw_experts(seed, T, k, n, none=0.1):
    rng = np.random.default_rng(seed)
    e = np.minimum(rng.integers(0, n, (T, k)), rng.integers(0, n, (T, k)))      # some are liked more
    e[rng.random((T, k)) < none] = -1 - int(rng.integers(0, 3))
    return e.astype(np.int32)


def sorted_by_hand(e, n):
    flat = e.reshape(-1)
    rows = [i for x in range(n) for i in np.nonzero(flat == x)[0]]
    src = np.full(flat.size, -1, np.int32)
    src[:len(rows)] = rows
    place = np.full(flat.size, -1, np.int32)
    place[rows] = np.arange(len(rows))
    return src, place.reshape(e.shape), np.concatenate([[0], np.cumsum([(flat == x).sum() for x in range(n)])])


def sort(ctx, e, n):
    T, k = e.shape
    out = [torch.full(s, -7, dtype=torch.int32, device=DEV) for s in ((T * k,), (T, k), (n + 1,))]
    L.stem_experts_sort(ctx, torch.from_numpy(e).to(DEV), *out)
    return out


# sizes around a wavefront's 64 pairs, a turn's 256 and a segment's 4096; experts around powers of two and to the limit
@pytest.mark.parametrize("T,k,n", [(1, 1, 1), (1, 16, 512), (3, 2, 2), (63, 1, 3), (64, 1, 4), (65, 1, 5), (257, 1, 7), (1000, 3, 8), (1365, 3, 64), (2048, 2, 63),
                                   (2049, 2, 65), (4097, 1, 511), (700, 16, 512), (9001, 2, 256), (20000, 8, 512)])
def test_sort(T, k, n):
    e = draw_experts(T + k, T, k, n)
    ctx = make_ctx(T)
    for src, place, offsets in (sort(ctx, e, n), sort(ctx, e, n)):
        want = sorted_by_hand(e, n)
        assert np.array_equal(src.cpu().numpy(), want[0]) and np.array_equal(place.cpu().numpy(), want[1])
        assert np.array_equal(offsets.cpu().numpy(), want[2])


@pytest.mark.parametrize("value", [-1, 0, 4])
def test_sort_of_one_kind(value):
    T, k, n = 5000, 2, 5
    e = np.full((T, k), value, np.int32)
    src, place, offsets = sort(make_ctx(T), e, n)
    want = sorted_by_hand(e, n)
    assert np.array_equal(src.cpu().numpy(), want[0]) and np.array_equal(place.cpu().numpy(), want[1]) and np.array_equal(offsets.cpu().numpy(), want[2])


def test_sort_of_no_tokens_and_of_unknown_experts():
    ctx = make_ctx(8)
    offsets = torch.full((4,), 9, dtype=torch.int32, device=DEV)
    none = torch.empty(0, 2, dtype=torch.int32, device=DEV)
    L.stem_experts_sort(ctx, none, torch.empty(0, dtype=torch.int32, device=DEV), none.clone(), offsets)
    assert offsets.tolist() == [0, 0, 0, 0]
    e = np.array([[0, 3], [2, 1 << 30], [1, 0]], np.int32)
    src, place, offsets = sort(ctx, e, 3)
    assert place.tolist() == [[0, -1], [3, -1], [2, 1]] and src.tolist() == [0, 5, 4, 2, -1, -1] and offsets.tolist() == [0, 2, 3, 4]
    with pytest.raises(L.StemError) as err:
        L.stem_sync_status(ctx)
    assert err.value.status == L.STEM_ERR_ID_RANGE


def rows_case(seed, T, k, n, width, dtype):
    gen = torch.Generator().manual_seed(seed)
    dt = TYPES[dtype][1]
    e = draw_experts(seed, T, k, n)
    src, place, offsets = sorted_by_hand(e, n)
    draw = lambda *shape: torch.randn(*shape, generator=gen).to(dt)
    return dict(e=e, src=src, place=place, x=draw(T, width), ys=draw(T * k, width), res=draw(T, width), dy=draw(T, width),
                w=torch.rand(T, k, generator=gen), ids=torch.arange(T, dtype=torch.int32) * 7)


WIDTHS = [(1, 1, 1, 8), (5, 2, 3, 1), (33, 3, 4, 7), (64, 2, 16, 1024), (129, 1, 5, 1001), (70, 16, 20, 72), (300, 2, 8, 2048), (9, 4, 6, 8200), (4, 2, 2, 513)]


def num(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,k,n,width", WIDTHS)
def test_dispatch(T, k, n, width, dtype):
    c = rows_case(3, T, k, n, width, dtype)
    xs = torch.full((T * k, width), 5.0, dtype=c["x"].dtype, device=DEV)
    ids = torch.full((T * k,), -5, dtype=torch.int32, device=DEV)
    ctx, src = make_ctx(T, dtype), torch.from_numpy(c["src"]).to(DEV)
    L.stem_experts_dispatch(ctx, c["x"].to(DEV), src, xs, choices=k, ids=c["ids"].to(DEV), ids_out=ids)
    real = c["src"] >= 0
    token = np.maximum(c["src"], 0) // k
    want = np.where(real[:, None], num(c["x"])[token], 5.0)
    assert np.array_equal(num(xs), want) and np.array_equal(ids.cpu().numpy(), np.where(real, token * 7, -5))
    again = torch.full_like(xs, 5.0)
    L.stem_experts_dispatch(ctx, c["x"].to(DEV), src, again, choices=k)
    assert torch.equal(xs, again)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("weights", [True, False])
@pytest.mark.parametrize("T,k,n,width", WIDTHS)
def test_combine(T, k, n, width, weights, dtype):
    c = rows_case(5, T, k, n, width, dtype)
    ctx, dt = make_ctx(T, dtype), c["x"].dtype
    place, ys, w = torch.from_numpy(c["place"]).to(DEV), c["ys"].clone(), c["w"].clone()
    # what has no place counts for nothing, whatever its weight; rows that are nobody's are not read
    w[torch.from_numpy(c["place"] < 0)] = float("nan")
    ys[torch.from_numpy(c["src"] < 0)] = float("inf")
    part = np.where(c["place"][:, :, None] >= 0, num(c["ys"])[np.maximum(c["place"], 0)] * (num(c["w"])[:, :, None] if weights else 1.0), 0.0)
    for res in (None, c["res"]):
        y = torch.full((T, width), float("nan"), dtype=dt, device=DEV)
        r = None if res is None else res.to(DEV)
        L.stem_experts_combine(ctx, ys.to(DEV), place, y, weights=w.to(DEV) if weights else None, residual=r)
        want, size = part.sum(1), np.abs(part).sum(1)
        if res is not None:
            want, size = want + num(res), size + np.abs(num(res))
        assert (np.abs(num(y) - want) <= torch.finfo(dt).eps / 2 * np.abs(want) * (1 + 2 ** -7) + (k + 1) * 2.0 ** -24 * size).all()
        if res is not None:   # in place
            L.stem_experts_combine(ctx, ys.to(DEV), place, r, weights=w.to(DEV) if weights else None, residual=r)
            assert torch.equal(r, y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,k,n,width", WIDTHS)
def test_combine_backward(T, k, n, width, dtype):
    c = rows_case(7, T, k, n, width, dtype)
    ctx, dt = make_ctx(T, dtype), c["x"].dtype
    place, real = torch.from_numpy(c["place"]).to(DEV), c["place"] >= 0
    dy, ys, w = c["dy"].to(DEV), c["ys"].to(DEV), c["w"].to(DEV)
    dys, dw = torch.full((T * k, width), 5.0, dtype=dt, device=DEV), torch.full((T, k), float("nan"), device=DEV)
    L.stem_experts_combine_backward(ctx, dy, place, dys, ys=ys, weights=w, dweights=dw)
    at = np.maximum(c["place"], 0)
    each = num(dy)[:, None, :] * num(ys)[at]
    want, size = np.where(real, each.sum(2), 0.0), np.abs(each).sum(2)
    assert (np.abs(num(dw) - want) <= (width / 64 + 14) * 2.0 ** -24 * size).all()
    rows = np.full((T * k, width), 5.0)
    rows[c["place"][real]] = (num(w)[:, :, None] * num(dy)[:, None, :])[real]
    off = np.abs(num(dys) - rows)
    assert (off <= (torch.finfo(dt).eps / 2 * (1 + 2 ** -7) + 2.0 ** -24) * np.abs(rows)).all()
    # either output by itself, without weights
    one, other = torch.full_like(dys, 5.0), torch.full_like(dw, float("nan"))
    L.stem_experts_combine_backward(ctx, dy, place, one, weights=w)
    L.stem_experts_combine_backward(ctx, dy, place, ys=ys, dweights=other)
    assert torch.equal(one, dys) and torch.equal(other, dw)
    L.stem_experts_combine_backward(ctx, dy, place, one)
    rows[c["place"][real]] = np.broadcast_to(num(dy)[:, None, :], (T, k, width))[real]
    assert np.array_equal(num(one), rows)


def test_gradients_against_differences():
    """The sum of y with a fixed weight for each element, moved by moving one weight or one row."""
    T, k, n, width, step = 6, 2, 3, 40, 2.0 ** -7
    c = rows_case(11, T, k, n, width, "f32")
    ctx, place = make_ctx(T, "f32"), torch.from_numpy(c["place"]).to(DEV)
    dy, ys, w = c["dy"].to(DEV), c["ys"].to(DEV), c["w"].to(DEV)
    dys, dw = torch.zeros_like(ys), torch.zeros_like(w)
    L.stem_experts_combine_backward(ctx, dy, place, dys, ys=ys, weights=w, dweights=dw)

    def value(ys, w):
        y = torch.empty(T, width, device=DEV)
        L.stem_experts_combine(ctx, ys, place, y, weights=w)
        return (y.double() * dy.double()).sum().item()

    scale = (dy.double().abs().sum() * (ys.abs().max() + 1)).item() * (k + 2) * 2.0 ** -24 / step   # of y's roundings, over the step
    for t in range(T):
        for j in range(k):
            up, down = w.clone(), w.clone()
            up[t, j] += step
            down[t, j] -= step
            width_of_step = (up[t, j] - down[t, j]).item()
            assert abs((value(ys, up) - value(ys, down)) / width_of_step - dw[t, j].item()) <= scale
    for r in range(T * k):
        up, down = ys.clone(), ys.clone()
        up[r, 17] += step
        down[r, 17] -= step
        assert abs((value(up, w) - value(down, w)) / (up[r, 17] - down[r, 17]).item() - dys[r, 17].item()) <= scale


def test_dispatch_and_combine_are_each_others_backward_pass():
    T, k, n, width = 500, 2, 7, 96
    c = rows_case(13, T, k, n, width, "f32")
    ctx = make_ctx(T, "f32")
    src, place, _ = sort(ctx, c["e"], n)
    x = c["x"].to(DEV)
    xs, dx = torch.zeros(T * k, width, device=DEV), torch.empty(T, width, device=DEV)
    L.stem_experts_dispatch(ctx, x, src, xs, choices=k)
    g = c["ys"].to(DEV)
    L.stem_experts_combine(ctx, g, place, dx)
    # <dispatch(x), g> = <x, combine(g)>
    a, b = (xs.double() * g.double()).sum().item(), (x.double() * dx.double()).sum().item()
    assert abs(a - b) <= 3 * 2.0 ** -24 * (x.double().abs() * dx.double().abs()).sum().item() + 1e-9 * abs(a)


def test_bad_places_and_sources():
    """Beyond the rows: reported, and nothing outside is touched."""
    T, k, width = 4, 2, 24
    ctx = make_ctx(T, "f32")
    x = torch.randn(T, width, device=DEV)
    src = torch.tensor([0, 1 << 29, -9], dtype=torch.int32, device=DEV)
    xs = torch.zeros(3, width, device=DEV)
    L.stem_experts_dispatch(ctx, x, src, xs, choices=k)
    with pytest.raises(L.StemError):
        L.stem_sync_status(ctx)
    assert torch.equal(xs[0], x[0]) and torch.equal(xs[1], x[3]) and not xs[2].any()
    place = torch.tensor([[0, 1], [2, 1 << 30], [-5, -1], [-1, -1]], dtype=torch.int32, device=DEV)
    y, ys = torch.empty(T, width, device=DEV), torch.randn(3, width, device=DEV)
    L.stem_experts_combine(ctx, ys, place, y)
    with pytest.raises(L.StemError):
        L.stem_sync_status(ctx)
    assert torch.equal(y[0], ys[0] + ys[1]) and torch.equal(y[1], ys[2] + ys[2]) and not y[2:].any()
    dys, dw = torch.zeros(3, width, device=DEV), torch.ones(T, k, device=DEV)
    L.stem_experts_combine_backward(ctx, x, place, dys, ys=ys, dweights=dw)
    with pytest.raises(L.StemError):
        L.stem_sync_status(ctx)
    assert torch.equal(dys, x[[0, 0, 1]]) and not dw[1, 1] and not dw[2:].any()


def test_refusals():
    ctx = make_ctx(8, "f32")
    i32 = dict(dtype=torch.int32, device=DEV)
    e, src, place, off = torch.zeros(4, 2, **i32), torch.zeros(8, **i32), torch.zeros(4, 2, **i32), torch.zeros(4, **i32)

    def refused(status, call, *args, **kw):
        with pytest.raises(L.StemError) as err:
            call(ctx, *args, **kw)
        assert err.value.status == status

    refused(L.STEM_ERR_SHAPE, L.stem_experts_sort, torch.zeros(9, 1, **i32), torch.zeros(9, **i32), torch.zeros(9, 1, **i32), off)     # over max_tokens
    refused(L.STEM_ERR_SHAPE, L.stem_experts_sort, e, src, place, torch.zeros(1, **i32))
    refused(L.STEM_ERR_SHAPE, L.stem_experts_sort, e, src, place, torch.zeros(514, **i32))
    refused(L.STEM_ERR_SHAPE, L.stem_experts_sort, torch.zeros(1, 17, **i32), torch.zeros(17, **i32), torch.zeros(1, 17, **i32), off)
    refused(L.STEM_ERR_INVALID_ARG, L.stem_experts_sort, e, src, e, off)
    refused(L.STEM_ERR_INVALID_ARG, L.stem_experts_sort, e, src, place, src[:4])
    x, xs = torch.zeros(4, 16, device=DEV), torch.zeros(8, 16, device=DEV)
    refused(L.STEM_ERR_INVALID_ARG, L.stem_experts_dispatch, x, src, xs, choices=2, ids=src[:4])
    refused(L.STEM_ERR_INVALID_ARG, L.stem_experts_dispatch, xs[:4], src, xs, choices=2)
    refused(L.STEM_ERR_SHAPE, L.stem_experts_dispatch, x, src, xs, choices=0)
    w = torch.zeros(4, 2, device=DEV)
    refused(L.STEM_ERR_INVALID_ARG, L.stem_experts_combine, xs, place, xs[:4])
    refused(L.STEM_ERR_INVALID_ARG, L.stem_experts_combine_backward, x, place, xs, dweights=w)
    refused(L.STEM_ERR_INVALID_ARG, L.stem_experts_combine_backward, x, place, xs, ys=xs, dweights=w)
    refused(L.STEM_ERR_INVALID_ARG, L.stem_experts_combine, torch.zeros(8 * 16 + 1, device=DEV)[1:].view(8, 16), place, x)
    with pytest.raises(ValueError):
        L.stem_experts_combine(ctx, xs, place, torch.zeros(5, 16, device=DEV))
    with pytest.raises(TypeError):
        L.stem_experts_combine(ctx, xs.bfloat16(), place, x)
