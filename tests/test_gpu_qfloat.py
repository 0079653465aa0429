"""Products in 8-bit floating point on the GPU, against the oracle in 64 bits.

Tolerances.  Without a norm the 8-bit values are the oracle's exactly and so is every product.  The matrix instruction adds eight products at a time, each cut towards
zero at 2^-13 of a power of two that is at most the largest product: an error in [0, L] of a product's sign, L <= 2^-13 max|a| max|b|, so at most
L^2 / 3 of variance each, and 6 sqrt(K / 3) L is six standard deviations of their sum.  Its fp32 accumulator adds 2^-24 of the sum of magnitudes for each 8.  An output in bf16 is off by half
a step besides, 2^-8 of itself.  A weight gradient's products are exact too, and its sums fp32 of unknown order: at most 16 additions inside an
instruction and one for each, a unit of the last place each: (T / 16 + 16) 2^-23 of the sum of magnitudes, and the K slices' 8.
With a norm, whose values are off by some 4e-7, a value next to the middle between two of the format's may go to the other one: one in 10^5.  Up to two in
a row are allowed, each of which moves an output by an eighth of the value at most, times the weight.
The layer: hidden values are off by some 1.5e-5, and one in 5000 goes to its neighbour, an eighth of itself at most: of 1536 in a row less than one, and eight in a row
are allowed.  The norm of the whole output's error is within bf16's rounding, and sqrt(1 / 5000) / 8 of the norm for the neighbours."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as B
from oracle import qfloat_oracle as Q
from paper_2601_10639_amd import stemlib as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
KINDS = {1: "rms", 2: "layer"}


def make_ctx(T, d, F=None, V=100, groups=1, backward=False):
    ctx = L.stem_create(d, F or d, V, L.STEM_BF16, T)
    L.stem_qfloat_reserve(ctx, groups, backward)
    return ctx


def wide(*sizes):
    return -(-max(sizes) // 64) * 64


def draw(seed, *shape, std=1.0, mean=0.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * std + mean).to(bf).to(DEV)


def num(t):
    return t.double().cpu().numpy()


def offsets_of(seed, T, groups, lo=0, hi=None):
    """Uneven groups, some without a row; rows outside lo .. hi belong to none."""
    hi = T if hi is None else hi
    rng = np.random.default_rng(seed)
    cuts = np.sort(rng.integers(lo, hi + 1, groups - 1)) if groups > 1 else np.array([], int)
    if groups > 3:
        cuts[1] = cuts[0]
    return np.concatenate([[lo], cuts, [hi]]).astype(np.int32)


def dev(offsets):
    return None if offsets is None else torch.from_numpy(np.asarray(offsets, np.int32)).to(DEV)


def values_of(form, rows, K):
    """The [rows, K] values of an 8-bit form, out of the blocks they lie in."""
    R, P = -(-rows // 128) * 128, -(-K // 128) * 128
    raw = form.cpu()
    q = raw[:R * P].view(torch.float8_e4m3fn).float().numpy().reshape(R // 32, P // 32, 2, 32, 16).transpose(0, 3, 1, 2, 4).reshape(R, P)
    s = raw[R * P:].numpy().reshape(R // 128, P // 128, 32, 4).transpose(0, 3, 2, 1).reshape(R, P // 128)
    return q.astype(np.float64) * np.ldexp(1.0, s.astype(int) - 127).repeat(128, 1)


@pytest.mark.parametrize("N,K", [(1, 1), (3, 17), (128, 128), (129, 127), (100, 1999), (256, 384), (31, 4104), (500, 130)])
@pytest.mark.parametrize("groups", [1, 3])
def test_weights(N, K, groups):
    W = draw(1, groups, N, K, std=0.02)
    W[0, 0] = 0
    if N > 2 and K > 16:
        W[0, 2, K // 2], W[0, 1, 0], W[0, 1, 16] = float("inf"), float("nan"), -float("inf")
        W[-1, 0, 1], W[-1, 2, 3] = 448.0, 450.0          # (a block whose largest value is just above a scale's)
    w = L.stem_qfloat_weights(make_ctx(1, 64), W, backward=True)
    size = L.stem_qfloat_bytes(N, K)
    for g in range(groups):
        want = Q.squares(num(W[g]))
        for form, rows, cols, v in ((w.q, N, K, want), (w.qt, K, N, want.T)):
            got = values_of(form[g * size:(g + 1) * size], rows, cols)
            assert np.array_equal(got[:rows, :cols], v, equal_nan=True)
            assert (got[:, cols:] == 0).all() and (got[rows:] == 0).all()


def test_every_bf16_value():
    """All finite magnitudes, each with its neighbours of a similar size in a block, and each by itself as the largest."""
    bits = torch.arange(0, 0x7f80, dtype=torch.int32).to(torch.int16).view(bf)
    rows = bits[: 255 * 128].reshape(255, 128)
    by_itself = torch.zeros(255 * 16, 128, dtype=bf)
    by_itself[:, 77] = -rows.reshape(-1)[::8]
    x = torch.cat([rows, by_itself]).to(DEV)
    w = L.stem_qfloat_weights(make_ctx(1, 64), torch.cat([x, x.flip(1)], 1)[:128])     # squares of mixed sizes too
    assert np.array_equal(values_of(w.q, 128, 256), Q.squares(num(torch.cat([x, x.flip(1)], 1)[:128])))
    # rows, through a product with the identity
    eye = torch.eye(128, dtype=bf, device=DEV)
    ctx, y = make_ctx(len(x), 128), torch.empty(len(x), 128, dtype=bf, device=DEV)
    L.stem_qfloat_linear(ctx, x, L.stem_qfloat_weights(ctx, eye), y)
    # (the largest magnitudes go up to 2^128, which an output in bf16 has as an infinity; all others are values of bf16)
    want = num(torch.from_numpy(Q.blocks(num(x), 1)).to(bf))
    ok = np.abs(want) >= 2.0 ** -110                     # (a product's scale may not reach below)
    assert np.array_equal(num(y)[ok], want[ok])


SHAPES = [(1, 1, 1), (1, 64, 128), (2, 130, 65), (16, 256, 384), (17, 100, 1999), (31, 33, 129), (64, 520, 1000), (65, 128, 128), (100, 1001, 700), (128, 256, 512),
          (129, 129, 129), (300, 64, 4096), (513, 300, 513), (1000, 200, 72), (260, 2048, 256)]
GROUPED = [(1, 3, 128, 128), (5, 2, 40, 72), (64, 4, 256, 256), (200, 7, 130, 300), (777, 5, 512, 384), (1000, 70, 64, 200), (300, 512, 32, 64), (2000, 3, 300, 129)]


def cut(a, b, size):
    """Of sums of Q's products of rows of a with rows of b."""
    K = a.shape[1]
    top = lambda v: np.where(np.isfinite(v), np.abs(v), 0.0).max(1)
    return 6 * np.sqrt(K / 3) * 2.0 ** -13 * top(a)[:, None] * top(b).max() + (K / 8 + 8) * 2.0 ** -24 * size


def test_sums_are_as_near_as_is_said():
    """Whatever the length: 1.5e-5 of the norm (and what bf16 rounds: the outputs here are compared with what they round to)."""
    for K in (128, 2048, 8192):
        ctx = make_ctx(256, 64, K)
        x, W = draw(1, 256, K), draw(2, 256, K)
        y = torch.empty(256, 256, dtype=bf, device=DEV)
        L.stem_qfloat_linear(ctx, x, L.stem_qfloat_weights(ctx, W), y)
        want, _ = Q.linear(num(x), num(W)[None])
        other = (num(y) != num(torch.from_numpy(want).to(bf))).mean()
        # a result whose error is 1.5e-5 sqrt(K) s rounds otherwise where the middle between two steps (2^-7 apart, relative) is as near: 2 E|error| / step
        assert other <= 4 * 1.5e-5 / 2.0 ** -8


def bound(K):
    return (K / 16 + 24) * 2.0 ** -23


def check_linear(ctx, T, N, K, groups=1, offsets=None, norm_kind=None, residual=False, seed=3):
    x, W = draw(seed, T, K) * draw(seed + 1, T, 1, std=0.5, mean=2.0), draw(seed + 2, groups, N, K, std=0.05)
    res = draw(seed + 3, T, N) if residual else None
    w = L.stem_qfloat_weights(ctx, W)
    y = torch.full((T, N), 7.0, dtype=bf, device=DEV)
    v, norm, slack = num(x), None, 0.0
    if norm_kind:
        g = draw(seed + 4, K, std=0.2, mean=1.0)
        norm = L.stem_norm(norm_kind, 1e-5, g)
        v = B.norm(x.float().cpu().numpy(), KINDS[norm_kind], 1e-5)[0] * num(g)
        slack = 2 / 8 * np.abs(v).max(1)[:, None] * np.abs(num(W)).max()
    L.stem_qfloat_linear(ctx, x, w, y, residual=res, norm=norm, offsets=dev(offsets))
    want, size = Q.linear(v, num(W), offsets)
    none = np.isnan(want)
    want = want + (num(res) if residual else 0.0)
    off = np.abs(num(y) - want)
    assert (none | (off <= np.abs(want) * 2.0 ** -8 * (1 + 2 ** -7) + slack + cut(v, num(W).reshape(-1, K), size) + 2.0 ** -22 * np.abs(want))).all(), np.nanmax(off)
    assert (num(y)[none] == 7.0).all()
    if residual and offsets is None:   # in place
        L.stem_qfloat_linear(ctx, x, w, res, residual=res, norm=norm)
        assert torch.equal(res, y)
    return y


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("T,N,K", SHAPES)
def test_linear(T, N, K, residual):
    check_linear(make_ctx(T, 64, wide(K)), T, N, K, residual=residual)


@pytest.mark.parametrize("kind", [L.STEM_NORM_RMS, L.STEM_NORM_LAYER])
@pytest.mark.parametrize("T,N,K", [(1, 128, 1024), (9, 100, 1999), (40, 64, 8192), (70, 300, 129), (3, 64, 8256), (2100, 40, 130)])
def test_linear_behind_a_norm(T, N, K, kind):
    check_linear(make_ctx(T, 64, wide(K)), T, N, K, norm_kind=kind, residual=True)


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("T,groups,N,K", GROUPED)
def test_linear_by_groups(T, groups, N, K, residual):
    ctx = make_ctx(T, 64, wide(K), groups=groups)
    check_linear(ctx, T, N, K, groups, offsets_of(T, T, groups), residual=residual)
    check_linear(ctx, T, N, K, groups, offsets_of(T + 1, T, groups, T // 7, T - T // 5), norm_kind=L.STEM_NORM_RMS)   # rows in front of and behind the groups


@pytest.mark.parametrize("T,groups,N,K", [(4500, 1, 2100, 200), (4500, 1, 2104, 2048), (2100, 1, 4097, 300), (9000, 3, 3001, 130), (6000, 2, 2304, 2200)])
def test_linear_of_many_rows(T, groups, N, K):
    """Large tiles: of odd columns, K tiles in all of the ring's places, and groups that end inside a tile."""
    ctx = make_ctx(T, 64, wide(K), groups=groups)
    check_linear(ctx, T, N, K, groups, None if groups == 1 else offsets_of(T, T, groups, 5, T - 77), residual=True)


@pytest.mark.parametrize("T,groups,d,F", [(4200, 1, 192, 2240), (4400, 3, 128, 3264)])
def test_ffn_of_many_rows(T, groups, d, F):
    check_ffn(make_ctx(T, d, F, groups=groups), T, d, F, groups=groups, offsets=None if groups == 1 else offsets_of(3, T, groups, 9, T - 70))


def test_offsets_that_are_none():
    """Descending, negative, beyond the rows: as the oracle takes them, and nothing outside is touched."""
    T, N, K = 300, 130, 200
    ctx = make_ctx(T, 64, 256, groups=5, backward=True)
    for offsets in ([0, 200, 100, 250, -3, 300], [-5, 50, 1 << 30, 20, 60, 70], [300, 0, 0, 0, 0, 0], [1 << 30, 0, -1, 5, 6, 9], [-(1 << 31), 10, 10, 10, 10, 10],
                    [0, 300, 0, 300, 0, 300]):
        check_linear(ctx, T, N, K, 5, np.array(offsets, np.int32))
        check_backward(ctx, T, N, K, 5, np.array(offsets, np.int32))


def check_backward(ctx, T, N, K, groups=1, offsets=None, seed=5):
    dy, x, W = draw(seed, T, N, std=1e-3), draw(seed + 1, T, K), draw(seed + 2, groups, N, K, std=0.05)
    w = L.stem_qfloat_weights(ctx, W, backward=True)
    dx, dW = torch.full((T, K), 7.0, dtype=bf, device=DEV), torch.full((groups, N, K), float("nan"), device=DEV)
    o = dev(offsets)
    L.stem_qfloat_linear_backward(ctx, dy, x, w, dx, dW, offsets=o)
    (want, size), (want_w, size_w) = Q.linear_backward(num(dy), num(x), num(W), offsets)
    none = np.isnan(want)
    assert (none | (np.abs(num(dx) - want) <= np.abs(want) * 2.0 ** -8 * (1 + 2 ** -7) + cut(num(dy), np.swapaxes(num(W), 1, 2).reshape(-1, N), size))).all()
    assert (num(dx)[none] == 7.0).all()
    assert (np.abs(num(dW) - want_w) <= bound(T) * size_w).all()
    # each by itself, added to what is there, and dx over dy
    one, more = torch.full_like(dx, 7.0), torch.ones_like(dW)
    L.stem_qfloat_linear_backward(ctx, dy, None, w, one, offsets=o)
    assert torch.equal(one, dx)
    L.stem_qfloat_linear_backward(ctx, dy, x, w, dW=more, offsets=o, accumulate=True)
    assert torch.equal(more, dW + 1.0)
    L.stem_qfloat_linear_backward(ctx, dy, x, w, x, dW, offsets=o)
    assert torch.equal(x[torch.from_numpy(~none).to(DEV)], dx[torch.from_numpy(~none).to(DEV)]) and torch.equal(more, dW + 1.0)




@pytest.mark.parametrize("T,N,K", SHAPES)
def test_backward(T, N, K):
    check_backward(make_ctx(T, 64, wide(K, N), backward=True), T, N, K)


@pytest.mark.parametrize("T,groups,N,K", GROUPED)
def test_backward_by_groups(T, groups, N, K):
    ctx = make_ctx(T, 64, wide(K, N), groups=groups, backward=True)
    check_backward(ctx, T, N, K, groups, offsets_of(T, T, groups))
    check_backward(ctx, T, N, K, groups, offsets_of(T + 1, T, groups, T // 7, T - T // 5))


def test_backward_against_differences():
    """Weights and inputs whose moves are values of the format: the product is linear in them."""
    T, N, K = 130, 40, 136
    ctx = make_ctx(T, 64, 192, backward=True)
    pick = lambda seed, *s: torch.randint(-4, 5, s, generator=torch.Generator().manual_seed(seed)).to(bf).to(DEV)
    x, W, dy = pick(1, T, K), pick(2, N, K), pick(3, T, N)
    w = L.stem_qfloat_weights(ctx, W, backward=True)
    dx, dW = torch.empty_like(x), torch.empty(N, K, device=DEV)
    L.stem_qfloat_linear_backward(ctx, dy, x, w, dx, dW)

    def value(x, W):
        y = torch.empty(T, N, dtype=bf, device=DEV)
        L.stem_qfloat_linear(ctx, x, L.stem_qfloat_weights(ctx, W), y)
        return num(y) * num(dy)

    small, s = 2.0 ** -7, (np.abs(num(dy)).max(), 2 * 5 * 4 * K)     # bf16's rounding of y, in both
    for t, k in ((0, 0), (129, 135), (64, 100)):
        up, down = x.clone(), x.clone()
        up[t, k] += 1
        down[t, k] -= 1
        diff = (value(up, W) - value(down, W))[t].sum() / 2
        assert abs(diff - num(dx)[t, k]) <= small * (s[1] * s[0] * N + abs(num(dx)[t, k]))
    for n, k in ((0, 0), (39, 135), (20, 128)):
        up, down = W.clone(), W.clone()
        up[n, k] += 1
        down[n, k] -= 1
        diff = (value(x, up) - value(x, down))[:, n].sum() / 2
        assert abs(diff - num(dW)[n, k]) <= small * s[1] * s[0] * T


def check_ffn(ctx, T, d, F, V=60, groups=1, offsets=None, kind=L.STEM_NORM_RMS, residual=True, seed=9):
    x, ids = draw(seed, T, d), torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(seed)).to(i32).to(DEV)
    Wg, Wd, E, g = draw(seed + 1, groups, F, d, std=0.04), draw(seed + 2, groups, d, F, std=0.04), draw(seed + 3, V, F), draw(seed + 4, d, std=0.2, mean=1.0)
    gate, down = L.stem_qfloat_weights(ctx, Wg), L.stem_qfloat_weights(ctx, Wd)
    norm = L.stem_norm(kind, 1e-5, g) if kind else None
    y = torch.full((T, d), 7.0, dtype=bf, device=DEV)
    L.stem_qfloat_ffn_forward(ctx, x, ids, gate, down, E, y, residual=x if residual else None, norm=norm, offsets=dev(offsets))
    n = B.norm(x.float().cpu().numpy(), KINDS[kind], 1e-5)[0] * num(g) if kind else num(x)
    args = (ids.cpu().numpy(), num(Wg), num(Wd), num(E), offsets)
    want = Q.ffn(n, *args)
    none = np.isnan(want)
    h = Q.hidden(n, args[0], args[1], args[3], offsets)
    want = want + (num(x) if residual else 0.0)
    off = np.where(none, 0.0, num(y) - want)
    real = np.where(none, 0.0, want)
    assert np.linalg.norm(off) <= (2.0 ** -8 + 5000 ** -0.5 / 8) * np.linalg.norm(real)
    slack = 8 / 8 * np.abs(h).max(1)[:, None] * np.abs(num(Wd)).max()
    assert (none | (np.abs(off) <= 2.0 ** -7 * np.abs(want) + slack)).all()
    assert (num(y)[none] == 7.0).all()
    if residual:   # in place
        L.stem_qfloat_ffn_forward(ctx, x, ids, gate, down, E, x, residual=x, norm=norm, offsets=dev(offsets))
        assert torch.equal(x[torch.from_numpy(~none).to(DEV)], y[torch.from_numpy(~none).to(DEV)])


@pytest.mark.parametrize("T,d,F", [(1, 64, 64), (1, 256, 1024), (2, 128, 192), (7, 64, 320), (16, 512, 1536), (17, 192, 448), (33, 256, 256), (65, 128, 704), (130, 320, 576),
                                   (300, 256, 1024), (1030, 128, 320)])
def test_ffn(T, d, F):
    ctx = make_ctx(T, d, F)
    check_ffn(ctx, T, d, F)
    check_ffn(ctx, T, d, F, kind=0, residual=False)
    check_ffn(ctx, T, d, F, kind=L.STEM_NORM_LAYER)


@pytest.mark.parametrize("T,groups,d,F", [(1, 2, 64, 128), (20, 3, 128, 320), (150, 6, 192, 448), (700, 4, 256, 512), (500, 40, 64, 192)])
def test_ffn_by_groups(T, groups, d, F):
    ctx = make_ctx(T, d, F, groups=groups)
    check_ffn(ctx, T, d, F, groups=groups, offsets=offsets_of(T, T, groups))
    check_ffn(ctx, T, d, F, groups=groups, offsets=offsets_of(T + 1, T, groups, T // 7, T - T // 5))


@pytest.mark.parametrize("T", [3, 40, 200])
def test_numbers_that_are_none(T):
    """They reach what depends on them and nothing else."""
    N, K = 150, 300
    ctx = make_ctx(T, 64, 320, backward=True)
    x, W, dy = draw(1, T, K), draw(2, N, K, std=0.05), draw(3, T, N)
    y, clean = torch.empty(T, N, dtype=bf, device=DEV), torch.empty(T, N, dtype=bf, device=DEV)
    w = L.stem_qfloat_weights(ctx, W, backward=True)
    L.stem_qfloat_linear(ctx, x, w, clean)
    bad = x.clone()
    bad[1, 5], bad[T - 1, K - 1] = float("inf"), float("nan")
    L.stem_qfloat_linear(ctx, bad, w, y)
    rows = torch.tensor([t in (1, T - 1) for t in range(T)], device=DEV)
    assert y[rows].isnan().all() and torch.equal(y[~rows], clean[~rows])
    W2 = W.clone()
    W2[7, 130] = -float("inf")
    L.stem_qfloat_linear(ctx, x, L.stem_qfloat_weights(ctx, W2), y)
    assert y[:, 7].isnan().all() and not y[:, :7].isnan().any() and not y[:, 8:].isnan().any()
    dx, dW, dx2, dW2 = (torch.empty(s, dtype=t, device=DEV) for s, t in (((T, K), bf), ((N, K), f32)) * 2)
    L.stem_qfloat_linear_backward(ctx, dy, x, w, dx, dW)
    L.stem_qfloat_linear_backward(ctx, dy, bad, w, dx2, dW2)
    assert torch.equal(dx, dx2) and not dW2[:, 5].isfinite().any() and dW2[:, K - 1].isnan().all() and torch.equal(dW[:, 6:K - 1], dW2[:, 6:K - 1])


def test_norm_and_hidden_numbers_that_are_none():
    T, d, F, V = 70, 128, 320, 40
    ctx = make_ctx(T, d, F)
    x, ids, E = draw(1, T, d), torch.arange(T, dtype=i32, device=DEV) % V, draw(2, V, F)
    gate, down = L.stem_qfloat_weights(ctx, draw(3, F, d, std=0.05)), L.stem_qfloat_weights(ctx, draw(4, d, F, std=0.05))
    norm = L.stem_norm(L.STEM_NORM_RMS, 1e-5, draw(5, d, mean=1.0, std=0.1))
    for n in (1, 16, T):
        clean, y = torch.empty(n, d, dtype=bf, device=DEV), torch.empty(n, d, dtype=bf, device=DEV)
        L.stem_qfloat_ffn_forward(ctx, x[:n], ids[:n], gate, down, E, clean, norm=norm)
        E2, x2 = E.clone(), x.clone()
        E2[0, 300], E2[0, 0] = float("inf"), float("nan")
        if n > 3:
            x2[3, 100] = float("inf")
        L.stem_qfloat_ffn_forward(ctx, x2[:n], ids[:n], gate, down, E2, y, norm=norm)
        bad = torch.tensor([t % V == 0 or t == 3 for t in range(n)], device=DEV)
        assert y[bad].isnan().all() and torch.equal(y[~bad], clean[~bad])


def test_ids_out_of_range_are_reported():
    ctx = make_ctx(3, 64, 128)
    x, E = draw(1, 3, 64), draw(2, 5, 128)
    gate, down = L.stem_qfloat_weights(ctx, draw(3, 128, 64)), L.stem_qfloat_weights(ctx, draw(4, 64, 128))
    y, want = torch.empty_like(x), torch.empty_like(x)
    L.stem_qfloat_ffn_forward(ctx, x, torch.tensor([0, 4, 3], dtype=i32, device=DEV), gate, down, E, want)
    L.stem_qfloat_ffn_forward(ctx, x, torch.tensor([-7, 5, 3], dtype=i32, device=DEV), gate, down, E, y)
    with pytest.raises(L.StemError) as err:
        L.stem_sync_status(ctx)
    assert err.value.status == L.STEM_ERR_ID_RANGE and torch.equal(y, want)


def test_no_tokens():
    ctx = make_ctx(8, 64, 128, groups=2, backward=True)
    W = L.stem_qfloat_weights(ctx, draw(1, 2, 128, 64), backward=True)
    o, none = torch.zeros(3, dtype=i32, device=DEV), torch.empty(0, 64, dtype=bf, device=DEV)
    none_y = torch.empty(0, 128, dtype=bf, device=DEV)
    dW = torch.ones(2, 128, 64, device=DEV)
    L.stem_qfloat_linear(ctx, none, W, none_y, offsets=o)
    L.stem_qfloat_linear_backward(ctx, none_y, none, W, none.clone(), dW, offsets=o, accumulate=True)
    assert (dW == 1).all()
    L.stem_qfloat_linear_backward(ctx, none_y, none, W, none.clone(), dW, offsets=o)
    assert not dW.any()


def test_refusals():
    ctx = make_ctx(8, 64, 128, groups=2)
    plain = L.stem_create(64, 128, 10, L.STEM_BF16, 8)
    single = L.stem_create(64, 128, 10, L.STEM_F32, 8)
    W, x, y = draw(1, 2, 128, 64), draw(2, 8, 64), torch.empty(8, 128, dtype=bf, device=DEV)
    w = L.stem_qfloat_weights(ctx, W)
    o = torch.tensor([0, 4, 8], dtype=i32, device=DEV)

    def refused(status, call, *args, **kw):
        with pytest.raises(L.StemError) as err:
            call(*args, **kw)
        assert err.value.status == status, err.value

    refused(L.STEM_ERR_UNSUPPORTED, L.stem_qfloat_reserve, single)
    refused(L.STEM_ERR_SHAPE, L.stem_qfloat_reserve, plain, 513)
    refused(L.STEM_ERR_SHAPE, L.stem_qfloat_reserve, plain, 0)
    refused(L.STEM_ERR_INVALID_ARG, L.stem_qfloat_reserve, ctx, 3)          # more groups than before
    refused(L.STEM_ERR_WORKSPACE, L.stem_qfloat_linear, plain, x, w, y, offsets=o)
    refused(L.STEM_ERR_INVALID_ARG, L.stem_qfloat_linear, ctx, x, w, y)     # two groups, no offsets
    refused(L.STEM_ERR_WORKSPACE, L.stem_qfloat_linear_backward, ctx, y, x, w, x, offsets=o)
    refused(L.STEM_ERR_SHAPE, L.stem_qfloat_linear, ctx, draw(1, 9, 64), w, torch.empty(9, 128, dtype=bf, device=DEV), offsets=o)
    L.stem_qfloat_reserve(ctx, 2, True)
    refused(L.STEM_ERR_INVALID_ARG, L.stem_qfloat_linear_backward, ctx, y, x, w, x, offsets=o)   # no transposed weights
    big = L.stem_qfloat_weights(ctx, draw(3, 128, 200))
    refused(L.STEM_ERR_SHAPE, L.stem_qfloat_linear, ctx, draw(4, 8, 200), big, y)               # K over the context's widths
    raw = torch.zeros(8 * 128 + 8, dtype=bf, device=DEV)
    refused(L.STEM_ERR_INVALID_ARG, L.stem_qfloat_linear, ctx, x, w, raw[4:4 + 1024].view(8, 128), offsets=o)
    refused(L.STEM_ERR_INVALID_ARG, L.stem_qfloat_linear, ctx, x, w, raw[:1024].view(8, 128), residual=raw[8:].view(8, 128), offsets=o)
    refused(L.STEM_ERR_INVALID_ARG, L.stem_qfloat_linear, ctx, x, w, y, offsets=y.view(-1).view(i32)[:3])
    with pytest.raises(ValueError):
        L.stem_qfloat_linear(ctx, x, w, y, offsets=o[:2])
    with pytest.raises(ValueError):
        L.stem_qfloat_linear(ctx, x, L.StemQfloat(w.q[:-1], None, 2, 128, 64), y, offsets=o)
    with pytest.raises(TypeError):
        L.stem_qfloat_linear(ctx, x.float(), w, y, offsets=o)
