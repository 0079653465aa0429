"""8-bit calls at the edges of their range."""
import pytest
import torch

from paper_2601_10639_amd import stemlib as L
from tests import test_gpu_quant as Q

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
bf = torch.bfloat16


def test_sums_that_32_bits_cannot_hold_are_refused():
    """Rows that are longer than stem_quant_weights takes, with integers from elsewhere."""
    T, d, F = 2, 64, 131136
    ctx = L.stem_create(d, F, 1, L.STEM_BF16, T, reserve=L.STEM_RESERVE_QUANT)

    def weights(N, K):
        return L.StemQuant(torch.zeros(L.stem_quant_bytes(N, K), dtype=torch.int8, device=DEV), torch.ones(N, device=DEV), N, K)

    def status(call, *a):
        with pytest.raises(L.StemError) as e:
            call(*a)
        return e.value.status

    x, y = torch.zeros(T, F, dtype=bf, device=DEV), torch.zeros(T, d, dtype=bf, device=DEV)
    ids, E = torch.zeros(T, dtype=torch.int32, device=DEV), torch.zeros(1, F, dtype=bf, device=DEV)
    assert status(L.stem_quant_linear, ctx, x, weights(d, F), y) == L.STEM_ERR_SHAPE
    assert status(L.stem_quant_ffn_forward, ctx, y, ids, weights(F, d), weights(d, F), E, y) == L.STEM_ERR_SHAPE
    w = L.stem_quant_weights(ctx, torch.ones(1, 131072, dtype=bf, device=DEV))
    z = torch.zeros(T, 1, dtype=bf, device=DEV)
    L.stem_quant_linear(ctx, torch.ones(T, 131072, dtype=bf, device=DEV), w, z)
    assert (z == 131072).all()      # 127 * 127 * 131072 = 2.114e9


@pytest.mark.parametrize("T,d,F", [(4096, 64, 8192), (2100, 512, 8192), (4096, 1024, 4096), (4096, 1024, 8192)])
def test_tokens_are_those_of_smaller_calls(T, d, F):
    """Integers, maxima and sums of integers: how many tokens a call has, and so which tile, changes no bit.  Several workgroups to a compute unit."""
    V = 50
    ctx = L.stem_create(d, F, V, L.STEM_BF16, T, reserve=L.STEM_RESERVE_QUANT)

    def draw(seed, *shape, std=1.0):
        return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * std).to(bf).to(DEV)

    x, E = draw(1, T, d), draw(4, V, F)
    g, w = L.stem_quant_weights(ctx, draw(2, F, d, std=1.5 * d ** -0.5)), L.stem_quant_weights(ctx, draw(3, d, F, std=F ** -0.5))
    ids = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(5), dtype=torch.int32).to(DEV)
    want = torch.empty_like(x)
    for t in range(0, T, 600):
        rows, y = x[t:t + 600].clone(), torch.empty_like(x[t:t + 600])
        L.stem_quant_ffn_forward(ctx, rows, ids[t:t + 600].clone(), g, w, E, y)
        want[t:t + 600] = y
    for _ in range(3):
        y = torch.empty_like(x)
        L.stem_quant_ffn_forward(ctx, x, ids, g, w, E, y)
        assert torch.equal(y, want)


# The large tiles: (tile, T, N, K).  Sides that end inside a tile, widths of whole 16 bytes and odd ones, every remainder of K tiles in the rings
# (five of 128 values and three of 64), and K long enough that the XCDs start apart.
TILES = [((256, 256), 4100, 2504, 128), ((256, 256), 4099, 2501, 300), ((256, 256), 3900, 2320, 640), ((256, 256), 4200, 2410, 700), ((256, 256), 4060, 2560, 2048),
         ((256, 256), 3850, 2305, 2300), ((128, 256), 4100, 1104, 128), ((128, 256), 4099, 1101, 64), ((128, 256), 4100, 1320, 192), ((128, 256), 4033, 1111, 380),
         ((128, 256), 4000, 1160, 2048), ((128, 128), 1500, 2047, 640), ((128, 128), 1450, 2056, 2048), ((128, 128), 2051, 1001, 129)]
# The layer's gate product on 128 x 256: d_ff that ends 64, 128 and 192 columns into a tile; and more tokens than have their hidden values at a time
PAIR = [(2100, 64, 2112), (2100, 192, 2240), (2070, 128, 2176), (2050, 320, 2304)]
CHUNKS = (4096 + 33, 64, 8192)
# Up to 8 tokens: x and hidden values quantised in place or by a kernel before the product, each by itself, and hidden values in slices of K
FEW = [(5, 3200, 8192), (8, 2112, 5632), (8, 1024, 4096), (6, 2048, 8192), (7, 192, 576), (1, 2048, 8192)]


@pytest.mark.parametrize("tile,T,N,K", TILES)
def test_large_tiles(tile, T, N, K):
    ctx = Q.make_ctx(T, 2304)
    Q.check_linear(ctx, T, N, K)
    Q.check_linear(ctx, T, N, K, residual=True, seed=30)


@pytest.mark.parametrize("T,d,F", PAIR + FEW + [CHUNKS])
@pytest.mark.parametrize("norm_kind", [None, 1])
def test_layer(T, d, F, norm_kind):
    Q.test_ffn(T, d, F, norm_kind)


@pytest.mark.parametrize("T,d,F", [PAIR[0], PAIR[1], CHUNKS])
def test_ids_outside_the_table(T, d, F):
    """In the large tile, and in a later turn of hidden values."""
    V = 10
    ctx = Q.make_ctx(T, d, F, V)
    x, E = Q.draw(1, T, d), Q.draw(4, V, F)
    g, w = L.stem_quant_weights(ctx, Q.draw(2, F, d, std=0.1)), L.stem_quant_weights(ctx, Q.draw(3, d, F, std=0.02))
    ids = (torch.arange(T, dtype=torch.int32) % (V - 1)).to(DEV)      # (the last row is nobody's own)
    clamped = ids.clone()
    clamped[[0, 130, T - 2]], clamped[T - 1] = 0, V - 1
    ids[[0, 130, T - 2]], ids[T - 1] = -3, V + 5
    y, z = torch.empty_like(x), torch.empty_like(x)
    L.stem_quant_ffn_forward(ctx, x, clamped, g, w, E, y)
    L.stem_sync_status(ctx)
    L.stem_quant_ffn_forward(ctx, x, ids, g, w, E, z)
    with pytest.raises(L.StemError) as e:
        L.stem_sync_status(ctx)
    assert e.value.status == L.STEM_ERR_ID_RANGE
    assert torch.equal(y, z)


@pytest.mark.parametrize("T,d,F", [PAIR[0], PAIR[1], CHUNKS, FEW[0], FEW[1]])
def test_what_is_no_number_spoils_its_tokens_only(T, d, F):
    V = 20
    ctx = Q.make_ctx(T, d, F, V)
    x, E = Q.draw(1, T, d), Q.draw(4, V, F)
    g, w = L.stem_quant_weights(ctx, Q.draw(2, F, d, std=d ** -0.5)), L.stem_quant_weights(ctx, Q.draw(3, d, F, std=F ** -0.5))
    ids = (torch.arange(T, dtype=torch.int32) % V).to(DEV)
    y = torch.empty_like(x)
    L.stem_quant_ffn_forward(ctx, x, ids, g, w, E, y)
    E[3, 0], E[5, F - 1], E[7, F // 2] = float("inf"), float("nan"), float("-inf")
    x[T - 1, d - 1] = float("nan")
    z = torch.empty_like(x)
    L.stem_quant_ffn_forward(ctx, x, ids, g, w, E, z)
    bad = (ids == 3) | (ids == 5) | (ids == 7)
    bad[T - 1] = True
    assert torch.isnan(z[bad]).all() and torch.equal(z[~bad], y[~bad])


@pytest.mark.parametrize("rows,K", [(2049, 700), (2050, 2500), (1030, 5000), (1024, 8192), (2079, 4096)])
def test_many_long_rows(rows, K):
    """As weights, where the integers are compared one by one, and as tokens behind a norm."""
    Q.test_weights(rows, K)
    ctx = Q.make_ctx(rows, 8192)
    Q.check_linear(ctx, rows, 40, K, 2)
    Q.check_linear(ctx, rows, 33, K, 1, residual=True)
