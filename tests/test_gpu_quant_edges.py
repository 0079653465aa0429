"""8-bit calls at the edges of their range."""
import pytest
import torch

from paper_2601_10639_amd import stemlib as L

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
