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
