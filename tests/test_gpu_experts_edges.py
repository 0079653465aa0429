"""Tokens to experts and back at calls and widths beside those of test_gpu_experts.py, whose tolerances these are."""
import pytest
import torch

from paper_2601_10639_amd import stemlib as L
from tests.test_gpu_block_bind import count   # noqa: F401 (a fixture)
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
