"""What the calls that bring tokens to experts and back refuse before they look at a device."""
import ctypes

import pytest
import torch

from paper_2601_10639_amd import stemlib as L


class Fake:
    handle = ctypes.c_void_p(None)
    torch_dtype = torch.float32
    d_model, d_ff = 64, 64


def test_a_gradient_of_weights_needs_rows():
    dy, place, dw = torch.zeros(4, 16), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    for width in (16, 0):
        with pytest.raises(L.StemError) as err:
            L.stem_experts_combine_backward(Fake(), dy[:, :width], place, dweights=dw)
        assert err.value.status == L.STEM_ERR_INVALID_ARG and "needs ys" in str(err.value)
