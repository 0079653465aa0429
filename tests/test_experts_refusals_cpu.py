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


def test_the_work_of_a_sort_grows_with_its_pairs():
    """Counts read by the placing workgroups, for each pair and 512 experts: all segments' by each of a few, one row and the totals by each of many."""
    route = (ctypes.c_int32 * 3)()
    for pairs in [0, 1, 256, 257, 1024, 1025, 4096, 4097, 65536, 65537, 262144, 262145, 524288, 524289, 1 << 20, 1 << 24, 1 << 28, 1 << 30]:
        L.lib().stem_route_experts_sort(pairs, route)
        waves, segments, launches = route
        assert waves * 256 * segments >= pairs and (segments - 1) * waves * 256 < max(pairs, 1)
        assert segments + 1 <= 64 + pairs // 4096 or segments <= 64                      # the rows that a context has
        reads = 0 if launches == 1 else segments * 513 * (segments if launches == 2 else 2)
        assert (launches > 1) == (segments > 1) and reads <= 33 * pairs
