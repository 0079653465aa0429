"""Where the partial sums of a block's gradients lie, asked through the function that stem_create asks; no GPU."""
import ctypes
import random

import pytest

from paper_2601_10639_amd import stemlib as L

SPLITK, HIDDEN, OWN = range(3)


def scratch(d, F, dtype, T):
    size = ctypes.c_int64()
    place = L.lib().stem_route_block_scratch(d, F, dtype, ctypes.c_int64(T), ctypes.byref(size))
    return place, size.value


@pytest.mark.parametrize("d,F,T", [(1024, 4096, 16384), (2048, 8192, 16384), (4096, 14336, 4096), (2048, 8192, 1), (2048, 8192, 300), (16384, 64, 512)])
def test_contexts_of_layers_have_no_scratch_for_the_block_alone(d, F, T):
    place, size = scratch(d, F, L.STEM_BF16, T)
    assert size == min(T, 512 if d <= 4096 else 256) * 3 * d * 4
    assert place == SPLITK
    if F > 64:
        assert scratch(d, F, L.STEM_F32, T) == (HIDDEN, size)


def test_there_is_room_where_they_lie():
    rng = random.Random(1)
    L.lib().stem_route_splitk_bytes.restype = ctypes.c_int64
    for _ in range(5000):
        dtype = rng.choice([L.STEM_F32, L.STEM_BF16])
        m = 64 if dtype == L.STEM_BF16 else 4
        d, F, T = m * int(1 + 400 ** rng.random()), m * int(1 + 400 ** rng.random()), int(40000 ** rng.random()) - (rng.random() < 0.05)
        place, size = scratch(d, F, dtype, T)
        assert size == (min(T, 512 if d <= 4096 else 256) * 3 * d * 4 if d <= 16384 else 0)
        room = {SPLITK: L.lib().stem_route_splitk_bytes(d, F, ctypes.c_int64(T)), HIDDEN: T * F * (2 if dtype == L.STEM_BF16 else 4), OWN: size}[place]
        assert room >= size and (place != SPLITK or dtype == L.STEM_BF16)
