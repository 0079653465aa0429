"""The shapes of the grouped products' and the layer's GPU tests reach the tiles that they are there for."""
import pytest

from tests import test_gpu_qfloat_ways as G
from tests.test_qfloat_reach_cpu import HIDDEN, tiles

TILES = {"ring": (256, 256), "pair": (128, 256), "128x128": (128, 128), "128x64": (128, 64)}
GATES = {"64x128": (64, 128), "128x128": (128, 128), "pair": (128, 256)}


@pytest.mark.parametrize("name,shape", [(n, s) for n, shapes in G.TILES.items() for s in shapes])
def test_tiles(name, shape):
    T, N, K, groups = shape
    assert groups > 1 and tiles(T, N, K, groups=groups) == (*TILES[name], 1) and T > 8


@pytest.mark.parametrize("name,shape", [(n, s) for n, shapes in G.GATES.items() for s in shapes])
def test_gates(name, shape):
    T, d, F, groups = shape
    few = T <= (16 if groups == 1 else 8)
    assert few == (name == "few") and (few or tiles(T, F, d, HIDDEN, groups)[:2] == GATES[name])


def test_a_step_is_found_where_a_value_is_between_two():
    import numpy as np
    h = np.full((1, 128), 1.0)
    h[0, 0], h[0, 1], h[0, 2] = 448.0, 1.0625, 0.0            # the middle of 1 and 1.125
    step = G.ends(h, np.abs(h) * 1e-6)
    assert step[0, 1] == 0.125 and not step[0, 2:].any()
    assert step[0, 0] == 0.0                                  # 448 + a little has the larger exponent, and is 448 there too
