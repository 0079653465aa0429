"""The shapes of tests/test_gpu_quant_edges.py reach the kernels that they are there for; no GPU."""
import pytest

from tests import test_gpu_quant_edges as E
from tests.test_quant_routes_cpu import ceil, route

WS = 256 * 128 * 64 * 4


@pytest.mark.parametrize("tile,T,N,K", E.TILES)
def test_tiles(tile, T, N, K):
    assert route(T, N, ceil(K, 128) * 128, False, WS)[:2] == tile


def test_every_remainder_of_the_rings():
    for tile, ring, k in (((256, 256), 5, 128), ((128, 256), 3, 64)):
        assert {ceil(K, 128) * (128 // k) % ring for t, _, _, K in E.TILES if t == tile} >= ({0, 1, 3} if ring == 5 else {0, 1, 2})


@pytest.mark.parametrize("T,d,F", E.PAIR + [E.CHUNKS])
def test_gate_products(T, d, F):
    chunk = max(256, (128 << 20) // (4 * ceil(F, 128) * 128) // 256 * 256)
    assert route(min(T, chunk), F, ceil(d, 128) * 128, True, WS)[:2] == (128, 256)
    assert (T > chunk) == ((T, d, F) == E.CHUNKS)
    assert (T, d, F) == E.CHUNKS or F % 256 in (0, 64, 128, 192)


def test_few_tokens():
    """Whether x and whether a slice of the hidden values are quantised in place, and whether K is cut."""
    def way(T, d, F):
        tiles, pitch = ceil(d, 32), ceil(F, 128)
        slices = min(8, max(1, 256 // tiles))
        while slices > 1 and pitch * 4 // slices < 32:
            slices -= 1
        while slices > 1 and ceil(pitch, slices) * (slices - 1) >= pitch:
            slices -= 1
        return T * ceil(d, 128) * 8 <= 1024, T * ceil(pitch, slices) * 8 <= 1024, slices > 1

    assert [way(*shape) for shape in E.FEW] == [(True, False, True), (False, True, True), (True, True, True), (True, True, True), (True, True, False), (True, True, True)]
