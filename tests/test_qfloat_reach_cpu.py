"""The shapes of the 8-bit floating point products' GPU tests reach the kernels that they are there for."""
import ctypes

import pytest

from paper_2601_10639_amd import stemlib as L
from tests import test_gpu_qfloat_edges as G

BF16, F32, HIDDEN = range(3)
WS = 256 * 128 * 128 * 4


def tiles(T, N, K, out=BF16, groups=1):
    r = (ctypes.c_int32 * 3)()
    L.lib().stem_route_qfloat(ctypes.c_int64(T), groups, N, -(-K // 128) * 128, out, ctypes.c_int64(WS), r)
    return tuple(r)


def few(T, N, K, grouped=0):
    return L.lib().stem_route_qfloat_few(ctypes.c_int64(T), grouped, N, K)


def decode(T, N, K, form, groups=1):
    r = (ctypes.c_int32 * 3)()
    L.lib().stem_route_qfloat_decode(ctypes.c_int64(T), groups, N, K, form, r)
    return tuple(r)


@pytest.mark.parametrize("name,want", [("ring", (256, 256, 1)), ("pair", (128, 256, 1)), ("128x128", (128, 128, 1)), ("128x64", (128, 64, 1)),
                                       ("2 slices", (128, 64, 2)), ("3 slices", (128, 64, 3)), ("4 slices", (128, 64, 4))])
def test_tiles(name, want):
    assert tiles(*G.TILES[name]) == want and not few(*G.TILES[name])


# (channels, 16-row tiles, depth), rows made to operands in place or a form
@pytest.mark.parametrize("name,form,want", [
    ("8 channels", 0, (8, 1, 1)), ("16 channels", 0, (16, 1, 2)), ("32 channels", 0, (32, 1, 4)), ("depth 8", 0, (8, 1, 8)), ("turns", 1, (8, 1, 8)),
    ("form, depth 1", 1, (8, 1, 1)), ("form, depth 2", 1, (8, 1, 2)), ("form, depth 4", 1, (16, 1, 4)), ("form, depth 8", 1, (8, 1, 8)), ("form, turns", 1, (8, 1, 8)),
    ("form, 32 rows", 1, (32, 2, 2)), ("form, 32 rows, 16 channels", 1, (32, 2, 2))])
def test_few_rows(name, form, want):
    T, N, K = G.FEW[name]
    assert few(T, N, K) and (T <= 16 and K <= 8192) == (not form) and decode(T, N, K, form) == want
    assert (K > 8192) == ("turns" in name)       # more blocks than a wavefront has under way


@pytest.mark.parametrize("name,want", [("64x128", (64, 128)), ("128x128", (128, 128)), ("pair", (128, 256))])
def test_gates(name, want):
    T, d, F = G.GATES[name]
    assert tiles(T, F, d, HIDDEN)[:2] == want and T > 16


def test_gates_of_few_rows():
    for name, inline in (("few, inline", True), ("few, by a kernel", False), ("16, by a kernel", False)):
        T, d, F = G.GATES[name]
        assert T <= 16 and (T * F <= 32768) == inline


def test_weight_gradient():
    T, N, K = G.WEIGHT_SLICES
    assert tiles(N, K, -(-T // 64) * 128, F32) == (128, 128, 5)
    for (T, N, K, groups), want in zip(G.WEIGHTS, [(128, 128, 8), (128, 128, 3), (128, 256, 1), (128, 256, 1)]):
        assert tiles(N, K, -(-T // groups // 64) * 128, F32, groups) == want


def test_slices_fit_their_room():
    for T in (1, 100, 256, 257, 700, 1000, 1300, 2048, 4096, 20000):
        for N in (1, 64, 200, 1001, 2048, 8192):
            for K in (1, 128, 4096, 8192, 30000):
                for out in (BF16, F32, HIDDEN):
                    for groups in (1, 4):
                        rows, cols, slices = tiles(T, N, K, out, groups)
                        n = -(-T // rows) * -(-N // cols) * (groups if out == F32 else 1)
                        assert slices == 1 or ((groups == 1 or out == F32) and out != HIDDEN and slices * n <= 256 and slices * n * rows * cols * 4 <= WS)
                        nk = -(-K // 128)
                        assert -(-nk // slices) * (slices - 1) < nk          # every slice has a part of K
