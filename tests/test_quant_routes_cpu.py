"""How the 8-bit products cut their work, asked through the function that their launcher asks; no GPU."""
import ctypes
import random

import pytest

from paper_2601_10639_amd import stemlib as L


def route(M, N, K, gate, ws):
    r = (ctypes.c_int32 * 3)()
    L.lib().stem_route_quant(M, N, K, int(gate), ctypes.c_int64(ws), r)
    return tuple(r)


def ceil(a, b):
    return -(-a // b)


def test_every_slice_has_a_part_of_k_and_room():
    rng = random.Random(1)
    for _ in range(20000):
        M, N, K = int(65 * 400 ** rng.random()), int(1 + 16000 ** rng.random()), 128 * int(1 + 100 ** rng.random())
        ws, gate = int(2 ** (10 + 17 * rng.random())), rng.random() < 0.5
        rows, cols, slices = route(M, N, K, gate, ws)
        assert (rows, cols) in ((128, 64), (128, 128), (128, 256), (256, 256))
        tiles, nk = ceil(M, rows) * ceil(N, cols), K // 128
        assert 1 <= slices <= 4 and (slices - 1) * ceil(nk, slices) < nk
        if slices > 1:
            assert cols == 64 and not gate and tiles <= 128 and slices * tiles * 128 * 64 * 4 <= ws
        assert not gate or (rows, cols) != (256, 256)


@pytest.mark.parametrize("M,N,K,gate,want", [(256, 8192, 2048, True, (128, 128, 1)), (256, 4096, 1024, True, (128, 64, 1)), (256, 2048, 8192, False, (128, 64, 3)),
                                             (400, 2048, 8192, False, (128, 64, 2)), (1024, 1024, 4096, False, (128, 64, 1)), (1500, 2048, 8192, False, (128, 128, 1)),
                                             (4096, 2048, 8192, False, (128, 256, 1)), (16384, 2048, 8192, False, (256, 256, 1)), (4096, 8192, 2048, True, (128, 256, 1))])
def test_measured_choices(M, N, K, gate, want):
    assert route(M, N, K, gate, 64 << 20) == want


@pytest.mark.parametrize("M,N,K,slices", [(700, 1001, 2048, 1), (256, 1024, 2048, 1), (512, 1024, 2944, 1), (128, 1024, 4096, 3), (1024, 512, 4096, 3), (80, 2048, 8192, 4)])
def test_short_products_are_not_cut(M, N, K, slices):
    assert route(M, N, K, False, 64 << 20) == (128, 64, slices)
