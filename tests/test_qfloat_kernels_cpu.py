"""Every kernel of few rows that is built is one that some call takes."""
import ctypes
import re
import shutil
import subprocess

import pytest

from paper_2601_10639_amd import stemlib as L

FORM, ROWS, HIDDEN = range(3)


def route(T, groups, N, K, form):
    r = (ctypes.c_int32 * 3)()
    L.lib().stem_route_qfloat_decode(ctypes.c_int64(T), groups, N, K, form, r)
    return tuple(r)


def few(T, N, K):
    return L.lib().stem_route_qfloat_few(ctypes.c_int64(T), 0, N, K)


@pytest.mark.skipif(shutil.which("nm") is None, reason="needs nm")
def test_kernels_of_few_rows():
    L.lib()
    names = subprocess.run(["nm", L.LIB_PATH], capture_output=True, text=True, check=True).stdout
    built = {tuple(map(int, m)) for m in re.findall(r"decode_kernelILi(\d+)ELi(\d+)ELNS_6SourceE(\d)ELi(\d+)ELb(\d)EEEv16QfloatDecodeArgs", names)}
    assert built
    taken = set()

    def take(T, groups, N, K, source, gate):
        channels, tiles, depth = route(T, groups, N, -(-K // 128) * 128, int(source == FORM))
        taken.add((channels, tiles, source, depth, gate))

    widths = (64, 1000, 2048, 3000, 4096, 5000, 8192)
    for N in (64, 500, 2000, 4096, 8192, 16400, 70000):
        for T in list(range(1, 17)) + [17, 20, 33, 64, 100, 200, 256]:
            for K in widths + (9000, 20000):
                if T <= 16 and K <= 8192:
                    take(T, 1, N, K, ROWS, 0)
                    if K % 64 == 0 and N % 64 == 0:
                        take(T, 1, N, K, ROWS, 1)
                    if T * K <= 32768:
                        take(T, 1, N, K, HIDDEN, 0)
                elif few(T, N, K):
                    take(T, 1, N, K, FORM, 0)
    assert built == taken


def test_two_tiles_of_rows_have_32_channels():
    for T in range(1, 257):
        for N in (1, 300, 1024, 2049, 4096, 8191, 16384, 70001):
            for groups in (1, 3, 512):
                channels, tiles, _ = route(T, groups, N, 1024, 1)
                assert tiles == 1 or channels == 32
