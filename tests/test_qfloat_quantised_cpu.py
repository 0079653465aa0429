"""Weight gradients of values in 8 bits: what is checked without a GPU, and pins of the oracle."""
import ctypes
import os

import numpy as np
import pytest
import torch

from oracle import qfloat_oracle as Q
from paper_2601_10639_amd import stemlib as L


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(L.LIB_PATH):
        from paper_2601_10639_amd import build
        build.build()
    return L.lib()


def test_refusals(lib):
    z = ctypes.c_void_p(None)
    assert lib.stem_qfloat_linear_backward_quantised(z, z, z, 1, 1, z, 1, 1, z, z, z, 0, z) == L.STEM_ERR_INVALID_ARG

    class Fake:
        handle = z
        torch_dtype = torch.bfloat16
        d_model, d_ff = 64, 64

    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    w = L.StemQfloat(torch.zeros(L.stem_qfloat_bytes(64, 64), dtype=torch.uint8), None, 1, 64, 64)
    with pytest.raises((TypeError, ValueError)):
        L.stem_qfloat_linear_backward_quantised(Fake(), x, x, w, x)


def test_oracle():
    """Element by element; whole numbers that the format has are kept, others move by a sixteenth at most; a group's blocks begin at its first row."""
    rng = np.random.default_rng(1)
    off = [3, 5, 5, 290, 300]
    dy, x = rng.standard_normal((310, 3)), rng.standard_normal((310, 4)) * np.exp(rng.standard_normal((310, 1)))
    dW, size = Q.weight_gradient_quantised(dy, x, 4, off)
    for g, (lo, hi) in enumerate(zip(off, off[1:])):
        for n in range(3):
            for k in range(4):
                total = 0.0
                for t0 in range(lo, hi, 128):
                    a, b = dy[t0:min(t0 + 128, hi), n], x[t0:min(t0 + 128, hi), k]
                    ea, eb = (2.0 ** float(Q.exponent(np.abs(v).max())) for v in (a, b))
                    total += (Q.e4m3(a / ea) * ea) @ (Q.e4m3(b / eb) * eb)
                assert abs(total - dW[g, n, k]) <= 1e-12 * size[g, n, k]
    exact = np.stack([dy[lo:hi].T @ x[lo:hi] for lo, hi in zip(off, off[1:])])
    assert not dW[1].any() and 0.005 < np.linalg.norm(dW - exact) / np.linalg.norm(exact) < 2 / 16
    dy, x = rng.integers(-8, 9, (310, 3)).astype(float), rng.integers(-8, 9, (310, 4)).astype(float)
    assert np.array_equal(Q.weight_gradient_quantised(dy, x, 4, off)[0], np.stack([dy[lo:hi].T @ x[lo:hi] for lo, hi in zip(off, off[1:])]))
