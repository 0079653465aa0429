"""What the 8-bit floating point calls and those of experts check without a GPU, and pins of their oracle."""
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


def test_null_context_is_refused(lib):
    z, bad = ctypes.c_void_p(None), L.STEM_ERR_INVALID_ARG
    assert lib.stem_qfloat_reserve(z, 1, 0) == bad
    assert lib.stem_qfloat_weights(z, z, 1, 1, 1, z, z, z) == bad
    assert lib.stem_qfloat_linear(z, z, 1, 1, None, z, 1, 1, z, z, z, z) == bad
    assert lib.stem_qfloat_linear_backward(z, z, z, 1, 1, z, 1, 1, z, z, z, 0, z) == bad
    assert lib.stem_qfloat_ffn_forward(z, z, z, 1, None, z, z, 1, z, z, 1, z, z, z) == bad
    assert lib.stem_experts_sort(z, z, 1, 1, 1, z, z, z, z) == bad
    assert lib.stem_experts_dispatch(z, z, 1, 1, z, 1, 1, z, z, z, z) == bad
    assert lib.stem_experts_combine(z, z, 1, 1, z, z, 1, 1, z, z, z) == bad
    assert lib.stem_experts_combine_backward(z, z, z, 1, 1, z, z, 1, 1, z, z, z) == bad


def test_bytes(lib):
    assert L.stem_qfloat_bytes(1, 1) == L.stem_qfloat_bytes(128, 128) == 128 * 129
    assert L.stem_qfloat_bytes(129, 128) == L.stem_qfloat_bytes(128, 129) == 2 * 128 * 129
    assert L.stem_qfloat_bytes(8192, 2048) == 8192 * 2048 // 128 * 129
    assert L.stem_qfloat_bytes(0, 5) == L.stem_qfloat_bytes(5, 0) == L.stem_qfloat_bytes(-1, 5) == 0


def test_binding_refuses_host_tensors_wrong_types_and_shapes(lib):
    class Fake:
        handle = ctypes.c_void_p(None)
        torch_dtype = torch.bfloat16
        d_model, d_ff = 64, 64

    x, i = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4, 2, dtype=torch.int32)
    w = L.StemQfloat(torch.zeros(L.stem_qfloat_bytes(64, 64), dtype=torch.uint8), None, 1, 64, 64)
    for call in (lambda: L.stem_qfloat_linear(Fake(), x, w, x), lambda: L.stem_qfloat_linear_backward(Fake(), x, x, w, x),
                 lambda: L.stem_qfloat_ffn_forward(Fake(), x, i[:, 0], w, w, x, x), lambda: L.stem_qfloat_weights(Fake(), x),
                 lambda: L.stem_experts_sort(Fake(), i, i.view(-1), i, i[:, 0]), lambda: L.stem_experts_dispatch(Fake(), x, i.view(-1), x, 2),
                 lambda: L.stem_experts_combine(Fake(), x, i, x), lambda: L.stem_experts_combine_backward(Fake(), x, i, x),
                 lambda: L.stem_qfloat_ffn_forward(Fake(), x, i[:, 0], w, L.StemQfloat(w.q, None, 2, 64, 64), x, x)):
        with pytest.raises((TypeError, ValueError)):
            call()


# ---- the oracle -----------------------------------------------------------------------------------------------------------

def test_values_of_the_format():
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    numbers = every[np.isfinite(every)]
    assert np.array_equal(Q.e4m3(numbers), numbers) and numbers.max() == 448
    rng = np.random.default_rng(0)
    v = np.concatenate([rng.standard_normal(20000) * 100, rng.standard_normal(20000) * 0.01, np.ldexp(rng.random(1000), -9)])
    v = v[np.abs(v) <= 448].astype(np.float32)
    assert np.array_equal(Q.e4m3(v), torch.from_numpy(v).to(torch.float8_e4m3fn).double().numpy())
    middles = (np.sort(numbers)[1:] + np.sort(numbers)[:-1]) / 2     # to even
    assert np.array_equal(Q.e4m3(middles), torch.from_numpy(middles.astype(np.float32)).to(torch.float8_e4m3fn).double().numpy())
    assert np.isnan(Q.e4m3([np.inf, -np.inf, np.nan])).all()


def test_exponents():
    assert Q.exponent([448.0, 448.0000001, 224.0, 449.0, 1.75, 1.76, 0.0, 1e-45]).tolist() == [0, 1, -1, 1, -8, -7, -126, -126]
    for top in np.random.default_rng(1).lognormal(0, 20, 1000):
        e = int(Q.exponent(top))
        assert top <= 448.0 * 2.0 ** e and (e == -126 or top > 448.0 * 2.0 ** (e - 1))


def test_blocks_are_their_own():
    rng = np.random.default_rng(2)
    v = rng.standard_normal((5, 300)) * np.exp(rng.standard_normal((5, 1)))
    q = Q.blocks(v, 1)
    assert np.abs(q - v).max() <= np.abs(v).max() / 16
    assert np.array_equal(Q.blocks(q, 1), q)                               # its own values
    assert np.array_equal(Q.blocks(4 * v, 1), 4 * q)
    assert np.array_equal(Q.blocks(v[:, :128], 1), q[:, :128]) and np.array_equal(Q.blocks(v.T, 0), q.T)
    W = rng.standard_normal((200, 140))
    assert np.array_equal(Q.squares(W.T), Q.squares(W).T)
    v[2, 7], v[2, 8] = np.inf, np.nan                                      # numbers beside them are what they would be without
    some = Q.blocks(v, 1)
    assert np.isnan(some[2, 7:9]).all() and np.array_equal(np.delete(some[2], [7, 8])[126:], np.delete(q[2], [7, 8])[126:])


def test_bounds():
    assert Q.bounds(None, 9, 1) == [(0, 9)]
    assert Q.bounds([2, 5, 3, 99], 9, 3) == [(2, 5), (5, 5), (5, 9)]
    assert Q.bounds([-4, -2, 6], 9, 2) == [(0, 0), (0, 6)]


def test_gradients_against_differences():
    """Of the product with Q taken as it is: moves that Q has as values, in both operands."""
    rng = np.random.default_rng(3)
    x, W, dy = rng.integers(-4, 5, (6, 130)).astype(float), rng.integers(-4, 5, (2, 5, 130)).astype(float), rng.integers(-4, 5, (6, 5)).astype(float)
    off = [0, 2, 6]
    (dx, _), (dW, _) = Q.linear_backward(dy, x, W, off)
    value = lambda x, W: (Q.linear(x, W, off)[0] * dy).sum()
    for t, k in ((0, 0), (3, 129), (5, 64)):
        up, down = x.copy(), x.copy()
        up[t, k] += 1
        down[t, k] -= 1
        assert (value(up, W) - value(down, W)) / 2 == dx[t, k]
    for g, n, k in ((0, 0, 0), (1, 4, 129), (1, 2, 70)):
        up, down = W.copy(), W.copy()
        up[g, n, k] += 1
        down[g, n, k] -= 1
        assert (value(x, up) - value(x, down)) / 2 == dW[g, n, k]


def test_layer_is_its_products():
    rng = np.random.default_rng(4)
    n, Wg, Wd, E = rng.standard_normal((7, 64)), rng.standard_normal((2, 128, 64)), rng.standard_normal((2, 64, 128)), rng.standard_normal((9, 128))
    ids, off = rng.integers(0, 9, 7), [0, 3, 7]
    y = Q.ffn(n, ids, Wg, Wd, E, off)
    for t in range(7):
        g = int(t >= 3)
        z = Q.blocks(n[t:t + 1], 1) @ Q.squares(Wg[g]).T
        h = z / (1 + np.exp(-z)) * E[ids[t]]
        assert np.allclose(y[t], (Q.blocks(h, 1) @ Q.squares(Wd[g]).T)[0], rtol=1e-12)
