"""What the calls around the layer check without a GPU."""
import ctypes
import os

import pytest
import torch

from paper_2601_10639_amd import stemlib as L


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(L.LIB_PATH):
        from paper_2601_10639_amd import build
        build.build()
    return L.lib()


def test_null_context_is_refused(lib):
    z = ctypes.c_void_p(None)
    bad = L.STEM_ERR_INVALID_ARG
    assert lib.stem_block_enter_forward(z, z, 1, None, z, z) == bad
    assert lib.stem_block_enter_backward(z, z, z, 1, None, z, z, z, 0, z) == bad
    assert lib.stem_block_leave_forward(z, z, z, 1, None, z, z, z) == bad
    assert lib.stem_block_leave_backward(z, z, z, z, z, 1, None, z, z, z, z, z, 0, z) == bad
    assert lib.stem_dropout(z, z, 1, 1, None, z, z) == bad
    assert lib.stem_quant_weights(z, z, 1, 1, z, z, z) == bad
    assert lib.stem_quant_linear(z, z, 1, 1, None, z, z, 1, z, z, z) == bad
    assert lib.stem_quant_ffn_forward(z, z, z, 1, None, z, z, z, z, z, 1, z, z, z) == bad


def test_quant_bytes(lib):
    assert L.stem_quant_bytes(1, 1) == 32 * 128
    assert L.stem_quant_bytes(32, 128) == 32 * 128
    assert L.stem_quant_bytes(33, 129) == 64 * 256
    assert L.stem_quant_bytes(8192, 2048) == 8192 * 2048
    assert L.stem_quant_bytes(0, 5) == L.stem_quant_bytes(5, 0) == L.stem_quant_bytes(-1, 5) == 0


def test_layout_of_the_argument_structures(lib):
    assert ctypes.sizeof(L.stem_norm) == 16 and ctypes.sizeof(L.stem_drop) == 32 and ctypes.sizeof(L.stem_leave) == 88
    leave = L.stem_leave(out=L.stem_norm(L.STEM_NORM_RMS, 0.5), residual_scale=2.0, branch_scale=3.0, p=0.25, seed=2 ** 63, offset=7)
    assert (leave.out.kind, leave.out.eps, leave.next.kind) == (L.STEM_NORM_RMS, 0.5, L.STEM_NORM_NONE)
    assert (leave.residual_scale, leave.branch_scale, leave.gate_kind, leave.gate) == (2.0, 3.0, L.STEM_GATE_NONE, None)
    assert (leave.drop.p, leave.drop.seed, leave.drop.offset, leave.drop.step) == (0.25, 2 ** 63, 7, None)


def test_binding_refuses_host_tensors_and_wrong_types(lib):
    class Fake:
        handle = ctypes.c_void_p(None)
        torch_dtype = torch.bfloat16
        d_model, d_ff = 64, 64

    x, f = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4, 64)
    norm = L.stem_norm(L.STEM_NORM_RMS)
    for call in (lambda: L.stem_block_enter_forward(Fake(), x, norm, x), lambda: L.stem_block_enter_forward(Fake(), f, norm, x),
                 lambda: L.stem_block_enter_backward(Fake(), x, x, norm, x), lambda: L.stem_block_leave_forward(Fake(), x, x, L.stem_leave(), x),
                 lambda: L.stem_block_leave_backward(Fake(), x, None, x, None, L.stem_leave(), x, x), lambda: L.stem_dropout(Fake(), x, x, 0.1, 1),
                 lambda: L.stem_norm(L.STEM_NORM_RMS, 1e-5, x), lambda: L.stem_leave(gate_kind=1, gate=x[0])):
        with pytest.raises((TypeError, ValueError)):
            call()
