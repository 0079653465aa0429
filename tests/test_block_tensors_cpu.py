"""What the block's structures hold of the tensors that they are given, without a GPU: host tensors stand for device tensors."""
import gc
import weakref

import pytest
import torch

from paper_2601_10639_amd import stemlib as L


class Context:
    torch_dtype, d_model = torch.float32, 8


@pytest.fixture(autouse=True)
def any_memory(monkeypatch):
    monkeypatch.setattr(L, "_ptr", lambda t, *args, **kwargs: None if t is None else t.data_ptr())


def test_pointers_are_those_of_the_call():
    a, b, g, step = torch.zeros(8), torch.zeros(8), torch.zeros(3, 8), torch.zeros(1, dtype=torch.int64)
    norm = L.stem_norm(L.STEM_NORM_RMS, 1e-5, a)
    leave = L.stem_leave(out=norm, next=L.stem_norm(L.STEM_NORM_RMS, 1e-5, b), gate_kind=L.STEM_GATE_FULL, gate=g, p=0.1, step=step)
    held = [t.data for t in (a, b, g, step)]
    for t in (a, b, g, step):
        t.data = t.data.clone()
    assert all(t.data_ptr() != h.data_ptr() for t, h in zip((a, b, g, step), held))
    norm._check(Context, 8, "norm")
    leave._check(Context, 3)
    assert norm.weight == a.data_ptr()
    assert (leave.out.weight, leave.next.weight, leave.gate, leave.drop.step) == (a.data_ptr(), b.data_ptr(), g.data_ptr(), step.data_ptr())
    with pytest.raises(ValueError):
        leave._check(Context, 2)


def test_what_is_given_anew_is_kept_alive():
    leave = L.stem_leave(out=L.stem_norm(L.STEM_NORM_RMS, 1e-5, torch.zeros(8)))
    step, w, v = torch.zeros(1, dtype=torch.int64), torch.zeros(8), torch.zeros(8)
    leave.drop = L.stem_drop(0.25, 1, 2, step=step)
    leave.out, leave.next = L.stem_norm(L.STEM_NORM_LAYER, 1e-3, w), L.stem_norm(L.STEM_NORM_RMS, 1e-4, v)
    here, at = [weakref.ref(t) for t in (step, w, v)], [t.data_ptr() for t in (step, w, v)]
    del step, w, v
    gc.collect()
    assert all(r() is not None for r in here)
    leave._check(Context, 3)
    assert [leave.drop.step, leave.out.weight, leave.next.weight] == at
    assert (leave.out.kind, leave.next.kind, leave.drop.p) == (L.STEM_NORM_LAYER, L.STEM_NORM_RMS, 0.25)
    # a pointer that is taken out stays out, and numbers that are changed stay changed
    leave.drop.step = None
    leave.out.eps = 0.5
    leave._check(Context, 3)
    assert leave.drop.step is None and leave.out.eps == 0.5


@pytest.mark.parametrize("short", ["q", "scale"])
def test_quantised_weights_of_another_size_are_refused(short):
    N, K = 40, 100
    q, scale = torch.zeros(L.stem_quant_bytes(N, K), dtype=torch.int8), torch.zeros(N)
    assert L._quant(L.StemQuant(q, scale, N, K), N, K, "W") == (q.data_ptr(), scale.data_ptr())
    bad = L.StemQuant(q[:-1], scale, N, K) if short == "q" else L.StemQuant(q, scale[:-1], N, K)
    with pytest.raises(ValueError):
        L._quant(bad, N, K, "W")


@pytest.mark.parametrize("n", [0, 2])
def test_a_step_is_one_element(n):
    step = torch.zeros(n, dtype=torch.int64)
    with pytest.raises(ValueError):
        L.stem_drop(0.1, 1, 2, step=step)
    with pytest.raises(ValueError):
        L.stem_leave(p=0.1, step=step)
    one = torch.zeros(1, dtype=torch.int64)
    leave = L.stem_leave(p=0.1, step=one)
    one.data = step
    with pytest.raises(ValueError):
        leave._check(Context, 3)
