"""The block's and the 8-bit calls' native binding against the same calls made from Python: the same bits, and the same refusals."""
import pytest
import torch

from paper_2601_10639_amd import stemlib as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
bf = torch.bfloat16


def native():
    return L._bind or L._load_bind()


@pytest.fixture
def count(monkeypatch):
    """How many calls were made natively; `count.off()` makes them from Python from then on."""
    real = native()
    if isinstance(real, L._NoBind):
        pytest.skip("no native binding here")

    class Counting:
        calls = 0

        def __getattr__(self, name):
            f = getattr(real, name)

            def call(*a):
                st = f(*a)
                self.calls += st is not None
                return st
            return call

        def off(self):
            monkeypatch.setattr(L, "_bind", L._NoBind())

    c = Counting()
    monkeypatch.setattr(L, "_bind", c)
    return c


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gate", ["none", "channel", "token", "full"])
def test_block_calls(count, dtype, gate):
    T, d = 13, 192
    dt = bf if dtype == "bf16" else torch.float32
    ctx = L.stem_create(d, 64, 10, L.STEM_BF16 if dtype == "bf16" else L.STEM_F32, T)
    gen = torch.Generator().manual_seed(1)

    def draw(*shape):
        return torch.randn(*shape, generator=gen).to(dt).to(DEV)

    x, f, dy, dn, w = draw(T, d), draw(T, d), draw(T, d), draw(T, d), draw(d)
    kind, shape = {"none": (0, None), "channel": (1, (d,)), "token": (2, (T,)), "full": (3, (T, d))}[gate]
    g = draw(*shape) if shape else None
    norm = L.stem_norm(L.STEM_NORM_RMS, 1e-5, w)
    leave = L.stem_leave(out=norm, next=norm, gate_kind=kind, gate=g, p=0.1, seed=5, offset=6)

    def run():
        y, n, m, dx, df, ex, z = (torch.zeros_like(x) for _ in range(7))
        dg = None if g is None else torch.zeros_like(g, dtype=torch.float32 if gate == "channel" else dt)
        a, b, c = (torch.zeros(d, device=DEV) for _ in range(3))
        L.stem_block_leave_forward(ctx, f, x, leave, y, n)
        L.stem_block_leave_backward(ctx, dy, dn, f, y, leave, dx, df, dg, a, b)
        L.stem_block_enter_forward(ctx, x, norm, m)
        L.stem_block_enter_backward(ctx, dn, x, norm, ex, c, dres=dy, accumulate=True)
        L.stem_dropout(ctx, x, z, 0.25, 7, 8)
        return [y, n, m, dx, df, ex, z, a, b, c] + ([] if dg is None else [dg])

    first = run()
    assert count.calls == 5
    count.off()
    assert all(torch.equal(p, q) for p, q in zip(first, run()))


def test_quant_calls(count):
    T, d, F = 9, 128, 320
    ctx = L.stem_create(d, F, 50, L.STEM_BF16, T, reserve=L.STEM_RESERVE_QUANT)
    gen = torch.Generator().manual_seed(2)

    def draw(*shape):
        return torch.randn(*shape, generator=gen).to(bf).to(DEV)

    x, E, norm = draw(T, d), draw(50, F), L.stem_norm(L.STEM_NORM_RMS, 1e-5, draw(d))
    g, w = L.stem_quant_weights(ctx, draw(F, d)), L.stem_quant_weights(ctx, draw(d, F))
    ids = torch.arange(T, dtype=torch.int32, device=DEV)

    def run():
        y, z = torch.zeros_like(x), torch.zeros(T, F, dtype=bf, device=DEV)
        L.stem_quant_ffn_forward(ctx, x, ids, g, w, E, y, residual=x, norm=norm)
        L.stem_quant_linear(ctx, x, g, z)
        return y, z

    first = run()
    assert count.calls == 2
    count.off()
    assert all(torch.equal(p, q) for p, q in zip(first, run()))


def test_what_is_not_ordinary_is_left_to_python(count):
    T, d = 5, 64
    ctx = L.stem_create(d, 64, 10, L.STEM_BF16, 8)
    x, w = torch.ones(T, d, dtype=bf, device=DEV), torch.ones(d, dtype=bf, device=DEV)
    norm, y = L.stem_norm(L.STEM_NORM_RMS, 1e-5, w), torch.empty_like(x)
    bad = [lambda: L.stem_block_enter_forward(ctx, x, L.stem_norm(1, 1e-5, w[:32]), y), lambda: L.stem_block_enter_forward(ctx, x, L.stem_norm(1, 1e-5, w.float()), y),
           lambda: L.stem_block_enter_forward(ctx, x, norm, y[:2]), lambda: L.stem_block_enter_forward(ctx, x, norm, y.float()),
           lambda: L.stem_block_leave_forward(ctx, x, x, L.stem_leave(gate_kind=1, gate=w[:8]), y),
           lambda: L.stem_block_leave_forward(ctx, x, x, L.stem_leave(gate_kind=3, gate=w), y),
           lambda: L.stem_block_leave_forward(ctx, x, x, L.stem_leave(out=L.stem_norm(0, 0.0, w.float())), y),
           lambda: L.stem_block_leave_backward(ctx, x, None, x, None, L.stem_leave(gate_kind=1, gate=w), y, None, w)]
    for call in bad:
        with pytest.raises((TypeError, ValueError)):
            call()
    assert count.calls == 0
    L.stem_dropout(ctx, x, y, 0.5, 2 ** 64 - 1)     # a seed that is no C long: made from Python
    assert count.calls == 0
    L.stem_dropout(ctx, x, y, 0.5, 2 ** 63 - 1)
    assert count.calls == 1
