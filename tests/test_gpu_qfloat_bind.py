"""The native binding of the 8-bit floating point calls and those of experts against the same calls made from Python: the same bits, and the same refusals."""
import pytest
import torch

from paper_2601_10639_amd import stemlib as L
from tests.test_gpu_block_bind import count, native   # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
bf, i32 = torch.bfloat16, torch.int32


def make():
    ctx = L.stem_create(64, 128, 20, L.STEM_BF16, 16)
    L.stem_qfloat_reserve(ctx, 2, True)
    gen = torch.Generator().manual_seed(1)
    draw = lambda *shape: torch.randn(*shape, generator=gen).to(bf).to(DEV)
    x, y, dy, r, E = draw(16, 64), draw(16, 128), draw(16, 128), draw(16, 128), draw(20, 128)
    gate, down = L.stem_qfloat_weights(ctx, draw(2, 128, 64), backward=True), L.stem_qfloat_weights(ctx, draw(2, 64, 128))
    off, ids = torch.tensor([1, 9, 15], dtype=i32, device=DEV), torch.arange(16, dtype=i32, device=DEV)
    norm = L.stem_norm(L.STEM_NORM_RMS, 1e-5, draw(64))
    e = torch.randint(-1, 3, (8, 2), generator=gen).to(i32).to(DEV)
    w = torch.rand(8, 2, generator=gen).to(DEV)
    return ctx, locals()


def run(ctx, c, stream=None):
    """Every call once; what they leave."""
    zeros = lambda *s, dtype=bf: torch.zeros(*s, dtype=dtype, device=DEV)
    y, z, dx, dW = zeros(16, 128), zeros(16, 64), zeros(16, 64), zeros(2, 128, 64, dtype=torch.float32)
    L.stem_qfloat_linear(ctx, c["x"], c["gate"], y, residual=c["r"], norm=c["norm"], offsets=c["off"], stream=stream)
    L.stem_qfloat_linear_backward(ctx, c["dy"], c["x"], c["gate"], dx, dW, offsets=c["off"], stream=stream)
    L.stem_qfloat_linear_backward(ctx, c["dy"], c["x"], c["gate"], dW=dW, offsets=c["off"], accumulate=True, stream=stream)
    L.stem_qfloat_ffn_forward(ctx, c["x"], c["ids"], c["gate"], c["down"], c["E"], z, norm=c["norm"], offsets=c["off"], stream=stream, E_rows=20)
    src, place, off = zeros(16, dtype=i32), zeros(8, 2, dtype=i32), zeros(4, dtype=i32)
    xs, ids, out, dys, dw = zeros(16, 64), zeros(16, dtype=i32), zeros(8, 64), zeros(16, 64), zeros(8, 2, dtype=torch.float32)
    L.stem_experts_sort(ctx, c["e"], src, place, off, stream=stream)
    L.stem_experts_dispatch(ctx, c["x"][:8], src, xs, choices=2, ids=c["ids"][:8], ids_out=ids, stream=stream)
    L.stem_experts_combine(ctx, c["x"], place, out, weights=c["w"], residual=c["x"][:8], stream=stream)
    L.stem_experts_combine_backward(ctx, c["x"][:8], place, dys, ys=c["x"], weights=c["w"], dweights=dw, stream=stream)
    torch.cuda.synchronize()
    return y, z, dx, dW, src, place, off, xs, ids, out, dys, dw


def test_calls(count):
    ctx, c = make()
    a = run(ctx, c)
    assert count.calls == 8
    s = torch.cuda.Stream()
    b = run(ctx, c, s)
    assert count.calls == 16
    count.off()
    for other in (b, run(ctx, c), run(ctx, c, s)):
        assert all(torch.equal(p, q) for p, q in zip(a, other))


def test_unusual_arguments_are_refused_as_from_python(count):
    ctx, c = make()
    x, y, off = c["x"], c["y"], c["off"]
    other = torch.zeros(16, 128, dtype=bf, device=DEV)
    for call, error in ((lambda: L.stem_qfloat_linear(ctx, x, c["gate"], y[:8], offsets=off), ValueError),
                        (lambda: L.stem_qfloat_linear(ctx, x.float(), c["gate"], y, offsets=off), TypeError),
                        (lambda: L.stem_qfloat_linear(ctx, x, c["gate"], y, offsets=off[:2]), ValueError),
                        (lambda: L.stem_qfloat_linear(ctx, x, c["gate"], y.t().contiguous().t(), offsets=off), ValueError),
                        (lambda: L.stem_qfloat_linear(ctx, x, L.StemQfloat(c["gate"].q[1:], None, 2, 128, 64), y, offsets=off), ValueError),
                        (lambda: L.stem_qfloat_linear_backward(ctx, y, x, c["gate"], dW=torch.zeros(128, 64, device=DEV), offsets=off), ValueError),
                        (lambda: L.stem_qfloat_linear_backward(ctx, y, x, c["down"], dx=other, offsets=off), ValueError),
                        (lambda: L.stem_qfloat_ffn_forward(ctx, x, c["ids"], c["down"], c["gate"], c["E"], x, offsets=off), ValueError),
                        (lambda: L.stem_experts_sort(ctx, c["e"], c["ids"][:3], c["e"].clone(), off), ValueError),
                        (lambda: L.stem_experts_dispatch(ctx, x, c["ids"], other, choices=2), ValueError),
                        (lambda: L.stem_experts_combine(ctx, x, c["e"], x[:7]), ValueError),
                        (lambda: L.stem_experts_combine_backward(ctx, x[:8], c["e"], x[:8].clone(), ys=x), ValueError),
                        (lambda: L.stem_qfloat_linear(ctx, x, c["gate"], x.cpu(), offsets=off), ValueError)):
        with pytest.raises(error):
            call()
    with pytest.raises(L.StemError) as err:
        L.stem_qfloat_linear(ctx, x, c["gate"], y)
    assert err.value.status == L.STEM_ERR_INVALID_ARG
    one = L.stem_qfloat_weights(ctx, torch.ones(128, 64, dtype=bf, device=DEV), backward=True)
    dW = torch.zeros(128, 64, device=DEV)
    before = count.calls
    L.stem_qfloat_linear_backward(ctx, y, x, one, dW=dW)          # [N, K] of one group
    assert count.calls == before + 1 and dW.any()
