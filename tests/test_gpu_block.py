"""Norms, dropout, gate and residual around the layer on the GPU, against the oracle in 64 bits.

Tolerances, max |gpu - ref| / max |ref| of a tensor.  fp32: values come of about ten roundings of 6e-8 and sums of up to a few
thousand terms in fp32, taken in parts: 1e-5.  bf16: inputs are exact and an output is rounded once to 8 bits, by up to 2^-8 of its own
magnitude: 2^-8 plus the fp32 error.  Sums over tokens are fp32 in both."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as B
from paper_2601_10639_amd import stemlib as L
from tests.harness import max_rel

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32_TOL = 1e-5
TOL = {"f32": F32_TOL, "bf16": 2.0 ** -8 + F32_TOL}
KINDS = {"none": L.STEM_NORM_NONE, "rms": L.STEM_NORM_RMS, "layer": L.STEM_NORM_LAYER}
GATES = {"none": L.STEM_GATE_NONE, "channel": L.STEM_GATE_CHANNEL, "token": L.STEM_GATE_TOKEN, "full": L.STEM_GATE_FULL}


def make_ctx(dtype, T, d):
    return L.stem_create(d, 64, 100, L.STEM_F32 if dtype == "f32" else L.STEM_BF16, T)


def draw(dtype, seed, *shape, std=1.0, mean=0.0):
    gen = torch.Generator().manual_seed(seed)
    t = torch.randn(*shape, generator=gen) * std + mean
    return t.to(torch.float32 if dtype == "f32" else torch.bfloat16).to(DEV)


def empty_like(t, dtype=None):
    return torch.full_like(t, float("nan"), dtype=dtype or t.dtype)


def num(t):
    return None if t is None else t.double().cpu().numpy()


# every width's kernel (each of the nine shapes at its edges), token counts of one and more, every norm
ENTER = [("bf16", 1, 64, "rms"), ("bf16", 3, 128, "layer"), ("bf16", 515, 64, "rms"), ("bf16", 65, 192, "rms"), ("bf16", 1030, 512, "layer"),
         ("bf16", 2, 576, "rms"), ("bf16", 77, 1024, "rms"), ("bf16", 700, 2048, "rms"), ("bf16", 19, 2112, "layer"), ("bf16", 5, 4096, "rms"),
         ("bf16", 9, 4160, "layer"), ("bf16", 3, 8192, "rms"), ("bf16", 2, 16384, "layer"), ("f32", 1, 4, "rms"), ("f32", 33, 12, "layer"),
         ("f32", 257, 68, "rms"), ("f32", 100, 260, "layer"), ("f32", 31, 516, "rms"), ("f32", 63, 1004, "layer"), ("f32", 7, 1028, "rms"),
         ("f32", 5, 3004, "rms"), ("f32", 3, 8196, "layer")]


@pytest.mark.parametrize("dtype,T,d,kind", ENTER)
def test_enter(dtype, T, d, kind):
    ctx = make_ctx(dtype, T, d)
    x, w = draw(dtype, 1, T, d, std=2.0, mean=0.5), draw(dtype, 2, d, std=0.3, mean=1.0)
    dn, dres = draw(dtype, 3, T, d), draw(dtype, 4, T, d)
    norm = L.stem_norm(KINDS[kind], 1e-5, w)
    n, dx, dw = empty_like(x), empty_like(x), empty_like(w, torch.float32)
    L.stem_block_enter_forward(ctx, x, norm, n)
    L.stem_block_enter_backward(ctx, dn, x, norm, dx, dw, dres=dres)
    X, W, DN = num(x), num(w), num(dn)
    unit = B.norm(X, kind, 1e-5)[0]
    assert max_rel(num(n), unit * W) <= TOL[dtype]
    assert max_rel(num(dx), num(dres) + B.norm_back(DN * W, X, kind, 1e-5)) <= TOL[dtype]
    assert max_rel(num(dw), (DN * unit).sum(0)) <= F32_TOL
    # added to, without a residual gradient, and in place
    again = dx.clone()
    L.stem_block_enter_backward(ctx, dn, x, norm, again, dw, accumulate=True)
    assert max_rel(num(dw), 2 * (DN * unit).sum(0)) <= 2 * F32_TOL
    assert max_rel(num(again), B.norm_back(DN * W, X, kind, 1e-5)) <= TOL[dtype]
    L.stem_block_enter_backward(ctx, dn, x, L.stem_norm(KINDS[kind], 1e-5), dn, dw)     # no weight; dx over dn
    assert max_rel(num(dn), B.norm_back(DN, X, kind, 1e-5)) <= TOL[dtype]
    L.stem_block_enter_forward(ctx, x, norm, x)
    assert torch.equal(x, n)


LEAVE = [  # dtype, T, d, out, next, gate, p
    ("bf16", 1, 64, "rms", "rms", "channel", 0.0), ("bf16", 3, 2048, "rms", "rms", "channel", 0.1), ("bf16", 1100, 2048, "rms", "layer", "channel", 0.1),
    ("bf16", 700, 1024, "layer", "rms", "token", 0.25), ("bf16", 33, 512, "none", "rms", "full", 0.5), ("bf16", 129, 4096, "rms", "none", "none", 0.1),
    ("bf16", 17, 320, "layer", "layer", "full", 0.0), ("bf16", 5, 8192, "rms", "rms", "token", 0.1), ("bf16", 2, 16384, "rms", "rms", "channel", 0.1),
    ("bf16", 257, 128, "none", "none", "none", 0.0), ("bf16", 600, 64, "rms", "rms", "channel", 0.1), ("f32", 1, 4, "layer", "rms", "token", 0.0),
    ("f32", 50, 20, "rms", "layer", "full", 0.1), ("f32", 1537, 260, "layer", "layer", "full", 0.1), ("f32", 600, 100, "rms", "rms", "channel", 0.9),
    ("f32", 70, 1004, "none", "layer", "channel", 0.1), ("f32", 9, 2052, "rms", "rms", "none", 0.25), ("f32", 40, 4000, "layer", "none", "token", 0.1),
    ("f32", 4, 8196, "rms", "rms", "channel", 0.1), ("f32", 30, 36, "rms", "rms", "token", 1.0)]


def leave_case(dtype, T, d, out, next, gate, p, seed=0x123456789ABCDEF, offset=1 << 33):
    f, x = draw(dtype, 11, T, d, std=0.7, mean=0.2), draw(dtype, 12, T, d, std=2.0)
    w_out = draw(dtype, 13, d, std=0.3, mean=1.0) if out != "none" else None
    w_next = draw(dtype, 14, d, std=0.3, mean=1.0) if next != "none" else None
    shape = {"none": None, "channel": (d,), "token": (T,), "full": (T, d)}[gate]
    g = draw(dtype, 15, *shape) if shape else None
    leave = L.stem_leave(out=L.stem_norm(KINDS[out], 1e-5, w_out), next=L.stem_norm(KINDS[next], 1e-5, w_next), residual_scale=0.75,
                         branch_scale=1.25, gate_kind=GATES[gate], gate=g, p=p, seed=seed, offset=offset)
    ref = dict(out=out, next=next, eps=1e-5, w_out=1.0 if w_out is None else num(w_out), w_next=1.0 if w_next is None else num(w_next), a=0.75,
               b=1.25, gate=gate, g=num(g), factor=B.drop_factor(T, d, p, seed, offset))
    return f, x, g, leave, ref


@pytest.mark.parametrize("dtype,T,d,out,next,gate,p", LEAVE)
def test_leave(dtype, T, d, out, next, gate, p):
    ctx = make_ctx(dtype, T, d)
    f, x, g, leave, ref = leave_case(dtype, T, d, out, next, gate, p)
    y, n = empty_like(x), empty_like(x) if next != "none" else None
    L.stem_block_leave_forward(ctx, f, x, leave, y, n)
    wy, wn = B.leave_forward(num(f), num(x), **ref)
    assert max_rel(num(y), wy) <= TOL[dtype]
    if n is not None:
        assert max_rel(num(n), wn) <= TOL[dtype]
    dy, dn = draw(dtype, 16, T, d), draw(dtype, 17, T, d) if next != "none" else None
    f32 = torch.float32
    dx, df = empty_like(x), empty_like(x)
    dg = None if g is None else empty_like(g, f32 if gate == "channel" else g.dtype)
    dwo = torch.full((d,), float("nan"), device=DEV) if out != "none" else None
    dwn = torch.full((d,), float("nan"), device=DEV) if next != "none" else None
    L.stem_block_leave_backward(ctx, dy, dn, f, y, leave, dx, df, dg, dwo, dwn)
    want = B.leave_backward(num(dy), num(dn), num(f), num(y), **ref)
    assert max_rel(num(dx), want["dx"]) <= TOL[dtype]
    assert max_rel(num(df), want["df"]) <= TOL[dtype]
    if dg is not None:
        assert max_rel(num(dg), want["dgate"]) <= (F32_TOL if gate == "channel" else TOL[dtype])
    if dwo is not None:
        assert max_rel(num(dwo), want["dw_out"]) <= F32_TOL
    if dwn is not None:
        assert max_rel(num(dwn), want["dw_next"]) <= F32_TOL
    # the same bits again, added to what is there, and with the outputs in the inputs' places
    sums = [t.clone() if t is not None else None for t in (dg if gate == "channel" else None, dwo, dwn)]
    L.stem_block_leave_backward(ctx, dy, dn, f, y, leave, dy, f, dg, dwo, dwn, accumulate=True)
    assert torch.equal(dy, dx) and torch.equal(f, df)
    for got, one in zip((dg, dwo, dwn), sums):
        assert one is None or torch.equal(got, one + one)
    L.stem_block_leave_forward(ctx, *leave_case(dtype, T, d, out, next, gate, p)[:1], x, leave, x, n)
    assert torch.equal(x, y)


# a workgroup takes several rows, of which each lane has two vectors
@pytest.mark.parametrize("dtype,T,d,out,next,gate,p", [("bf16", 600, 8256, "rms", "layer", "channel", 0.1), ("f32", 530, 9004, "layer", "rms", "token", 0.1),
                                                       ("bf16", 300, 16384, "none", "rms", "full", 0.0), ("f32", 257, 16384, "rms", "none", "channel", 0.0),
                                                       ("bf16", 700, 8192, "rms", "rms", "channel", 0.1)])
def test_leave_of_many_wide_rows(dtype, T, d, out, next, gate, p):
    test_leave(dtype, T, d, out, next, gate, p)


@pytest.mark.parametrize("dtype,T,d", [("bf16", 300, 12032), ("f32", 515, 9004), ("bf16", 515, 8192)])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_enter_of_many_wide_rows(dtype, T, d, kind):
    test_enter(dtype, T, d, kind)


@pytest.mark.parametrize("dtype,T,d", [("bf16", 16500, 2048), ("bf16", 33000, 1088), ("f32", 8300, 2044)])
def test_leave_forward_of_64_mib(dtype, T, d):
    ctx = make_ctx(dtype, T, d)
    f, x, g, leave, ref = leave_case(dtype, T, d, "rms", "layer", "channel", 0.1)
    y, n = empty_like(x), empty_like(x)
    L.stem_block_leave_forward(ctx, f, x, leave, y, n)
    for rows in (slice(0, 40), slice(T // 2, T // 2 + 40), slice(T - 40, T)):
        wy, wn = B.leave_forward(num(f[rows]), num(x[rows]), **dict(ref, factor=ref["factor"][rows]))
        assert max_rel(num(y[rows]), wy) <= TOL[dtype] and max_rel(num(n[rows]), wn) <= TOL[dtype]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_leave_with_one_gradient_or_few_outputs(dtype):
    T, d = 37, 192
    ctx = make_ctx(dtype, T, d)
    f, x, g, leave, ref = leave_case(dtype, T, d, "rms", "layer", "channel", 0.1)
    y, n = empty_like(x), empty_like(x)
    L.stem_block_leave_forward(ctx, f, x, leave, y, n)
    dy, dn = draw(dtype, 16, T, d), draw(dtype, 17, T, d)
    for a, b in ((dy, None), (None, dn)):
        dx, df = empty_like(x), empty_like(x)
        L.stem_block_leave_backward(ctx, a, b, f, y, leave, dx, df)
        want = B.leave_backward(num(a), num(b), num(f), num(y), **ref)
        assert max_rel(num(dx), want["dx"]) <= TOL[dtype] and max_rel(num(df), want["df"]) <= TOL[dtype]
    dg = torch.full((d,), float("nan"), device=DEV)
    L.stem_block_leave_backward(ctx, dy, dn, f, y, leave, None, None, dg)
    assert max_rel(num(dg), B.leave_backward(num(dy), num(dn), num(f), num(y), **ref)["dgate"]) <= F32_TOL


def test_layer_norm_of_a_large_mean():
    """A mean of 1000 deviations: the variance is of centred values, so it keeps its digits."""
    T, d = 5, 1024
    ctx = make_ctx("f32", T, d)
    x = draw("f32", 5, T, d) + 1000.0
    n = empty_like(x)
    L.stem_block_enter_forward(ctx, x, L.stem_norm(L.STEM_NORM_LAYER, 1e-6), n)
    # the mean is off by 1000 * 6e-8 * a few, against deviations of 1
    assert max_rel(num(n), B.norm(num(x), "layer", 1e-6)[0]) <= 1e-3 * 0.5


def test_rows_of_zeros_infinities_and_nan_stay_by_themselves():
    T, d = 9, 128
    ctx = make_ctx("bf16", T, d)
    x = draw("bf16", 6, T, d)
    clean = x.clone()
    x[2], x[4, 7], x[6, 100] = 0, float("inf"), float("nan")
    n, m = empty_like(x), empty_like(x)
    norm = L.stem_norm(L.STEM_NORM_RMS, 1e-6)
    L.stem_block_enter_forward(ctx, x, norm, n)
    L.stem_block_enter_forward(ctx, clean, norm, m)
    rest = [0, 1, 3, 5, 7, 8]
    assert torch.equal(n[rest], m[rest])
    assert (n[2] == 0).all() and torch.isnan(n[6]).all() and torch.isnan(n[4, 7])
    # a dropped NaN is 0
    leave = L.stem_leave(p=1.0)
    y = empty_like(x)
    L.stem_block_leave_forward(ctx, x, clean, leave, y)
    assert torch.equal(y, clean)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(1, 1), (1, 7), (3, 8), (5, 9), (300, 1), (999, 1001), (64, 4096), (2, 8191), (17, 24), (65, 333)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
def test_dropout(dtype, T, d, p):
    ctx = make_ctx(dtype, T, 64)
    x = draw(dtype, 8, T, d)
    y = empty_like(x)
    L.stem_dropout(ctx, x, y, p, seed=2 ** 64 - 3, offset=2 ** 40 + 1)
    want = num(x) * B.drop_factor(T, d, p, 2 ** 64 - 3, 2 ** 40 + 1)
    assert ((num(y) == 0) == (want == 0)).all()
    assert max_rel(num(y), want) <= TOL[dtype]
    L.stem_dropout(ctx, x, x, p, seed=2 ** 64 - 3, offset=2 ** 40 + 1)
    assert torch.equal(x, y)


def test_dropout_of_a_large_tensor_and_the_block_draw_the_same_mask():
    T, d = 300, 2048
    ctx = make_ctx("f32", T, d)
    ones = torch.ones(T, d, device=DEV)
    y, z = empty_like(ones), empty_like(ones)
    L.stem_dropout(ctx, ones, y, 0.3, seed=5, offset=6)
    L.stem_block_leave_forward(ctx, ones, ones, L.stem_leave(residual_scale=0.0, p=0.3, seed=5, offset=6), z)
    assert torch.equal(y, z)


def test_masks_count_on_in_a_graph():
    """A captured call with a device step draws another mask on every replay, the one of an eager call with that offset."""
    T, d = 40, 256
    ctx = make_ctx("bf16", T, d)
    x, f = draw("bf16", 1, T, d), draw("bf16", 2, T, d)
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    leave = L.stem_leave(out=L.stem_norm(L.STEM_NORM_RMS, 1e-5), p=0.2, seed=9, offset=100, step=step)
    y, z = empty_like(x), empty_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        L.stem_block_leave_forward(ctx, f, x, leave, y)
        L.stem_dropout(ctx, x, z, 0.2, 9, 100, step=step)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        L.stem_block_leave_forward(ctx, f, x, leave, y)
        L.stem_dropout(ctx, x, z, 0.2, 9, 100, step=step)
    seen = []
    for k in range(4):
        step.fill_(k)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager, ez = empty_like(x), empty_like(x)
        L.stem_block_leave_forward(ctx, f, x, L.stem_leave(out=leave.norms[0], p=0.2, seed=9, offset=100 + k), eager)
        L.stem_dropout(ctx, x, ez, 0.2, 9, 100 + k)
        torch.cuda.synchronize()
        assert torch.equal(y, eager) and torch.equal(z, ez)
        seen.append(z.clone())
    assert not torch.equal(seen[0], seen[1])


def test_block_calls_on_another_stream():
    T, d = 500, 1024
    ctx = make_ctx("bf16", T, d)
    f, x, g, leave, ref = leave_case("bf16", T, d, "rms", "rms", "channel", 0.1)
    y, n = empty_like(x), empty_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        L.stem_block_leave_forward(ctx, f, x, leave, y, n)
    s.synchronize()
    wy, wn = B.leave_forward(num(f), num(x), **ref)
    assert max_rel(num(y), wy) <= TOL["bf16"] and max_rel(num(n), wn) <= TOL["bf16"]


def test_refusals():
    T, d = 8, 64
    ctx = make_ctx("bf16", T, d)
    x, y = draw("bf16", 1, T, d), draw("bf16", 2, T, d)
    w = draw("bf16", 3, d)

    def status(call, *a, **k):
        with pytest.raises(L.StemError) as e:
            call(*a, **k)
        return e.value.status

    rms = L.stem_norm(L.STEM_NORM_RMS, 1e-5, w)
    bad = L.STEM_ERR_INVALID_ARG
    assert status(L.stem_block_enter_forward, ctx, x, L.stem_norm(), y) == bad                       # no norm
    assert status(L.stem_block_enter_forward, ctx, x, L.stem_norm(7, 1e-5), y) == bad
    for eps in (-1.0, float("nan"), float("inf")):
        assert status(L.stem_block_enter_forward, ctx, x, L.stem_norm(1, eps), y) == bad
    assert status(L.stem_block_enter_forward, ctx, x, rms, None) == bad
    both = torch.empty(T * d + 64, dtype=torch.bfloat16, device=DEV)
    assert status(L.stem_block_enter_forward, ctx, both[:T * d].view(T, d), rms, both[64:].view(T, d)) == bad   # half over it
    assert status(L.stem_block_leave_forward, ctx, x, y, L.stem_leave(next=rms), x, None) == bad     # n belongs to the next norm
    assert status(L.stem_block_leave_forward, ctx, x, y, L.stem_leave(), x, y) == bad
    assert status(L.stem_block_leave_forward, ctx, x, y, L.stem_leave(gate_kind=L.STEM_GATE_CHANNEL), x) == bad
    assert status(L.stem_block_leave_forward, ctx, x, y, L.stem_leave(gate_kind=9, gate=w), x) == bad
    for p in (-0.1, 1.1, float("nan")):
        assert status(L.stem_block_leave_forward, ctx, x, y, L.stem_leave(p=p), x) == bad
        assert status(L.stem_dropout, ctx, x, y, p, 1) == bad
    assert status(L.stem_block_leave_forward, ctx, x, y, L.stem_leave(next=rms), x, x) == bad        # both outputs in one place
    dw = torch.zeros(d, device=DEV)
    assert status(L.stem_block_leave_backward, ctx, x, None, y, None, L.stem_leave(next=rms), None, None, None, None, dw) == bad
    assert status(L.stem_block_leave_backward, ctx, x, y, y, None, L.stem_leave(next=rms), None, None) == bad
    assert status(L.stem_block_leave_backward, ctx, x, None, None, None, L.stem_leave(out=rms), None, y) == bad
    assert status(L.stem_block_leave_backward, ctx, x, None, y, None, L.stem_leave(), None, None, y) == bad
    big = draw("bf16", 1, T + 1, d)
    assert status(L.stem_block_enter_forward, ctx, big, rms, empty_like(big)) == L.STEM_ERR_SHAPE
    for call in (lambda: L.stem_block_enter_forward(ctx, x.float(), rms, y), lambda: L.stem_block_enter_forward(ctx, x.cpu(), rms, y),
                 lambda: L.stem_block_enter_forward(ctx, x, rms, y[:3]), lambda: L.stem_block_enter_forward(ctx, x, L.stem_norm(1, 1e-5, w[:32]), y),
                 lambda: L.stem_block_enter_forward(ctx, x.t(), rms, y), lambda: L.stem_dropout(ctx, x, y[:, :32], 0.1, 1)):
        with pytest.raises((TypeError, ValueError)):
            call()
    none = draw("bf16", 1, 0, d)
    L.stem_block_enter_forward(ctx, none, rms, none)
    L.stem_dropout(ctx, none, none, 0.1, 1)
    wide = L.stem_create(16448, 64, 10, L.STEM_BF16, 2)
    t = draw("bf16", 1, 2, 16448)
    assert status(L.stem_block_enter_forward, wide, t, L.stem_norm(1, 1e-5), empty_like(t)) == L.STEM_ERR_UNSUPPORTED
