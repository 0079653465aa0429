"""The block's calls at the edges of their range: no tokens, gates that are no numbers where an element is dropped, tensors that get other memory."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as B
from paper_2601_10639_amd import stemlib as L
from tests import test_gpu_block as M

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make_ctx(dtype, T, d):
    return L.stem_create(d, 64, 100, L.STEM_F32 if dtype == "f32" else L.STEM_BF16, T)


def draw(dtype, seed, *shape):
    t = torch.randn(*shape, generator=torch.Generator().manual_seed(seed))
    return t.to(torch.float32 if dtype == "f32" else torch.bfloat16).to(DEV)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sums_over_no_tokens_are_zero(dtype):
    d = 192
    ctx = make_ctx(dtype, 4, d)
    none, w = draw(dtype, 1, 0, d), draw(dtype, 2, d)
    norm = L.stem_norm(L.STEM_NORM_RMS, 1e-5, w)
    leave = L.stem_leave(out=norm, next=norm, gate_kind=L.STEM_GATE_CHANNEL, gate=draw(dtype, 3, d), p=0.1)
    sums = [torch.full((d,), float("nan"), device=DEV) for _ in range(4)]

    def backward(accumulate):
        L.stem_block_enter_backward(ctx, none, none, norm, none, sums[0], accumulate=accumulate)
        L.stem_block_leave_backward(ctx, none, none, none, none, leave, none, none, *sums[1:], accumulate=accumulate)

    backward(False)
    assert all((s == 0).all() for s in sums)
    for s in sums:
        s.fill_(3.0)
    backward(True)
    assert all((s == 3).all() for s in sums)
    # a gate's gradient for each token or element has no element; sums that are not asked for
    for kind, gate in ((L.STEM_GATE_TOKEN, none[:, 0].contiguous()), (L.STEM_GATE_FULL, none)):
        L.stem_block_leave_backward(ctx, none, none, none, none, L.stem_leave(next=norm, gate_kind=kind, gate=gate), None, None, gate)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("where,out", [("full", "none"), ("full", "rms"), ("channel", "none"), ("channel", "layer"), ("token", "none"), ("w_out", "rms")])
def test_what_is_dropped_counts_for_nothing(dtype, where, out):
    """An infinity or a NaN in the gate or the norm's weight reaches nothing where the element that it multiplies is dropped."""
    T, d, p, seed, offset = 40, 192, 0.3, 5, 6
    ctx = make_ctx(dtype, T, d)
    dropped = torch.from_numpy(B.drop_factor(T, d, p, seed, offset) == 0).to(DEV)
    f, x, dy = draw(dtype, 1, T, d), draw(dtype, 2, T, d), draw(dtype, 3, T, d)
    kind = {"none": L.STEM_NORM_NONE, "rms": L.STEM_NORM_RMS, "layer": L.STEM_NORM_LAYER}[out]
    gate_kind, shape = {"full": (L.STEM_GATE_FULL, (T, d)), "channel": (L.STEM_GATE_CHANNEL, (d,)), "token": (L.STEM_GATE_TOKEN, (T,)),
                        "w_out": (L.STEM_GATE_TOKEN, (T,))}[where]
    w, g = draw(dtype, 4, d), draw(dtype, 5, *shape)
    wild, wild_f = (w if where == "w_out" else g).clone(), f.clone()
    if where == "full":
        wild[dropped] = float("inf")
        wild[0][dropped[0]] = float("nan")
        same = torch.ones_like(dropped)
    elif where == "token":
        wild[::2] = float("inf")
        same = dropped.clone()
        same[1::2] = True
    else:
        wild[7], wild[100] = float("inf"), float("nan")
        same = (dropped[:, [7, 100]].all(1, keepdim=True)).expand(T, d).clone()   # rows that neither reaches
        assert same[:, 0].sum() > 0
    if out == "none":
        wild_f[dropped] = float("nan")

    def run(f, w, g):
        norm = L.stem_norm(kind, 1e-5, w if out != "none" else None)
        leave = L.stem_leave(out=norm, gate_kind=gate_kind, gate=g, p=p, seed=seed, offset=offset)
        y, dx, df = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
        dg, dw = torch.empty_like(g, dtype=torch.float32 if where == "channel" else g.dtype), torch.empty(d, device=DEV)
        L.stem_block_leave_forward(ctx, f, x, leave, y)
        L.stem_block_leave_backward(ctx, dy, None, f, None, leave, dx, df, dg, dw)
        return y, dx, df, dg, dw

    clean = run(f, w, g)
    got = run(wild_f, wild if where == "w_out" else w, g if where == "w_out" else wild)
    for a, b in zip(clean[:3], got[:3]):
        assert torch.equal(a[same], b[same])
    assert (got[2][dropped & same] == 0).all() or out != "none"
    if where == "full":
        assert torch.equal(clean[3], got[3]) and (got[3][dropped] == 0).all() and torch.equal(clean[4], got[4])
    elif where == "w_out":
        rows = same[:, 0]
        assert torch.equal(clean[3][rows], got[3][rows])
    else:
        assert torch.equal(clean[3], got[3])      # (a gate's own gradient does not hold the gate)


@pytest.mark.parametrize("way", ["native", "python"])
def test_tensors_that_get_other_memory(way, monkeypatch):
    """A norm, a gate and a step are read where their tensors are when a call is made."""
    if way == "python":
        monkeypatch.setattr(L, "_bind", L._NoBind())
    T, d = 5, 128
    ctx = make_ctx("bf16", T, d)
    f, x = draw("bf16", 1, T, d), draw("bf16", 2, T, d)
    w_out, w_next, gate, step = draw("bf16", 3, d), draw("bf16", 4, d), draw("bf16", 5, d), torch.zeros(1, dtype=torch.int64, device=DEV)
    held = [t.data for t in (w_out, w_next, gate, step)]      # (the memory of before stays allocated)

    def parts():
        norm = L.stem_norm(L.STEM_NORM_RMS, 1e-5, w_next)
        return norm, L.stem_leave(out=L.stem_norm(L.STEM_NORM_RMS, 1e-5, w_out), next=norm, gate_kind=L.STEM_GATE_CHANNEL, gate=gate, p=0.5, seed=1, step=step)

    def run(norm, leave):
        m, y, n, dx, df = (torch.empty_like(x) for _ in range(5))
        sums = [torch.empty(d, device=DEV) for _ in range(3)]
        L.stem_block_enter_forward(ctx, x, norm, m)
        L.stem_block_leave_forward(ctx, f, x, leave, y, n)
        L.stem_block_leave_backward(ctx, x, f, f, y, leave, dx, df, *sums)
        return [m, y, n, dx, df, *sums]

    early = parts()
    before = run(*early)
    w_out.data, w_next.data, gate.data = draw("bf16", 13, d), draw("bf16", 14, d), draw("bf16", 15, d)
    step.data = torch.full((1,), 3, dtype=torch.int64, device=DEV)
    after, want = run(*early), run(*parts())
    assert all(torch.equal(a, b) for a, b in zip(after, want))
    assert not any(torch.equal(a, b) for a, b in zip(before, want))
    # other norms and another dropout in a structure's places
    norm, leave = parts()
    leave.drop = L.stem_drop(0.25, 7, 8, step=step)
    leave.out = L.stem_norm(L.STEM_NORM_LAYER, 1e-5, held[0])
    leave.next = L.stem_norm(L.STEM_NORM_LAYER, 1e-5, held[1])
    want = L.stem_leave(out=L.stem_norm(L.STEM_NORM_LAYER, 1e-5, held[0]), next=L.stem_norm(L.STEM_NORM_LAYER, 1e-5, held[1]),
                        gate_kind=L.STEM_GATE_CHANNEL, gate=gate, p=0.25, seed=7, offset=8 + 3)
    assert all(torch.equal(a, b) for a, b in zip(run(norm, leave), run(norm, want)))
    # a weight that is not of one row any more
    w_out.data = draw("bf16", 3, d + 1)
    with pytest.raises(ValueError):
        run(*early)
    assert len(held) == 4


def refused(call, *a, **k):
    with pytest.raises(L.StemError) as e:
        call(*a, **k)
    assert e.value.status == L.STEM_ERR_INVALID_ARG


@pytest.mark.parametrize("at", [0, 16, 1024, 8192 - 256, 8192 - 16])
def test_a_sum_over_another_output_is_refused(at):
    T, d = 64, 64
    ctx = make_ctx("bf16", T, d)
    x, dn, w = draw("bf16", 1, T, d), draw("bf16", 2, T, d), draw("bf16", 3, d)
    memory = torch.zeros(T * d * 2 + 256, dtype=torch.uint8, device=DEV)
    dx, dw = memory[:T * d * 2].view(torch.bfloat16).view(T, d), memory[at:at + 4 * d].view(torch.float32)
    norm = L.stem_norm(L.STEM_NORM_RMS, 1e-5, w)
    refused(L.stem_block_enter_backward, ctx, dn, x, norm, dx, dw)
    leave = L.stem_leave(out=norm, next=norm, gate_kind=L.STEM_GATE_CHANNEL, gate=w)
    for k in range(3):
        sums = [None] * 3
        sums[k] = dw
        refused(L.stem_block_leave_backward, ctx, x, dn, x, x, leave, dx, None, *sums)
        refused(L.stem_block_leave_backward, ctx, x, dn, x, x, leave, None, dx, *sums)
    torch.cuda.synchronize()
    assert (memory == 0).all()


def test_an_output_over_a_weight_is_refused():
    d = 64
    ctx = make_ctx("bf16", 1, d)
    x, w = draw("bf16", 1, 1, d), draw("bf16", 2, d)
    norm, over = L.stem_norm(L.STEM_NORM_RMS, 1e-5, w), w.view(1, d)
    refused(L.stem_block_enter_forward, ctx, x, norm, over)
    refused(L.stem_block_enter_backward, ctx, x, x, norm, over)
    refused(L.stem_block_leave_forward, ctx, x, x, L.stem_leave(out=norm), over)
    refused(L.stem_block_leave_backward, ctx, x, None, x, None, L.stem_leave(out=norm), over, None)


@pytest.mark.parametrize("at", [0, 8, 64])
def test_an_output_over_the_step_is_refused(at):
    T, d = 4, 64
    ctx = make_ctx("bf16", T, d)
    x, w = draw("bf16", 1, T, d), draw("bf16", 2, d)
    memory = torch.zeros(T * d * 2, dtype=torch.uint8, device=DEV)
    y, step = memory.view(torch.bfloat16).view(T, d), memory[at:at + 8].view(torch.int64)
    norm = L.stem_norm(L.STEM_NORM_RMS, 1e-5, w)
    leave = L.stem_leave(out=norm, next=norm, gate_kind=L.STEM_GATE_CHANNEL, gate=w, p=0.1, seed=1, step=step)
    refused(L.stem_dropout, ctx, x, y, 0.1, 1, step=step)
    refused(L.stem_block_leave_forward, ctx, x, x, leave, y, torch.empty_like(x))
    refused(L.stem_block_leave_forward, ctx, x, x, leave, torch.empty_like(x), y)
    refused(L.stem_block_leave_backward, ctx, x, x, x, x, leave, y, None)
    refused(L.stem_block_leave_backward, ctx, x, x, x, x, leave, None, y)
    for k in range(3):
        sums = [None] * 3
        sums[k] = memory[:4 * d].view(torch.float32)
        refused(L.stem_block_leave_backward, ctx, x, x, x, x, leave, None, None, *sums)
    torch.cuda.synchronize()
    assert (memory == 0).all()


@pytest.mark.parametrize("n", [0, 2])
def test_a_step_of_another_size_is_refused(n):
    """A counter of no elements has no address, which would be none at all: the same mask in every replay."""
    T, d = 4, 64
    ctx = make_ctx("bf16", T, d)
    x, step = draw("bf16", 1, T, d), torch.zeros(n, dtype=torch.int64, device=DEV)
    with pytest.raises(ValueError):
        L.stem_dropout(ctx, x, torch.empty_like(x), 0.1, 1, step=step)
    one = torch.zeros(1, dtype=torch.int64, device=DEV)
    leave = L.stem_leave(p=0.1, step=one)
    one.data = step
    with pytest.raises(ValueError):
        L.stem_block_leave_forward(ctx, x, x, leave, torch.empty_like(x))


def test_dropout_of_more_than_a_launch_holds():
    """More than 2^32 threads: rows of 2056 take 512 each."""
    T, d, p, seed, offset = (1 << 23) + 9, 2056, 0.25, 11, 12
    ctx = make_ctx("bf16", T, 64)
    x = torch.ones(T, d, dtype=torch.bfloat16, device=DEV)
    L.stem_dropout(ctx, x, x, p, seed, offset)
    rows = [0, 1, (1 << 22) - 1, 1 << 22, (1 << 22) + 1, (1 << 23) - 1, 1 << 23, T - 1]
    c = np.zeros((len(rows), d // 8, 4), np.uint64)
    c[..., 0], c[..., 1], c[..., 2] = np.arange(d // 8), np.array(rows)[:, None], offset
    words = B.philox(c, (seed, 0))
    bits = np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], -1).reshape(len(rows), d)
    want = torch.from_numpy(np.where(bits >= 16384, 4.0 / 3.0, 0.0)).to(torch.bfloat16)
    assert torch.equal(x[rows].cpu(), want)
    del x
    torch.cuda.empty_cache()


# 385 to 512 workgroups of the backward pass take two rows, or two sets of rows, in turn: at both ends, one more, and an odd number of them
@pytest.mark.parametrize("dtype,T,d", [("bf16", 769, 2048), ("bf16", 801, 2048), ("bf16", 1024, 2048), ("bf16", 1025, 2048), ("bf16", 385, 4096), ("bf16", 511, 2112), ("bf16", 401, 8192),
                                       ("f32", 770, 2044), ("f32", 1023, 1028), ("f32", 387, 4096), ("f32", 512, 2052), ("f32", 3201, 260), ("f32", 390, 5000)])
def test_rows_in_turn(dtype, T, d):
    M.test_leave(dtype, T, d, "rms", "layer", "channel", 0.1)
    M.test_leave(dtype, T, d, "layer", "rms", "token", 0.0)
    M.test_enter(dtype, T, d, "rms")


@pytest.mark.parametrize("dtype,T,d", [("bf16", 37, 192), ("f32", 700, 260), ("bf16", 300, 2048), ("bf16", 5, 8256)])
def test_outputs_in_the_place_of_any_input(dtype, T, d):
    """Every [T,d] output over every [T,d] input, against the same call with memory of its own for each."""
    ctx = make_ctx(dtype, T, d)
    (f, x, dy, dn, gate), w = (draw(dtype, s, T, d) for s in range(5)), draw(dtype, 9, d)
    norm = L.stem_norm(L.STEM_NORM_RMS, 1e-5, w)

    def leave(g):
        return L.stem_leave(out=norm, next=norm, residual_scale=0.5, branch_scale=2.0, gate_kind=L.STEM_GATE_FULL, gate=g, p=0.2, seed=3, offset=4)

    def forward(y_over=None, n_over=None):
        t = dict(f=f.clone(), x=x.clone(), gate=gate.clone())
        y, n = t.get(y_over, torch.empty_like(x)), t.get(n_over, torch.empty_like(x))
        L.stem_block_leave_forward(ctx, t["f"], t["x"], leave(t["gate"]), y, n)
        return y, n

    y, n = forward()
    for a in ("f", "x", "gate", None):
        for b in ("f", "x", "gate", None):
            if a != b or a is None:
                assert all(torch.equal(p, q) for p, q in zip((y, n), forward(a, b)))

    def backward(**over):
        t = dict(dy=dy.clone(), dn=dn.clone(), f=f.clone(), y=y.clone(), gate=gate.clone())
        out = [t.get(over.get(k), torch.empty_like(x)) for k in ("dx", "df", "dgate")]
        sums = [torch.empty(d, device=DEV) for _ in range(2)]
        L.stem_block_leave_backward(ctx, t["dy"], t["dn"], t["f"], t["y"], leave(t["gate"]), *out, *sums)
        return out + sums

    want = backward()
    inputs = ("dy", "dn", "f", "y", "gate")
    for i, a in enumerate(inputs):
        places = {"dx": a, "df": inputs[(i + 1) % 5], "dgate": inputs[(i + 2) % 5]}
        for one in [places, {"dx": inputs[(i + 2) % 5], "df": a, "dgate": inputs[(i + 1) % 5]}] + [{k: a} for k in places]:
            assert all(torch.equal(p, q) for p, q in zip(want, backward(**one)))

    def enter(over=None):
        t = dict(dn=dn.clone(), x=x.clone(), dres=dy.clone())
        dx, dw = t.get(over, torch.empty_like(x)), torch.empty(d, device=DEV)
        L.stem_block_enter_backward(ctx, t["dn"], t["x"], norm, dx, dw, dres=t["dres"])
        return dx, dw

    want = enter()
    for a in ("dn", "x", "dres"):
        assert all(torch.equal(p, q) for p, q in zip(want, enter(a)))
