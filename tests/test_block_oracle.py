"""Pins of the oracle of the block around the layer: differences, autograd, the generator's published answers, brute force."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as B


def test_philox_known_answers():
    # the answers that the generator's authors publish for the counters of all zeros, all ones, and the digits of pi
    zero = B.philox(np.zeros((1, 4), np.uint64), (0, 0))[0]
    assert [int(v) for v in zero] == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = B.philox(np.full((1, 4), 0xFFFFFFFF, np.uint64), (0xFFFFFFFF, 0xFFFFFFFF))[0]
    assert [int(v) for v in ones] == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    pi = B.philox(np.array([[0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344]], np.uint64), (0xA4093822, 0x299F31D0))[0]
    assert [int(v) for v in pi] == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_drop_factor_statistics():
    f = B.drop_factor(300, 1001, 0.1, 1234567890123, 5)
    kept = (f != 0).mean()
    assert abs(kept - 0.9) < 5 * np.sqrt(0.09 / f.size)
    assert np.allclose(f[f != 0], 65536 / (65536 - 6554))
    assert (B.drop_factor(3, 9, 1.0, 1, 2) == 0).all() and (B.drop_factor(3, 9, 0.0, 1, 2) == 1).all()
    assert (B.drop_factor(64, 64, 0.5, 1, 2) != B.drop_factor(64, 64, 0.5, 1, 3)).mean() > 0.4


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_norm_back_against_differences(kind):
    rng = np.random.default_rng(1)
    v, h = rng.normal(size=(2, 7)) + 0.5, rng.normal(size=(2, 7))
    got = B.norm_back(h, v, kind, 1e-3)
    e = 1e-6
    for i in np.ndindex(v.shape):
        a, b = v.copy(), v.copy()
        a[i] += e
        b[i] -= e
        assert abs(((B.norm(a, kind, 1e-3)[0] - B.norm(b, kind, 1e-3)[0]) * h).sum() / (2 * e) - got[i]) < 1e-8


@pytest.mark.parametrize("out,next,gate", [("rms", "layer", "channel"), ("layer", "rms", "token"), ("none", "rms", "full"), ("rms", "none", "none")])
def test_leave_backward_against_autograd(out, next, gate):
    rng = np.random.default_rng(2)
    T, d, eps = 5, 12, 1e-4
    g = {"none": None, "channel": rng.normal(size=d), "token": rng.normal(size=T), "full": rng.normal(size=(T, d))}[gate]
    f, x, dy, dn = (rng.normal(size=(T, d)) for _ in range(4))
    w_out, w_next = rng.normal(size=d), rng.normal(size=d)
    factor = B.drop_factor(T, d, 0.25, 77, 1)
    arg = dict(out=out, next=next, eps=eps, w_out=w_out, w_next=w_next, a=0.7, b=1.3, gate=gate, g=g, factor=factor)
    y, n = B.leave_forward(f, x, **arg)
    t = {k: torch.tensor(v, requires_grad=True) for k, v in dict(f=f, x=x, w_out=w_out, w_next=w_next).items()}
    tg = None if g is None else torch.tensor(g, requires_grad=True)

    def tnorm(v, kind):
        if kind == "layer":
            v = v - v.mean(-1, keepdim=True)
        return v if kind == "none" else v / (v.pow(2).mean(-1, keepdim=True) + eps).sqrt()

    ty = 0.7 * t["x"] + 1.3 * tnorm(t["f"], out) * t["w_out"] * torch.tensor(factor) * (1 if tg is None else tg[:, None] if gate == "token" else tg)
    loss = (ty * torch.tensor(dy)).sum()
    assert np.abs(ty.detach().numpy() - y).max() < 1e-12
    if next != "none":
        tn = tnorm(ty, next) * t["w_next"]
        assert np.abs(tn.detach().numpy() - n).max() < 1e-12
        loss = loss + (tn * torch.tensor(dn)).sum()
    loss.backward()
    r = B.leave_backward(dy, dn if next != "none" else None, f, y, **arg)
    for got, want in ((r["dx"], t["x"]), (r["df"], t["f"]), (r["dw_out"], t["w_out"])):
        assert np.abs(got - want.grad.numpy()).max() < 1e-12
    if next != "none":
        assert np.abs(r["dw_next"] - t["w_next"].grad.numpy()).max() < 1e-12
    if g is not None:
        assert np.abs(r["dgate"] - tg.grad.numpy()).max() < 1e-12


def test_quantise():
    v = np.array([[0.0, 0.0, 0.0], [127.0, -127.0, 0.5], [127.0, 1.5, -2.5], [np.inf, 1.0, 2.0], [1e-40, 0.0, -1e-40]], np.float32)
    q, s = B.quantise(v)
    assert q.tolist()[:4] == [[0, 0, 0], [127, -127, 0], [127, 2, -2], [0, 0, 0]]   # halves go to the even neighbour
    assert s[1] == 1 and np.isnan(s[3]) and s[0] == np.float32(2.0 ** -126)
    rng = np.random.default_rng(3)
    v, W = rng.normal(size=(9, 50)), rng.normal(size=(7, 50))
    # each value is off by half a step at most, so a product by this much
    (q, s), (p, t) = B.quantise(v), B.quantise(W)
    most = (np.abs(v) @ (np.ones_like(W) * t / 2).T + np.ones_like(v) * s / 2 @ np.abs(W).T + 50 * s * t.T / 4)
    assert (np.abs(B.quant_product(v, W) - v @ W.T) <= most * (1 + 1e-5)).all()
    rows = rng.normal(size=(9, 7))
    z = np.maximum(-50, v @ W.T)
    want = (z / (1 + np.exp(-z)) * rows) @ rng.normal(size=(7, 7)).T
    assert B.quant_ffn(v, W, np.eye(7), rows).shape == want.shape
