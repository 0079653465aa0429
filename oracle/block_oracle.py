"""CPU oracle, in 64 bits, of what stands around the layer: norms, dropout, gate and residual of a decoder block, and products in
8-bit integers.  Written from the definitions, sharing no code with the GPU path."""
from __future__ import annotations

import numpy as np

f64 = np.float64


def norm(v, kind: str, eps: float):
    """N(v) by rows, and 1 / sqrt(...)."""
    v = np.asarray(v, f64)
    if kind == "none":
        return v.copy(), np.ones(v.shape[:-1] + (1,))
    if kind == "layer":
        v = v - v.mean(-1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        r = 1.0 / np.sqrt((v ** 2).mean(-1, keepdims=True) + eps)
        return v * r, r


def norm_back(h, v, kind: str, eps: float):
    """Gradient of N's input v for the gradient h of its output: h's product with N's Jacobian."""
    h = np.asarray(h, f64)
    if kind == "none":
        return h
    n, r = norm(v, kind, eps)
    g = h - n * (h * n).mean(-1, keepdims=True)
    if kind == "layer":
        g = g - h.mean(-1, keepdims=True)
    return g * r


def philox(c, key):
    """Philox 4x32 with ten rounds: counters [..., 4] and a key of two words, as Python integers or arrays of uint64."""
    m, low = (0xD2511F53, 0xCD9E8D57), np.uint64(0xFFFFFFFF)
    x = [np.asarray(c[..., i], np.uint64) for i in range(4)]
    k = [int(key[0]), int(key[1])]
    for _ in range(10):
        p0, p1 = x[0] * np.uint64(m[0]), x[2] * np.uint64(m[1])
        x = [(p1 >> np.uint64(32)) ^ x[1] ^ np.uint64(k[0]), p1 & low, (p0 >> np.uint64(32)) ^ x[3] ^ np.uint64(k[1]), p0 & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(x, -1)


def drop_factor(T: int, d: int, p: float, seed: int, offset: int):
    """What each element is multiplied by: 0 or 65536 / (65536 - threshold)."""
    threshold = int(np.rint(np.float32(p).astype(f64) * 65536))
    blocks = -(-d // 8)
    c = np.empty((T, blocks, 4), np.uint64)
    c[..., 0] = np.arange(blocks)[None, :]
    c[..., 1] = np.arange(T)[:, None]
    c[..., 2], c[..., 3] = offset & 0xFFFFFFFF, offset >> 32 & 0xFFFFFFFF
    words = philox(c, (seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF))
    bits = np.empty((T, blocks, 8), np.uint64)
    bits[..., 0::2], bits[..., 1::2] = words & np.uint64(0xFFFF), words >> np.uint64(16)
    bits = bits.reshape(T, blocks * 8)[:, :d]
    return np.where(bits >= threshold, 65536.0 / max(1, 65536 - threshold), 0.0)


def _gate(g, kind):
    return 1.0 if kind == "none" else np.asarray(g, f64)[:, None] if kind == "token" else np.asarray(g, f64)


def leave_forward(f, x, *, out="none", next="none", eps=0.0, w_out=1.0, w_next=1.0, a=1.0, b=1.0, gate="none", g=None, factor=1.0):
    """(y, n)."""
    u = norm(f, out, eps)[0] * w_out
    y = a * np.asarray(x, f64) + b * _gate(g, gate) * np.where(factor == 0, 0.0, u * factor)
    return y, norm(y, next, eps)[0] * w_next if next != "none" else None


def leave_backward(dy, dn, f, y, *, out="none", next="none", eps=0.0, w_out=1.0, w_next=1.0, a=1.0, b=1.0, gate="none", g=None, factor=1.0):
    """dict of dx, df, dgate, dw_out, dw_next; y as it was kept."""
    G = np.zeros(np.shape(f)) if dy is None else np.asarray(dy, f64)
    r = {}
    if dn is not None:
        dn = np.asarray(dn, f64)
        G = G + norm_back(dn * w_next, y, next, eps)
        r["dw_next"] = (dn * norm(y, next, eps)[0]).sum(0)
    r["dx"] = a * G
    h, fn = b * G, norm(f, out, eps)[0]
    dg = h * np.where(factor == 0, 0.0, fn * w_out * factor)
    r["dgate"] = {"none": None, "channel": dg.sum(0), "token": dg.sum(1), "full": dg}[gate]
    du = h * _gate(g, gate) * factor
    r["dw_out"] = (du * fn).sum(0)
    r["df"] = norm_back(du * w_out, f, out, eps)
    return r


def quantise(v):
    """Integers and scales of rows, with the scale and the quotient in fp32 as they are defined (the integers of a bf16 row are exact)."""
    v = np.asarray(v, np.float32)
    with np.errstate(invalid="ignore", over="ignore"):
        top = np.abs(v).max(-1, keepdims=True)
        s = np.maximum(top / np.float32(127), np.float32(2.0 ** -126)).astype(np.float32)
        q = np.rint(v * (np.float32(1) / s))
    bad = ~np.isfinite(v).all(-1, keepdims=True)
    return np.where(bad, 0, q).astype(np.int32), np.where(bad, np.float32(np.nan), s)


def quant_product(v, W):
    """Q(v) Q(W)^T with exact sums."""
    (q, s), (p, t) = quantise(v), quantise(W)
    return (q.astype(f64) @ p.astype(f64).T) * s.astype(f64) * t.astype(f64).T


def quant_ffn(n, Wg, Wd, rows):
    """The layer on (normed) rows n with the gathered table rows; hidden values unrounded."""
    z = quant_product(n, Wg)
    return quant_product(z / (1.0 + np.exp(-z)) * np.asarray(rows, f64), Wd)
