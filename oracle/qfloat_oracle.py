"""Plain definitions of the products in 8-bit floating point, in 64 bits: numpy only, no code of the library's."""
import numpy as np


def exponent(top):
    """The least e with top <= 448 2^e, at least -126."""
    top = np.asarray(top, np.float64)
    e = np.full(top.shape, -126)
    for k in range(-126, 128):
        e = np.where(top > np.ldexp(448.0, e), k + 1, e)
    return np.maximum(e, -126)


def e4m3(v):
    """The nearest of the format's values (1 sign, 4 exponent, 3 fraction bits, bias 7), to even; beyond 448 (by half a step) none: NaN."""
    v = np.asarray(v, np.float64)
    with np.errstate(invalid="ignore"):
        _, e = np.frexp(v)
        step = np.ldexp(1.0, np.maximum(e - 4, -9))
        out = np.rint(v / step) * step
        return np.where(np.abs(out) <= 448.0, out, np.nan)


def magnitude(v, axis):
    v = np.abs(np.asarray(v, np.float64))
    return np.where(np.isfinite(v), v, 0.0).max(axis=axis, keepdims=True)


def _scaled(v, top):
    s = np.ldexp(1.0, exponent(top))
    return e4m3(v / s) * s


def blocks(v, axis):
    """Q in blocks of 128 along an axis."""
    v = np.asarray(v, np.float64)
    out = np.empty_like(v)
    for lo in range(0, v.shape[axis], 128):
        at = [slice(None)] * v.ndim
        at[axis] = slice(lo, lo + 128)
        out[tuple(at)] = _scaled(v[tuple(at)], magnitude(v[tuple(at)], axis))
    return out


def squares(W):
    """Q in blocks of 128 x 128."""
    W = np.asarray(W, np.float64)
    out = np.empty_like(W)
    for i in range(0, W.shape[0], 128):
        for j in range(0, W.shape[1], 128):
            part = W[i:i + 128, j:j + 128]
            out[i:i + 128, j:j + 128] = _scaled(part, magnitude(part, (0, 1)))
    return out


def bounds(offsets, T, groups):
    """First rows and ends of the groups: offsets as the nearest that don't descend and stay within the rows."""
    if offsets is None:
        return [(0, T)]
    at, out = min(max(offsets[0], 0), T), []
    for g in range(groups):
        end = max(at, min(max(offsets[g + 1], 0), T))
        out.append((at, end))
        at = end
    return out


def linear(x, W, offsets=None):
    """Q(x) Q(W_g)^T, and the sum of the products' magnitudes; NaN in rows of no group."""
    T, (G, N, _) = x.shape[0], W.shape
    y, size = np.full((T, N), np.nan), np.full((T, N), np.nan)
    q = blocks(x, 1)
    for g, (lo, hi) in enumerate(bounds(offsets, T, G)):
        w = squares(W[g])
        y[lo:hi], size[lo:hi] = q[lo:hi] @ w.T, np.abs(q[lo:hi]) @ np.abs(w).T
    return y, size


def linear_backward(dy, x, W, offsets=None):
    """(dx, its products' magnitudes), (dW, its); NaN in rows of no group."""
    T, (G, N, K) = x.shape[0], W.shape
    dx, sx = linear(dy, np.swapaxes(W, 1, 2), offsets)
    dW, sW = np.zeros((G, N, K)), np.zeros((G, N, K))
    for g, (lo, hi) in enumerate(bounds(offsets, T, G)):
        if hi > lo:
            a, b = np.asarray(dy[lo:hi], np.float64), np.asarray(x[lo:hi], np.float64)
            dW[g], sW[g] = a.T @ b, np.abs(a).T @ np.abs(b)
    return (dx, sx), (dW, sW)


def weight_gradient_quantised(dy, x, groups, offsets=None):
    """Q'(dy)^T Q'(x) over each group's rows, Q' in blocks of 128 of them, column by column; and its products' magnitudes."""
    shape = (groups, dy.shape[1], x.shape[1])
    dW, size = np.zeros(shape), np.zeros(shape)
    for g, (lo, hi) in enumerate(bounds(offsets, x.shape[0], groups)):
        if hi > lo:
            a, b = blocks(dy[lo:hi], 0), blocks(x[lo:hi], 0)
            dW[g], size[g] = a.T @ b, np.abs(a).T @ np.abs(b)
    return dW, size


def hidden(n, ids, Wg, E, offsets=None):
    z, _ = linear(n, Wg, offsets)
    with np.errstate(over="ignore"):
        return z / (1.0 + np.exp(-z)) * np.asarray(E, np.float64)[np.clip(ids, 0, len(E) - 1)]


def ffn(n, ids, Wg, Wd, E, offsets=None):
    """Q(SiLU(Q(n) Q(Wg)^T) * E[ids]) Q(Wd)^T."""
    return linear(hidden(n, ids, Wg, E, offsets), Wd, offsets)[0]
