"""Norm and rotation of queries and keys in 64 bits, forwards and backwards, with the size of the terms that errors are
measured by. Test infrastructure only."""
import numpy as np


def fractions(theta):
    """Turns of one position as 64-bit fractions, uint64."""
    return np.array([round(float(t) / (2 * np.pi) * 2.0 ** 64) % (1 << 64) for t in theta], np.uint64)


def angles(pos, freq):
    """[T, rot / 2] in radians: the product of whole numbers wraps at a turn."""
    with np.errstate(over="ignore"):
        turn = np.asarray(pos, np.int64).astype(np.uint64)[:, None] * freq[None]
    return turn.astype(np.int64).astype(np.float64) * (2 * np.pi / 2.0 ** 64)


def members(rot, interleaved):
    half = rot // 2
    return (np.arange(0, rot, 2), np.arange(1, rot, 2)) if interleaved else (np.arange(half), np.arange(half, rot))


def turned(x, angle, rot, interleaved, scale, back=False):
    """x [T, heads, D] rotated, and |a| + |b| of each pair (times scale)."""
    y, size = x.copy(), np.abs(x)
    i, j = members(rot, interleaved)
    c, s = (scale * f(angle)[:, None] for f in (np.cos, np.sin))
    a, b = x[..., i], x[..., j]
    s = -s if back else s
    y[..., i], y[..., j] = a * c - b * s, b * c + a * s
    size[..., i] = size[..., j] = (np.abs(a) + np.abs(b)) * abs(scale)
    return y, size


def forward(x, w, eps, angle, rot, interleaved, scale):
    n = x if w is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    return turned(n, angle, rot, interleaved, scale)


def backward(x, w, eps, gy, angle, rot, interleaved, scale):
    """gx, its error scale, gw, its error scale."""
    g, size = turned(gy, angle, rot, interleaved, scale, back=True)
    if w is None:
        return g, size, None, None
    D = x.shape[-1]
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    h = x * r
    u = g * w
    gx = r * (u - h * (u * h).mean(-1, keepdims=True))
    su = size * np.abs(w)
    sx = r * (su + np.abs(h) * (su * np.abs(h)).sum(-1, keepdims=True) / D)
    return gx, sx, (g * h).sum((0, 1)), (size * np.abs(h)).sum((0, 1))
