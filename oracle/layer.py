"""The training operators of a temporal attention layer in 64 bits, from their
definitions: rows by type, products with a type's weights, layer norm, and the
gradients of both.  Test infrastructure; the library never calls it."""
import numpy as np


def group_rows(types, num_types, ids=None):
    """(order, offsets, type of every row or -1)."""
    types = np.asarray(types, np.int64)
    if ids is None:
        t = types.copy()
    else:
        t = np.array([types[i] if 0 <= i < len(types) else -1 for i in ids], np.int64)
    t[(t < 0) | (t >= num_types)] = -1
    lists = [np.flatnonzero(t == g) for g in range(num_types)]
    offsets = np.cumsum([0] + [len(r) for r in lists])
    return np.concatenate(lists + [np.flatnonzero(t < 0)]).astype(np.int32), offsets.astype(np.int64), t


def linear(x, w, t, bias=None):
    y = np.zeros((len(x), w.shape[1]))
    for i, g in enumerate(t):
        if g >= 0:
            y[i] = w[g].astype(np.float64) @ x[i].astype(np.float64) + (0 if bias is None else bias[g])
    return y


def linear_backward(dy, x, w, t):
    dy, x, w = (np.asarray(a, np.float64) for a in (dy, x, w))
    dx, dw, db = np.zeros((len(dy), w.shape[2])), np.zeros_like(w), np.zeros(w.shape[:2])
    for g in range(len(w)):
        rows = np.flatnonzero(t == g)
        dx[rows] = dy[rows] @ w[g]
        dw[g] = dy[rows].T @ x[rows]
        db[g] = dy[rows].sum(0)
    return dx, dw, db


def layer_norm(h, weight=None, bias=None, eps=1e-5):
    """(y, mean, rstd, (h - mean) rstd)."""
    h = np.asarray(h, np.float64)
    mean = h.mean(1, keepdims=True)
    rstd = 1 / np.sqrt(np.square(h - mean).mean(1, keepdims=True) + eps)
    xh = (h - mean) * rstd
    return xh * (1 if weight is None else weight) + (0 if bias is None else bias), mean[:, 0], rstd[:, 0], xh


def layer_norm_backward(dy, h, weight=None, eps=1e-5):
    """(dx, dweight, dbias)."""
    dy = np.asarray(dy, np.float64)
    _, _, rstd, xh = layer_norm(h, eps=eps)
    g = dy * (1 if weight is None else np.asarray(weight, np.float64))
    dx = (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True)) * rstd[:, None]
    return dx, (dy * xh).sum(0), dy.sum(0)
