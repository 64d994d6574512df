"""Plain definitions of the 8-bit operators (include/tgl.h), on host arrays.

The rounding of a set of numbers to bytes is float32 operations in a fixed
order, so it is done in float32 here too and bytes and steps are compared
exactly; everything else is float64.
"""
import numpy as np

TINY = np.float32(2.0 ** -100)


def round16(d):
    return (d + 15) // 16 * 16


def to_bf16(x):
    """float32 -> the nearest bfloat16 (ties to even), as float32."""
    x = np.ascontiguousarray(x, np.float32)
    b = x.view(np.uint32).astype(np.uint64)
    r = ((b + 0x7FFF + ((b >> 16) & 1)) >> 16 << 16).astype(np.uint32).view(np.float32)
    return np.where(np.isfinite(x), r, x).reshape(x.shape)


def step_of(x):
    """The float32 step of a set of numbers."""
    x = np.asarray(x, np.float32)
    a = np.float32(0) if x.size == 0 else np.abs(x).max()       # NaN if any is
    if not np.isfinite(a):
        return np.float32(np.nan)
    return np.float32(0) if a < TINY else np.float32(a * (np.float32(1) / np.float32(127)))


def to_bytes(x, step):
    """Numbers in units of a step, as signed bytes; zeros for a step of 0 or NaN."""
    x = np.asarray(x, np.float32)
    if not step > 0:
        return np.zeros(x.shape, np.int8)
    return np.rint(x * np.float32(np.float32(1) / step)).astype(np.int8)


def norm_quant(x, residual, weight, eps, normalize=True):
    """(q, scale in float64, h in float32) of rows; x and residual float32."""
    h = np.asarray(x, np.float32)
    if residual is not None:
        h = (h + np.asarray(residual, np.float32)).astype(np.float32)
    t = h if weight is None else (h * np.asarray(weight, np.float32)).astype(np.float32)
    q = np.zeros(h.shape, np.int8)
    scale = np.zeros(len(h))
    for i in range(len(h)):
        s = step_of(t[i])
        q[i] = to_bytes(t[i], s)
        scale[i] = float(s) / np.sqrt(np.mean(h[i].astype(np.float64) ** 2) + eps) if normalize else float(s)
    return q, scale, h


def linear_i8(x, xs, w, ws, bias):
    y = x.astype(np.float64) @ w.astype(np.float64).T       # exact: whole numbers below 2^53
    y = y * np.asarray(xs, np.float64)[:, None] * np.asarray(ws, np.float64)[None, :]
    return y if bias is None else y + np.asarray(bias, np.float64)


class Cache:
    """data int8 [pages, heads, 2, P, Dp], scales float32 [pages, heads, 2]."""

    def __init__(self, data, scales, dim):
        self.data, self.scales, self.dim = data.copy(), scales.copy(), dim
        self.P = data.shape[3]

    def page(self, table, b, i):
        if i < 0 or i >= table.shape[1]:
            return -1
        p = int(table[b, i])
        return p if 0 <= p < len(self.data) else -1

    def write(self, k, v, table, start, offsets):
        P, D = self.P, self.dim
        for b in range(len(table)):
            s0, n = int(start[b]), int(offsets[b + 1] - offsets[b])
            if n <= 0:
                continue
            for i in range(s0 // P, (s0 + n - 1) // P + 1):
                page = self.page(table, b, i)
                if page < 0:
                    continue
                lo, hi = max(s0, i * P), min(s0 + n, (i + 1) * P)
                r0, r1, t0 = lo - i * P, hi - i * P, int(offsets[b]) + lo - s0
                for h in range(self.data.shape[1]):
                    for kind, x in enumerate((k, v)):
                        rows = x[t0:t0 + r1 - r0, h].astype(np.float32)
                        s, old = step_of(rows), self.scales[page, h, kind]
                        if r0:
                            s = np.maximum(s, old)              # NaN if either is
                        block = self.data[page, h, kind]
                        if r0 and s != old:
                            f = np.float32(old * (np.float32(1) / s if s > 0 else np.float32(0)))
                            block[:r0] = np.rint(block[:r0].astype(np.float32) * f).astype(np.int8) if f != 0 and f == f else 0
                        block[r0:r1] = 0
                        block[r0:r1, :D] = to_bytes(rows, s)
                        self.scales[page, h, kind] = s

    def tokens(self, table, b, positions):
        """(k, v, ok) of positions of sequence b, float64 [n, heads, dim]."""
        n, H = len(positions), self.data.shape[1]
        out = np.zeros((2, n, H, self.dim))
        ok = np.zeros(n, bool)
        for j, p in enumerate(positions):
            page = self.page(table, b, int(p) // self.P) if p >= 0 else -1
            if page >= 0:
                ok[j] = True
                q = self.data[page, :, :, int(p) % self.P, :self.dim].astype(np.float32)
                out[:, j] = (q * self.scales[page][:, :, None]).astype(np.float64).transpose(1, 0, 2)
        return out[0], out[1], ok

    def attend(self, q, table, begin, end, scale):
        """q [B, T, H, D] -> (out, lse) in float64."""
        B, T, H, D = q.shape
        heads = self.data.shape[1]
        g = H // heads
        out, lse = np.zeros((B, T, H, D)), np.full((B, T, H), -np.inf)
        for b in range(B):
            hi = table.shape[1] * self.P
            e = hi if end is None else min(hi, int(end[b]))
            a = 0 if begin is None else max(0, int(begin[b]))
            k, v, ok = self.tokens(table, b, range(a, max(a, e)))
            for t in range(T):
                see = ok.copy()
                last = (hi if end is None else int(end[b])) - (T - 1 - t)
                see[max(0, last - a):] = False
                if not see.any():
                    continue
                for h in range(H):
                    s = (k[see, h // g] @ q[b, t, h].astype(np.float64)) * scale
                    m = s.max()
                    p = np.exp(s - m)
                    out[b, t, h] = p @ v[see, h // g] / p.sum()
                    lse[b, t, h] = m + np.log(p.sum())
        return out, lse
