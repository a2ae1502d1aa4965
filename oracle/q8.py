"""The 8-bit operators in plain numpy: float64 arithmetic, float32 where a value is kept in 32 bits (scales).  TEST
INFRASTRUCTURE ONLY, like the rest of this package."""
import numpy as np


def bf16(x):
    """float64 -> nearest bf16, as float64."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16 << 16).astype(np.uint32).view(np.float32)
    return np.where(np.isnan(x), np.nan, r.astype(np.float64))


def quantize(x):
    """Rows, rounded to float32, in 8 bits: integers, float32 scales, and the distance of every float32 quotient from the nearest border
    between integers."""
    x = np.asarray(x, dtype=np.float64).astype(np.float32)
    bad = ~np.isfinite(x).all(-1)
    most = np.abs(np.where(np.isfinite(x), x, 0)).max(-1)
    scale = np.where(bad, np.float32(np.nan), most / np.float32(127))
    live = (scale > 0) & ~bad
    with np.errstate(invalid="ignore"):
        t = np.where(live[..., None], x / np.where(live, scale, np.float32(1))[..., None], 0).astype(np.float64)
    t = np.where(np.isfinite(t), t, 0)
    return np.clip(np.rint(t), -127, 127).astype(np.int64), scale, np.abs(np.abs(t - np.floor(t)) - 0.5)


def rmsnorm(x, add, gain, eps):
    """(x + add in float32, the normalised rows in float64)."""
    s = np.asarray(x, dtype=np.float32) + (0 if add is None else np.asarray(add, dtype=np.float32))
    w = s.astype(np.float64)
    return s, w / np.sqrt((w * w).mean(-1, keepdims=True) + eps) * np.asarray(gain, dtype=np.float64)


def gemm(x, sx, w, sw):
    return (x.astype(np.int64) @ w.astype(np.int64).T).astype(np.float64) * sx.astype(np.float64)[:, None] * sw.astype(np.float64)


def swiglu(y):
    g, u = np.split(y, 2, axis=-1)
    return g / (1 + np.exp(np.minimum(-g, 700))) * u


def rotate(x, cos, sin):
    """x [rows, heads, hd], cos, sin [rows, hd/2]: pairs (i, i + hd/2)."""
    a, b = np.split(np.asarray(x, dtype=np.float64), 2, axis=-1)
    c, s = cos.astype(np.float64)[:, None], sin.astype(np.float64)[:, None]
    return np.concatenate([a * c - b * s, a * s + b * c], -1)


class Cache:
    """One layer and sequence: [positions, heads, hd] integers and [blocks, heads] float32 scales, for keys or for values."""

    def __init__(self, heads, hd, capacity, block):
        self.q = np.zeros((capacity, heads, hd), np.int64)
        self.s = np.zeros((capacity // block, heads), np.float32)
        self.block = block

    def append(self, pos0, x):
        x = np.asarray(x, dtype=np.float32)
        n, B = len(x), self.block
        for b in range(pos0 // B, (pos0 + n - 1) // B + 1):
            lo, hi = max(pos0, b * B), min(pos0 + n, (b + 1) * B)
            new = x[lo - pos0:hi - pos0]
            held = slice(b * B, lo) if b * B < pos0 else slice(0, 0)
            bad = ~np.isfinite(new).all((0, 2))
            most = np.abs(np.where(np.isfinite(new), new, 0)).max((0, 2))
            was = self.s[b] if b * B < pos0 else np.zeros_like(self.s[b])
            now = np.maximum(was, most / np.float32(127))                 # (a NaN that is held stays)
            now[bad] = np.nan
            live = now > 0
            ratio = np.where(live, was / np.where(live, now, 1), np.where(np.isnan(now), 0, 1)).astype(np.float32)
            self.q[held] = np.rint(self.q[held].astype(np.float32) * ratio[:, None])          # in float32, as the quotient below
            safe = np.where(live, now, 1).astype(np.float32)[:, None]
            self.q[lo:hi] = np.where(live[:, None], np.clip(np.rint((np.where(np.isfinite(new), new, 0) / safe).astype(np.float32)), -127, 127), 0)
            self.s[b] = now

    def values(self, n):
        return self.q[:n] * np.repeat(self.s, self.block, 0)[:n, :, None].astype(np.float64)


def attention(q, k, v, pos0, scale):
    """q [rows, Hq, hd] at positions pos0 ..; k, v [positions, Hkv, hd] -> (out, softmax-weighted mean of |v|, weights' scores
    [rows, Hq, positions] with -inf where a row does not see)."""
    q, k, v = (np.asarray(a, dtype=np.float64) for a in (q, k, v))
    rows, hq, hd = q.shape
    group = hq // k.shape[1]
    s = np.einsum("rhd,phd->rhp", q, np.repeat(k, group, 1)) * scale
    s = np.where(np.arange(k.shape[0]) <= (pos0 + np.arange(rows))[:, None, None], s, -np.inf)
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    vg = np.repeat(v, group, 1)
    return np.einsum("rhp,phd->rhd", p, vg), np.einsum("rhp,phd->rhd", p, np.abs(vg)), s
