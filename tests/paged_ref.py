"""Float64 reference of the rotary and paged-cache calls, in numpy, from their formulas in
include/retopk.h; it shares no code with the library."""
import math

import numpy as np

GROUP = 64
LEVELS = np.arange(16) - 7.5


def bf16_round(x):
    """float32 values of x rounded to bf16, nearest even (finite x)."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    u = (u + 0x7FFF + ((u >> np.uint64(16)) & np.uint64(1))) & np.uint64(0xFFFF0000)
    return u.astype(np.uint32).view(np.float32)


def rotate(x, pos, freq, factor, rot, interleaved, inverse=False):
    """x [T, H, d] float64, pos [T]."""
    y = np.array(x, np.float64)
    ang = np.asarray(pos, np.float64)[:, None, None] * np.asarray(freq)[None, None, :rot // 2]
    c, s = factor * np.cos(ang), factor * np.sin(ang) * (-1 if inverse else 1)
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * c - b * s, a * s + b * c
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2], y[..., rot // 2:rot] = a * c - b * s, a * s + b * c
    return y


def group_params(x):
    """(mid, scale) float64 [..., d / 64] of float32 rows."""
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, GROUP)
    mid = bf16_round(((g.max(-1) + g.min(-1)) / 2).astype(np.float32)).astype(np.float64)
    reach = np.maximum(g.max(-1) - mid, mid - g.min(-1))
    return mid, bf16_round((reach / 7.5).astype(np.float32)).astype(np.float64)


def unpack(codes):
    """c of every element, float64 [..., d], of code bytes [..., d / 2]."""
    b = np.asarray(codes).reshape(*codes.shape[:-1], -1, 2).astype(np.int64)
    bits = [(b[..., i, None] >> np.arange(7, -1, -1)) & 1 for i in (0, 1)]     # top bit first
    mag = lambda z, at: 4 * z[..., at] + 2 * z[..., at + 1] + z[..., at + 2]   # noqa: E731
    m = [mag(bits[0], 1), mag(bits[0], 5), mag(bits[1], 1), mag(bits[1], 5)]
    s = [bits[1][..., 0], bits[1][..., 4], bits[0][..., 0], bits[0][..., 4]]
    c = np.stack([(mm + 0.5) * np.where(ss == 1, -1.0, 1.0) for mm, ss in zip(m, s)], -1)
    return c.reshape(*codes.shape[:-1], -1)


def params_of_words(words):
    w = np.asarray(words).view(np.uint32)
    scale = (w << np.uint32(16)).view(np.float32).astype(np.float64)
    mid = (w & np.uint32(0xFFFF0000)).view(np.float32).astype(np.float64)
    return mid, scale


def values4(codes, words):
    """float64 values (before the rounding to float32) of 4-bit rows."""
    mid, scale = params_of_words(words)
    return np.repeat(mid, GROUP, -1) + np.repeat(scale, GROUP, -1) * unpack(codes)


def attend(q, k, v, keep=None):
    """(out, lse, spread) of one head: q [d], k and v [n, d] float64; spread is the largest
    sum |q k| / sqrt(d) over the kept rows, which bounds a score's rounding."""
    d = q.shape[0]
    if keep is not None:
        k, v = k[keep], v[keep]
    if k.shape[0] == 0:
        return np.zeros(d), -math.inf, 0.0, np.zeros(d)
    s = (k @ q) / math.sqrt(d)
    m = s.max()
    p = np.exp(s - m)
    spread = float((np.abs(k) @ np.abs(q)).max() / math.sqrt(d))
    return p @ v / p.sum(), float(m + math.log(p.sum())), spread, p @ np.abs(v) / p.sum()
