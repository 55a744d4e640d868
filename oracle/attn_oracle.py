"""Rotary positions, the paged cache and attention in 64-bit numpy, written from the definitions; shares no code with the GPU path."""
import numpy as np

from oracle import mx4_oracle as MX4

BLOCK = 32
# e4m3: sign, four exponent bits with bias 7, three mantissa bits; code 127 is NaN, the largest value 448
E4M3 = np.array([(c & 7) * 2.0**-9 if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(127)])


def turned(x, positions, frequencies, interleaved=False, magnitude=1.0):
    """x [T, heads, dim] with its first 2 len(frequencies) values turned; angles in extended precision."""
    n = len(frequencies)
    y = np.array(x, dtype=np.float64)
    angle = np.asarray(positions).astype(np.longdouble)[:, None] * np.asarray(frequencies, dtype=np.longdouble)
    c, s = (f(angle).astype(np.float64)[:, None, :] * magnitude for f in (np.cos, np.sin))
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    a, b = y[..., first].copy(), y[..., second].copy()
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    return y


def mx8_quantize(x):
    """codes u8 and scale bytes u8 [..., dim / 32] of x [..., dim]."""
    x = np.asarray(x, dtype=np.float64)
    v = x.reshape(*x.shape[:-1], -1, BLOCK)
    bad = ~np.isfinite(v).all(-1)
    v = np.where(bad[..., None], 0.0, v)
    top = np.abs(v).max(-1)
    _, e = np.frexp(top)
    e = np.where(top > 0, np.maximum(e - 1 - 8, -127), -127)
    a = np.minimum(np.abs(np.ldexp(v, -e[..., None])), 448.0)
    # the nearest of the table; of two that are as near the one with the even index
    up = np.searchsorted(E4M3, a).clip(0, 126)
    low = np.maximum(up - 1, 0)
    near_up, near_low = E4M3[up] - a, a - E4M3[low]
    code = np.where((near_up < near_low) | ((near_up == near_low) & (up % 2 == 0)), up, low)
    code = code + 128 * np.signbit(v)
    return code.astype(np.uint8).reshape(x.shape), np.where(bad, 255, e + 127).astype(np.uint8)


def mx8_values(codes, scales):
    v = E4M3[codes & 127] * np.where(codes & 128, -1.0, 1.0)
    s = np.repeat(scales.astype(np.int64), BLOCK, -1)
    return np.where(s == 255, np.nan, np.ldexp(v, s - 127))


def mx_quantize(x, kind):
    """codes u8 (4-bit ones two a byte) and scale bytes of x [..., dim]."""
    if kind == "mx8":
        return mx8_quantize(x)
    flat = np.asarray(x).reshape(-1, x.shape[-1])
    codes, scales = MX4.quantize(flat)
    return codes.reshape(*x.shape[:-1], -1), scales.reshape(*x.shape[:-1], -1)


def mx_values(codes, scales, kind):
    if kind == "mx8":
        return mx8_values(codes, scales)
    dim = codes.shape[-1] * 2
    return MX4.dequantize(codes.reshape(-1, dim // 2), scales.reshape(-1, dim // BLOCK), dim).reshape(*codes.shape[:-1], dim)


def attend(q, k, v, seen, scale):
    """softmax over what is seen of scale q k^T, times v, for one head: q [n, dim], k and v [m, dim], seen [n, m]; rows that see nothing are 0.
    Also the sum of the weights' and values' magnitudes, and the largest sum of a score's products' magnitudes among those seen of each row."""
    out, size, products = np.zeros((len(q), v.shape[1])), np.zeros((len(q), v.shape[1])), np.zeros(len(q))
    for i in range(len(q)):
        at = np.nonzero(seen[i])[0]
        if not len(at):
            continue
        with np.errstate(all="ignore"):
            s = scale * (k[at] @ q[i])
            if s.max() == -np.inf:
                continue
            p = np.exp(s - s.max())
            p = p / p.sum()
            out[i] = p @ v[at]
            size[i] = p @ np.abs(v[at])
            products[i] = abs(scale) * (np.abs(k[at]) @ np.abs(q[i])).max()
    return out, size, products
