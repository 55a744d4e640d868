"""Microscaled 4-bit matrices and the expert block in 64-bit numpy, written from the definitions; shares no code with the GPU path.

A value is an e2m1 float (sign, two exponent bits with bias 1, one mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6) times
2^(byte - 127), one byte for each 32 successive values of a row; byte 255 is NaN."""
import numpy as np

BLOCK = 32
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantize(x):
    """codes u8 [rows, (K + 1) // 2], scales u8 [rows, (K + 31) // 32] of x [rows, K]."""
    x = np.asarray(x, dtype=np.float64)
    rows, K = x.shape
    nb = -(-K // BLOCK)
    v = np.zeros((rows, nb * BLOCK))
    v[:, :K] = x
    v = v.reshape(rows, nb, BLOCK)
    with np.errstate(invalid="ignore"):
        bad = ~np.isfinite(v).all(-1)
    top = np.where(bad, 0.0, np.abs(np.where(np.isfinite(v), v, 0.0)).max(-1))
    _, e = np.frexp(top)                       # top = m 2^e, 0.5 <= m < 1
    e = np.where(top > 0, np.maximum(e - 1 - 2, -127), -127)
    scaled = np.ldexp(np.where(bad[..., None], 0.0, v), -e[..., None])
    a = np.abs(scaled)
    # the nearest of the eight; of two that are as near the one with the even index
    d = np.abs(a[..., None] - GRID)
    code = d.argmin(-1)                        # the lower of a tie
    up = np.minimum(code + 1, 7)
    code = np.where((np.take_along_axis(d, up[..., None], -1)[..., 0] == d.min(-1)) & (code % 2 == 1), up, code)
    code = (code + 8 * np.signbit(scaled)).astype(np.uint8).reshape(rows, -1)
    code[:, K:] = 0
    code = code[:, :(K + 1) // 2 * 2]
    return code[:, 0::2] | (code[:, 1::2] << 4), np.where(bad, 255, e + 127).astype(np.uint8)


def dequantize(codes, scales, K):
    c = np.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[0], -1)[:, :K]
    v = GRID[c & 7] * np.where(c & 8, -1.0, 1.0)
    s = np.repeat(scales.astype(np.int64), BLOCK, 1)[:, :K]
    return np.where(s == 255, np.nan, np.ldexp(v, s - 127))


def rounded(x):
    """The values that x stands for in the 4-bit form."""
    return dequantize(*quantize(x), x.shape[1])


def gate(p):
    h = p.shape[1] // 2
    g, u = p[:, :h], p[:, h:]
    with np.errstate(over="ignore"):
        return g / (1.0 + np.exp(-g)) * u


def route(logits, k, renorm):
    """ids, weights, offsets, rows, slots."""
    x = np.asarray(logits, dtype=np.float64)
    T, E = x.shape
    x = np.where(np.isnan(x), -np.inf, np.minimum(x, float(np.finfo(np.float32).max)))
    ids, w = np.full((T, k), -1, np.int32), np.zeros((T, k))
    for t in range(T):
        order = [e for e in np.argsort(-x[t], kind="stable") if x[t, e] > -np.inf]
        pick = order[:k]
        if pick:
            p = np.exp(x[t, pick] - x[t, pick[0]])
            total = p.sum() if renorm else np.exp(x[t, order] - x[t, pick[0]]).sum()
            ids[t, :len(pick)], w[t, :len(pick)] = pick, p / total
    rows, slots, offsets = np.full(T * k, -1, np.int32), np.full((T, k), -1, np.int32), [0]
    at = 0
    for e in range(E):
        for t, i in zip(*np.nonzero(ids == e)):
            rows[at], slots[t, i] = t, at
            at += 1
        offsets.append(at)
    return ids, w, np.array(offsets, np.int32), rows, slots
