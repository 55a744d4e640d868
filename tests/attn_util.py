"""What the tests of attention and its cache share: inputs, layouts in numpy, and how far a result may be off.

Bounds.  A score is a sum of dim exact products in fp32: with an addition off by 2^-23 of what is summed (the matrix core may cut off instead of
rounding) it is off by at most (dim + 4) 2^-23 S, S the sum of its products' magnitudes; the two factors it is multiplied by, the difference and the
exponential add 2^-21 (1 + |score|) <= 2^-21 (1 + S) more.  A weight is off by that relative to itself, twice (numerator and sum), and by what it is
rounded by, h: once if the sum is of the weights before (`weight` = h), and if the sum is of the rounded ones twice (`weight` = 2 h), since then
sum p~ v / sum p~ - y = sum (p~ - p) (v - y) / sum p~ for the result y = sum p v / sum p, at most h (A + |y|) <= 2 h A.  With A the weighted sum of the values' magnitudes a result is off by at most
    A (2 (dim + 4) 2^-23 S + 2^-20 (1 + S) + weight + n 2^-23) + n 2^-25 max|v|,
the last two for n additions and, in f16, for weights below its smallest normal number, and then by its own rounding."""
import numpy as np
import torch

from oracle import attn_oracle as O
from paper_2510_19482_amd import binding as B

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"f16": 2.0**-11, "bf16": 2.0**-8, "f32": 2.0**-24}
SMALLEST = {"f16": 2.0**-25, "bf16": 2.0**-134, "f32": 2.0**-150}
KINDS = {"f16": torch.float16, "bf16": torch.bfloat16, "mx8": B.HLQ_MX8, "mx4": B.HLQ_MX4}


def rng(*key):
    return np.random.default_rng([ord(c) for c in repr(key)])


def rounded(x, dtype):
    """A tensor of the type on the host, and its values."""
    t = torch.from_numpy(np.asarray(x, dtype=np.float64)).to(TYPES[dtype])
    return t, t.double().numpy()


def host(t):
    return t.double().cpu().numpy()


def bound(size, products, n, dim, most, weight, dtype, value):
    e = size * (2 * (dim + 4) * 2.0**-23 * products + 2.0**-20 * (1 + products) + weight + n * 2.0**-23) + n * 2.0**-25 * most
    return e + HALF_STEP[dtype] * (np.abs(value) + e) + SMALLEST[dtype]


class Cache:
    """A cache on the GPU whose every unwritten number is NaN, and what its slots hold."""

    def __init__(self, pages, page, heads, dim, kind):
        self.kind, self.page, self.heads, self.dim, self.pages = kind, page, heads, dim, pages
        self.kv = B.alloc_kv_cache(pages, page, heads, dim, KINDS[kind])
        self.kv.blob.fill_(255)
        self.values = np.full((2, pages * page, heads, dim), np.nan)

    def put(self, slots, k, v, dtype):
        """Rows by way of hlq_kv_write; k and v are values of the type."""
        T = {n: torch.from_numpy(x).to(TYPES[dtype]).cuda() for n, x in (("k", k), ("v", v))}
        B.hlq_kv_write(self.kv, T["k"], T["v"], torch.from_numpy(np.asarray(slots, dtype=np.int64)).cuda())
        for i, x in enumerate((k, v)):
            self.values[i, slots] = stored(x, self.kind)


def stored(x, kind):
    """The values that a cache of this kind holds of x."""
    if kind in ("mx8", "mx4"):
        return O.mx_values(*O.mx_quantize(x, kind), kind)
    return rounded(x, kind)[1]
