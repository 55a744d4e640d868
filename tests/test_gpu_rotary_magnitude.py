"""A rotation's magnitude is a number of 64 bits: f32 rows are turned in 64 bits and rounded once with any magnitude, not only with one that 32 bits hold.

Bound: sine and cosine as in test_gpu_rotary_cancel, 2^-46 of the pair, then half a step of f32."""
import math

import numpy as np
import pytest
import torch

from attn_util import host, rng, rounded
from oracle import attn_oracle as O
from paper_2510_19482_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("magnitude", [1 + 0.1 * math.log(8), 1 + 0.1 * math.log(32), 0.1, 1 / 3])
def test_magnitude(magnitude, interleaved):
    assert float(np.float32(magnitude)) != magnitude
    r = rng("magnitude", magnitude, interleaved)
    t, x = rounded(r.normal(size=(64, 3, 64)), "f32")
    at = np.zeros(64, np.int32)                # no turn: the product alone, rounded once
    f = B.rotary_frequencies(64)
    got = host(B.hlq_rotary(t.cuda(), torch.from_numpy(at).cuda(), B.Rotary(f, interleaved, magnitude)))
    np.testing.assert_array_equal(got, (x * magnitude).astype(np.float32).astype(np.float64))
    at = r.integers(0, 4096, size=64).astype(np.int32)
    got = host(B.hlq_rotary(t.cuda(), torch.from_numpy(at).cuda(), B.Rotary(f, interleaved, magnitude)))
    y = O.turned(x, at, f, interleaved, magnitude)
    a = np.abs(x)
    pair = np.repeat(a[..., 0::2] + a[..., 1::2], 2, -1) if interleaved else np.tile(a[..., :32] + a[..., 32:], 2)
    e = 2.0**-46 * magnitude * pair
    assert (np.abs(got - y) <= e + 2.0**-24 * (np.abs(y) + e)).all()
