"""Rotary positions where a pair's parts nearly cancel, so that the error of sine and cosine shows: f32 pairs next to the one that is turned onto an axis.

Bound: frequencies are fractions of a turn off by 2^-65, times positions below 2^12; sine, cosine, their products with 24-bit values and the sum are off by a few units of 2^-53: together
below 2^-46 of the pair, then half a step of f32."""
import numpy as np
import pytest
import torch

from attn_util import host
from oracle import attn_oracle as O
from paper_2510_19482_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("first", [0, 1])
def test_pairs_that_nearly_cancel(first, interleaved):
    f = B.rotary_frequencies(128)
    at = np.arange(0, 4096, 13).astype(np.int32)
    angle = at[:, None] * np.asarray(f)
    a, b = (np.sin(angle), np.cos(angle)) if first == 0 else (np.cos(angle), -np.sin(angle))
    x = np.stack((a, b), -1).reshape(len(at), 1, 128) if interleaved else np.concatenate((a, b), 1)[:, None]
    x = x.astype(np.float32).astype(np.float64)
    got = host(B.hlq_rotary(torch.from_numpy(x).float().cuda(), torch.from_numpy(at).cuda(), B.Rotary(f, interleaved)))
    y = O.turned(x, at, f, interleaved)
    e = 2.0**-46
    assert (np.abs(got - y) <= e + 2.0**-24 * (np.abs(y) + e)).all(), np.abs(got - y).max()
