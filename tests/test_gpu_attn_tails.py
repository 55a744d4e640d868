"""What many small weights add up to beside a few large ones.

Scores here are exact: one channel of the queries is 1, the keys' is the score.  A peak of score 0 stands in each tile or piece of keys that takes its exponentials by itself, the
others' scores are -`nats`; the peaks' values are 0, the others' 1, so that a result is the others' share.

Bounds.  A weight is off by 2^-21 (1 + nats) relative to itself for the factors, the difference and the exponential, by what it is rounded by (h: 2^-22 as two terms, 2^-11 as one; bf16
2^-16 and 2^-8), and in f16 by half of the smallest step: the largest weight of a piece is 2^6 or more and the step 2^-24 (of the second term, 2^11 smaller, 2^-35), so relative to the largest by 2^-25 / 2^6 = 2^-31, as two
terms 2^-42.  In numerator and sum, with n additions off by 2^-23: a result y of n weights is off by at most
    y (2 (2^-21 (1 + nats) + h) + 2 n' 2^-23) + 2 n 2^-31 (or 2^-42),
n' the additions that a number goes through, 32 at least in one product of the matrix cores and otherwise one for each tile: n / 32 + 64; and then by its own rounding."""
import math

import pytest
import torch

from attn_util import HALF_STEP, SMALLEST, host
from paper_2510_19482_amd import binding as B

pytestmark = pytest.mark.gpu


def off(y, nats, n, h, floor, dtype):
    e = y * (2 * (2.0**-21 * (1 + nats) + h) + 2 * (n / 32 + 64) * 2.0**-23) + 2 * n * floor
    return e + HALF_STEP[dtype] * (y + e) + SMALLEST[dtype]


DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
TERMS = {"f16": ((2.0**-11, 2.0**-31), (2.0**-22, 2.0**-42)), "bf16": ((2.0**-8, 2.0**-126), (2.0**-16, 2.0**-126))}   # (h, floor) of one term, of two


def rows(n, D, every, first, nats, dtype):
    """Keys and values [n, 1, D]: peaks at every .. th row, `first` of them next to each other."""
    peak = torch.arange(n) % every < first
    k, v = torch.zeros((n, 1, D)), torch.ones((n, 1, D))
    k[:, 0, 0] = torch.where(peak, 0.0, -nats)
    v[peak] = 0
    return k.to(DTYPES[dtype]).cuda(), v.to(DTYPES[dtype]).cuda(), int(peak.sum())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("nats", [5.0, 9.0, 11.0, 14.0, 16.0, 17.0, 18.0, 21.0])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("sequences,n,every", [(1000, 8192, 8192), (1, 131072, 1024)])
def test_decode(sequences, n, every, D, nats, dtype):
    # many sequences are not cut: their four wavefronts have a peak in their first tiles.  One is, 1024 tokens a workgroup or more
    k, v, peaks = rows(n, D, every, 128, nats, dtype)
    kv = B.alloc_kv_cache(n // 128, 128, 1, D, DTYPES[dtype])
    B.hlq_kv_write(kv, k, v, torch.arange(n, device="cuda"))
    q = torch.zeros((sequences, 1, D), dtype=DTYPES[dtype], device="cuda")
    q[:, :, 0] = 1
    table = torch.arange(n // 128, dtype=torch.int32, device="cuda").expand(sequences, -1).contiguous()
    got = host(B.hlq_attn_decode(kv, q, table, torch.full((sequences,), n, dtype=torch.int32, device="cuda"), scale=1.0, out_dtype=torch.float32))
    tail = (n - peaks) * math.exp(-nats)
    y = tail / (tail + peaks)
    worst = abs(got - y).max()
    most = off(y, nats, n, *TERMS[dtype][1], "f32")
    assert worst <= most, (worst / y, most / y)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("nats", [5.0, 9.0, 11.0, 14.0, 16.0, 17.0, 18.0])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n_q,n_k", [(1, 65536), (700, 65536), (4096, 16384)])
def test_prompt(n_q, n_k, D, nats, dtype):
    # a workgroup has 256 keys at least
    k, v, peaks = rows(n_k, D, 4096, 2, nats, dtype)
    q = torch.zeros((n_q, 2, D), dtype=DTYPES[dtype], device="cuda")
    q[:, :, 0] = 1
    q_at, k_at = (torch.tensor([0, n], dtype=torch.int32, device="cuda") for n in (n_q, n_k))
    got = host(B.hlq_attn_prompt(q, k, v, q_at, k_at, causal=False, scale=1.0))
    tail = (n_k - peaks) * math.exp(-nats)
    y = tail / (tail + peaks)
    worst = abs(got - y).max()
    most = off(y, nats, n_k, *TERMS[dtype][0], dtype)
    assert worst <= most, (worst / y, most / y)
