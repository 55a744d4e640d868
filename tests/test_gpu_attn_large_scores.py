"""Scores so large that neighbouring 32-bit numbers are further apart than what an exponential holds: still a mean of the values with the largest score.

One channel of q and k is not 0, so scores are exact products; scores that differ, differ by more than 1000, so a result is the mean of the values whose score is the largest."""
import pytest
import torch

from attn_util import HALF_STEP, TYPES, rng, rounded
from paper_2510_19482_amd import binding as B
from test_gpu_attn_corners import shifted

pytestmark = pytest.mark.gpu

# powers of two of q and k
SIZES = {"f16": [(8, 15), (13, 14), (15, 15)], "bf16": [(8, 15), (10, 22), (20, 25), (30, 40), (50, 60)]}
CASES = [(t, a, b) for t, s in SIZES.items() for a, b in s]


def inputs(r, n_q, n_k, Hq, D, dtype, a, b, sign):
    """Queries 2^a to 2^(a + 1), keys 2^b times 1, 1 - 2^-3 and 1 - 2^-2: one in eight is the largest."""
    q, k = torch.zeros((n_q, Hq, D), dtype=torch.float64), torch.zeros((n_k, 1, D), dtype=torch.float64)
    q[:, :, 3] = torch.from_numpy((1 + r.integers(0, 128, size=(n_q, Hq)) / 128.0) * 2.0**a * 0.49)
    k[:, 0, 3] = torch.from_numpy(2.0**b * (1 - r.integers(0, 8, size=n_k) / 16.0)) * sign
    v = torch.from_numpy(r.integers(1, 9, size=(n_k, 1, D)).astype(float))
    return [x.to(TYPES[dtype]) for x in (q, k, v)]


def check(got, q, k, v, seen, scale, dtype, weight=0.0):
    got, k0, v = got.double().cpu(), k[:, 0, 3].double(), v[:, 0].double()
    for i in range(q.shape[0]):
        at = torch.nonzero(seen(i)).flatten()
        s = scale * k0[at]                                    # (q is positive)
        best = at[s == s.max()]
        want = v[best].mean(0)
        # Weights of the same score are the same number w; sums of small whole numbers times it are off by 2^-23 an addition at most, above and below.  One token's weights are two
        # terms above, each off by half a step of what it holds (`weight` = h h for half steps h of 2^-8 or 2^-11), and w itself below.
        e = want * (len(best) * 2.0**-22 + weight)
        e = e + HALF_STEP[dtype] * (want + e)
        assert (abs(got[i] - want) <= e).all(), (i, got[i, 0, :4], want[:4])


@pytest.mark.parametrize("dtype,a,b", CASES)
@pytest.mark.parametrize("sign,scale", [(1, 1.0), (-1, 1.0), (1, -0.7), (-1, 0.3)])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_prompt(D, sign, scale, dtype, a, b):
    for n_q, n_k, causal in ((150, 150, True), (40, 2000, True), (70, 100, False)):
        q, k, v = inputs(rng("large", D, sign, scale, dtype, a, b, n_q), n_q, n_k, 2, D, dtype, a, b, sign)
        q_at, k_at = (torch.tensor([0, n], dtype=torch.int32, device="cuda") for n in (n_q, n_k))
        got = B.hlq_attn_prompt(q.cuda(), k.cuda(), v.cuda(), q_at, k_at, causal=causal, scale=scale)
        j = torch.arange(n_k)
        check(got, q, k, v, lambda i: (j <= n_k - n_q + i) if causal else j >= 0, scale, dtype)
        assert torch.equal(B.hlq_attn_prompt(shifted(q.cuda()), shifted(k.cuda()), shifted(v.cuda()), q_at, k_at, causal=causal, scale=scale), got)


@pytest.mark.parametrize("kind,dtype,a,b", [(t, t, a, b) for t, a, b in CASES] + [("mx8", "bf16", 20, 25), ("mx8", "f16", 15, 15), ("mx4", "bf16", 30, 40), ("mx4", "f16", 13, 14)])
@pytest.mark.parametrize("sign,scale", [(1, 1.0), (-1, 1.0), (1, -0.7), (-1, 0.3)])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_decode(D, sign, scale, kind, dtype, a, b):
    for n in (100, 5000):
        q, k, v = inputs(rng("large one", D, sign, scale, kind, dtype, a, b, n), 2, n, 3, D, dtype, a, b, sign)
        pages = -(-n // 64)
        kv = B.alloc_kv_cache(pages, 64, 1, D, TYPES[kind] if kind in TYPES else {"mx8": B.HLQ_MX8, "mx4": B.HLQ_MX4}[kind])
        slots = torch.arange(n, device="cuda")
        B.hlq_kv_write(kv, k.cuda(), v.cuda(), slots)
        k, v = (x.double().cpu() for x in B.hlq_kv_read(kv, slots))
        table = torch.arange(pages, dtype=torch.int32, device="cuda")[None].expand(2, -1).contiguous()
        got = B.hlq_attn_decode(kv, q.cuda(), table, torch.full((2,), n, dtype=torch.int32, device="cuda"), scale=scale, out_dtype=torch.float32)
        check(got, q, k, v, lambda i: torch.arange(n) >= 0, scale, "f32", 2.0**-22 if kind == "f16" else 2.0**-16)
