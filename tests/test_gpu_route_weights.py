"""The router's weights in fp32 against 64 bits.  Logits are multiples of 2^-10 below 2^7, so that a difference of two is exact in fp32.  With h = 2^-24, half
of a unit in the last place: a term's exponential 2 h (one unit), the sum 2 h of its terms and h for each addition that a term goes through (one
sixteenth of the terms one after another, then four), the quotient h, and one for what these make of each other.  A weight below the smallest normal
number may be 0."""
import pytest
import torch

from paper_2510_19482_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("span", [8.0, 40.0, 100.0])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("T,E,k", [(40, 16, 16), (3, 64, 8), (300, 100, 64), (200, 256, 30), (64, 384, 8), (33, 512, 40), (40, 1024, 64)])
def test_weights(T, E, k, dtype, renorm, span):
    g = torch.Generator("cuda").manual_seed(T + E + k)
    x = ((torch.rand(T, E, device="cuda", generator=g) - 0.5) * span * 1024).round() / 1024
    x = x.to(dtype)
    r = B.hlq_route(x, k, renorm)
    top, ids = torch.sort(x.double(), dim=1, descending=True, stable=True)
    assert torch.equal(r.ids.long(), ids[:, :k])
    p = torch.exp(top - top[:, :1])
    want = p[:, :k] / (p[:, :k] if renorm else p).sum(1, keepdim=True)
    additions = -(-(k if renorm else E) // 16) + 4
    d, bound = (r.weights.double() - want).abs(), (6 + additions) * 2.0**-24 * want + 2.0**-126
    assert bool((d <= bound).all()), f"{float((d / bound).max())} of the bound"
