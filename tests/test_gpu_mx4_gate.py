"""The gated epilogue, silu(g) u, in fp32: g and u are exact here (one product of two 4-bit values, or a sum of a few that fp32 holds), so what a
result is off is the epilogue's own.  With h = 2^-24, half of a unit in the last place: the exponential 2 h (one unit), what its argument was rounded
by 2 h, its sum with 1 another h, the reciprocal 2 h, two products h each: 9 h of the result, 10 h with what the steps add to each other.
Where silu(g) is below fp32's smallest normal number it may be 0.  For 16-bit results the argument's rounding stays: half a unit of |g| log2 e, and what
log2 e itself is rounded by, 1.25 |g| h at most.  Then the result is rounded once, or to 0 below the smallest normal number."""
import pytest
import torch

from paper_2510_19482_amd import binding as B

pytestmark = pytest.mark.gpu

HALF = 2.0**-24
HALF_ULP = {torch.float32: HALF, torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11}
SMALLEST = {torch.float32: 2.0**-126, torch.bfloat16: 2.0**-126, torch.float16: 2.0**-25}


def operands(R, N, top, u_exponent):
    """x [R, 96] of whole numbers, weights so that g spreads over +-top and u is of size 2^u_exponent; all exact."""
    g = torch.Generator("cuda").manual_seed(R + N)
    x = torch.zeros(R, 96, device="cuda")
    x[:, 0], x[:, 32], x[:, 64] = 4.0, 4.0 / 16, 4.0 / 256        # three blocks, each one's value its largest
    x *= torch.randint(0, 2, (R, 1), device="cuda", generator=g) * 2 - 1
    codes = torch.zeros(2 * N, 48, dtype=torch.uint8, device="cuda")
    for k in (0, 32, 64):
        codes[:, k // 2] = torch.randint(0, 16, (2 * N,), device="cuda", generator=g).to(torch.uint8)
    scales = torch.full((2 * N, 3), 127, dtype=torch.uint8, device="cuda")
    e = round(torch.tensor(top / 24.0).log2().item())
    scales[:N] += e + torch.randint(-2, 1, (N, 1), device="cuda", generator=g).to(torch.uint8)
    scales[N:] = 127 + u_exponent
    return x, B.hlq_mx4_pack(codes, scales, 96)


# rows for each kernel; the largest tiles take one round of the card at least
@pytest.mark.parametrize("R,N", [(3, 300), (40, 500), (150, 2000), (600, 2100), (4096, 4000)])
@pytest.mark.parametrize("dtype", list(HALF_ULP), ids=str)
@pytest.mark.parametrize("top,u_exponent", [(10, 0), (48, 0), (96, 0), (96, 90), (96, -20)])
def test_gate(R, N, top, u_exponent, dtype):
    if dtype is torch.float16 and u_exponent > 0:
        pytest.skip("the results are past the type's largest")
    x, W = operands(R, N, top, u_exponent)
    y = B.hlq_mx4_gemm(W, x, gated=True, out_dtype=dtype).double()
    p = x.double() @ B.hlq_mx4_dequantize(W).double().T.contiguous()
    assert torch.equal(p, p.float().double())
    g, u = p[:, :N], p[:, N:]
    silu = g * torch.sigmoid(g)
    want = silu * u
    off = (10 + (1.25 * g.abs() if dtype is not torch.float32 else 0)) * HALF * want.abs() + torch.where(g < 0, 2.0**-126, 0.0) * u.abs()
    off = off + (want.abs() + off) * HALF_ULP[dtype] + SMALLEST[dtype]
    d = (y - want).abs()
    assert bool((d <= off).all()), f"{int((d > off).sum())} off, {float((d / off).max())} of the bound at g = {float(g.flatten()[(d / off).flatten().argmax()])}"
    assert float(g.min()) < -0.75 * top


@pytest.mark.parametrize("R,N", [(3, 300), (40, 500), (600, 2100)])
def test_gate_of_what_is_large(R, N):
    # up to fp32's largest: silu(g) is g, or 0
    for e in (20, 100, 122):
        x, W = operands(R, N, 24.0 * 2.0**e, -30)
        y = B.hlq_mx4_gemm(W, x, gated=True, out_dtype=torch.float32).double()
        p = x.double() @ B.hlq_mx4_dequantize(W).double().T.contiguous()
        g, u = p[:, :N], p[:, N:]
        want = torch.where(g > 0, g, 0.0) * u
        assert bool(((y - want).abs() <= 10 * HALF * want.abs()).all())
