"""Large products of microscaled 4-bit matrices, whose tiles workgroups take one after another: panels fewer and more than the stages in
flight, one round of tiles and several, ragged ends, rows that are whole lines of the memory and rows that are not.  The plain form in
64 bits runs on the GPU.

A block's sum of 32 products is exact, each of a row's ceil(K / 32) block sums is added once to an fp32 sum; with u = 2^-23 an addition
(the matrix core may cut off instead of rounding) the error is at most (blocks + 32) u times the sum of the products' magnitudes.  A
gated result adds what its two sums' errors make of silu (|silu'| <= 1.1, |silu(g)| <= |g|), the exponential and four operations.  Then a
result is rounded once to its type: 11, 8 or 24 significant bits."""
import pytest
import torch

from paper_2510_19482_amd import binding as B

pytestmark = pytest.mark.gpu

HALF_ULP = {torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8, torch.float32: 2.0**-24}
SMALLEST = {torch.float16: 2.0**-25, torch.bfloat16: 2.0**-126, torch.float32: 2.0**-126}


def mx4(rows, K, seed, size=1.0):
    """A matrix and its values in 64 bits."""
    g = torch.Generator("cuda").manual_seed(seed)
    m = B.hlq_mx4_quantize(torch.randn(rows, K, device="cuda", generator=g) * size)
    return m, B.hlq_mx4_dequantize(m, torch.empty(rows, K, device="cuda")).double()


def check(y, a, w, gated):
    p, mag = a @ w.T.contiguous(), a.abs() @ w.abs().T.contiguous()
    e = (-(-a.shape[1] // 32) + 32) * 2.0**-23 * mag
    if gated:
        h = p.shape[1] // 2
        gate, up = p[:, :h], p[:, h:]
        want = gate * torch.sigmoid(gate) * up
        e = 1.1 * e[:, :h] * (up.abs() + e[:, h:]) + gate.abs() * e[:, h:] + (16 + gate.abs()) * 2.0**-23 * want.abs() + 2.0**-120
    else:
        want = p
    e = e + (want.abs() + e) * HALF_ULP[y.dtype] + SMALLEST[y.dtype]
    d = (y.double() - want).abs()
    assert bool((d <= e).all()), f"{float((d / e).max())} of the bound"


# 235 tiles of 256 x 256 at least: a round of the card's workgroups, and more
@pytest.mark.parametrize("dtype", list(HALF_ULP), ids=str)
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M,N,K", [(4001, 4090, 33), (4096, 4096, 128), (4000, 4096, 257), (3841, 8130, 385), (8100, 4000, 512), (4096, 4096, 600), (3900, 4096, 1300),
                                   (8192, 8192, 160), (12290, 8000, 700)])
def test_product(M, N, K, gated, dtype):
    W, w = mx4(N, K, N + K, K**-0.5)
    X, x = mx4(M, K, M)
    check(B.hlq_mx4_gemm(W, X, gated=gated, out_dtype=dtype), x, w, gated)


@pytest.mark.parametrize("dtype", list(HALF_ULP), ids=str)
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("at,room", [(0, 0), (3, 5), (64, 64), (64, 8)])
def test_strides_and_what_lies_beside_the_results(at, room, gated, dtype):
    M, N, K = 4010, 4160, 200
    cols = N // 2 if gated else N
    W, w = mx4(N, K, 5, K**-0.5)
    X, x = mx4(M, K, 6)
    out = torch.full((M + 2, at + cols + room), 5.0, dtype=dtype, device="cuda")
    y = out[1:1 + M, at:at + cols]
    B.hlq_mx4_gemm(W, X, y, gated=gated)
    check(y, x, w, gated)
    again = y.clone()
    B.hlq_mx4_gemm(W, X, y, gated=gated)
    assert torch.equal(again, y)
    y[:] = 5.0
    assert bool((out == 5).all())


def test_infinities_and_nan_stay_in_their_rows_and_columns():
    M, N, K = 4096, 4096, 700
    g = torch.Generator("cuda").manual_seed(1)
    a, b = torch.randn(M, K, device="cuda", generator=g), torch.randn(N, K, device="cuda", generator=g)
    a[5, 650], a[M - 1, 3], b[7, 70] = float("inf"), float("nan"), float("nan")
    y = B.hlq_mx4_gemm(B.hlq_mx4_quantize(b), a)
    nan = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    nan[[5, M - 1]] = True
    nan[:, 7] = True
    assert torch.equal(torch.isnan(y), nan)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("counts", [[7300], [1, 7299], [0, 7300, 0], [2000, 0, 3000, 2400], [7300, 100, 0, 0], [1850, 1850, 1850, 1850]], ids=str)
def test_expert_product(counts, gated):
    E, R, N, K, T = len(counts), sum(counts), 4096, 224, 3000
    g = torch.Generator("cuda").manual_seed(R + E)
    rows = torch.randint(0, T, (R,), dtype=torch.int32, device="cuda", generator=g)
    W, w = mx4(E * N, K, 3, K**-0.5)
    X, x = mx4(T, K, 4)
    off = torch.tensor([0] + counts, dtype=torch.int32, device="cuda").cumsum(0).int()
    y = B.hlq_expert_gemm(W, off, X, rows=rows, gated=gated, out_dtype=torch.float32)
    at = 0
    for e, n in enumerate(counts):
        if n:
            check(y[at:at + n], x[rows[at:at + n].long()], w[e * N:(e + 1) * N], gated)
        at += n


def test_offsets_that_overlap_write_rows_only():
    E, R, N, K = 4, 7400, 4096, 128
    W, w = mx4(E * N, K, 3)
    X, x = mx4(R, K, 4)
    out = torch.full((R + 8, N), 3.0, device="cuda")
    for off in ([0, R, 0, R, 0], [-5, R + 5, -5, 1 << 30, R], [R] * 5, [0] * 4 + [R]):
        B.hlq_expert_gemm(W, torch.tensor(off, dtype=torch.int32, device="cuda"), X, out[4:4 + R])
        torch.cuda.synchronize()
        assert bool((out[:4] == 3).all()) and bool((out[4 + R:] == 3).all())
    check(out[4:4 + R], x, w[-N:], False)


@pytest.mark.parametrize("gated", [False, True])
def test_many_experts_of_few_rows(gated):
    # weights enough that their way from memory decides
    E, N, K, T = 64, 2048, 1024, 500
    g = torch.Generator("cuda").manual_seed(9)
    counts = torch.randint(0, 200, (E,), device="cuda", generator=g)
    counts[:6] = torch.tensor([0, 1, 64, 65, 128, 129])
    off = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), counts.cumsum(0)]).int()
    R = int(off[-1])
    rows = torch.randint(0, T, (R,), dtype=torch.int32, device="cuda", generator=g)
    W, w = mx4(E * N, K, 3, K**-0.5)
    X, x = mx4(T, K, 4)
    y = B.hlq_expert_gemm(W, off, X, rows=rows, gated=gated, out_dtype=torch.bfloat16)
    at = 0
    for e, n in enumerate(counts.tolist()):
        if n:
            check(y[at:at + n], x[rows[at:at + n].long()], w[e * N:(e + 1) * N], gated)
        at += n


# the same where K is long enough for the largest tiles by its own
@pytest.mark.parametrize("dtype", list(HALF_ULP), ids=str)
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("at,room", [(0, 0), (3, 5), (64, 64)])
def test_strides_of_longer_rows(at, room, gated, dtype):
    M, N, K = 4010, 4032, 1500
    cols = N // 2 if gated else N
    W, w = mx4(N, K, 5, K**-0.5)
    X, x = mx4(M, K, 6)
    out = torch.full((M + 2, at + cols + room), 5.0, dtype=dtype, device="cuda")
    y = out[1:1 + M, at:at + cols]
    B.hlq_mx4_gemm(W, X, y, gated=gated)
    check(y, x, w, gated)
    y[:] = 5.0
    assert bool((out == 5).all())


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("counts", [[7300], [1, 7299], [2000, 0, 3000, 2400], [7300, 100, 0, 0], [1850, 1850, 1850, 1850]], ids=str)
def test_expert_product_of_longer_rows(counts, gated):
    E, R, N, K, T = len(counts), sum(counts), 4096, 1500, 3000
    g = torch.Generator("cuda").manual_seed(R + E)
    rows = torch.randint(0, T, (R,), dtype=torch.int32, device="cuda", generator=g)
    W, w = mx4(E * N, K, 3, K**-0.5)
    X, x = mx4(T, K, 4)
    off = torch.tensor([0] + counts, dtype=torch.int32, device="cuda").cumsum(0).int()
    y = B.hlq_expert_gemm(W, off, X, rows=rows, gated=gated, out_dtype=torch.bfloat16)
    at = 0
    for e, n in enumerate(counts):
        if n:
            check(y[at:at + n], x[rows[at:at + n].long()], w[e * N:(e + 1) * N], gated)
        at += n


@pytest.mark.parametrize("gated", [False, True])
def test_more_experts_of_few_longer_rows(gated):
    E, N, K, T = 24, 4096, 2048, 500
    g = torch.Generator("cuda").manual_seed(10)
    counts = torch.randint(0, 200, (E,), device="cuda", generator=g)
    counts[:8] = torch.tensor([0, 1, 64, 65, 128, 129, 256, 257])
    off = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), counts.cumsum(0)]).int()
    R = int(off[-1])
    rows = torch.randint(0, T, (R,), dtype=torch.int32, device="cuda", generator=g)
    W, w = mx4(E * N, K, 3, K**-0.5)
    X, x = mx4(T, K, 4)
    y = B.hlq_expert_gemm(W, off, X, rows=rows, gated=gated, out_dtype=torch.float32)
    at = 0
    for e, n in enumerate(counts.tolist()):
        if n:
            check(y[at:at + n], x[rows[at:at + n].long()], w[e * N:(e + 1) * N], gated)
        at += n
