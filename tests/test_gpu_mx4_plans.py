"""Products of microscaled 4-bit matrices on every kernel, tile and cut of K, with operands whose results are exact: any codes, scales 2^-1
and 1, so a product is a multiple of 1/16 and a sum of up to 400000 of them, whose size is that of a random walk, far below 2^20.  Every order
of fp32 sums gives it.  A plain result is therefore the sum itself, rounded once to its type.  Gated: the sums are exact, and the silu of one
times the other is within (16 + |g|) 2^-23 of its own size (the exponential's argument and the operations around it), then rounded once."""
import pytest
import torch

from mx4_plans import INSIDE, PLANS
from paper_2510_19482_amd import binding as B

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF_ULP = {torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8, torch.float32: 2.0**-24}
SMALLEST = {torch.float16: 2.0**-25, torch.bfloat16: 2.0**-126, torch.float32: 2.0**-126}
COUNTERS = 131064


def matrix(rows, K, g, low=0):
    """Random codes with scales 2^(low - 1) and 2^low."""
    codes = torch.randint(0, 256, (rows, (K + 1) // 2), dtype=torch.uint8, device="cuda", generator=g)
    scales = torch.randint(126 + low, 128 + low, (rows, (K + 31) // 32), dtype=torch.uint8, device="cuda", generator=g)
    return B.hlq_mx4_pack(codes, scales, K)


def values(m):
    return B.hlq_mx4_dequantize(m).double()


def product(a, w, gated):
    """The result, and what it may be off before its rounding."""
    p = a @ w.T.contiguous()
    if not gated:
        return p, torch.zeros(())
    h = p.shape[1] // 2
    g, u = p[:, :h], p[:, h:]
    y = g * torch.sigmoid(g) * u
    return y, (16 + g.abs()) * 2.0**-23 * y.abs() + 2.0**-120


def check(y, a, w, gated):
    want, e = product(a, w, gated)
    if not gated:
        assert torch.equal(y, want.to(y.dtype))
        return
    e = e + (want.abs() + e) * HALF_ULP[y.dtype] + SMALLEST[y.dtype]
    past = y.isinf() & (y.sign() == want.sign()) & (want.abs() + e >= torch.finfo(y.dtype).max)
    assert bool((((y.double() - want).abs() <= e) | past).all())


def counts(R, E, g):
    """R rows of E experts: some without, some with one, some that fill a tile."""
    at = torch.randint(0, R + 1, (E - 1,), device="cuda", generator=g)
    at[: E // 4] = at[: E // 4] // 64 * 64
    if E > 3:
        at[1] = at[0]
        at[2] = (at[0] + 1).clamp(max=R)
    return torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), at.sort().values, torch.full((1,), R, device="cuda")]).int()


class Case:
    def __init__(self, R, N, K, E, gated, seed=0):
        g = torch.Generator("cuda").manual_seed(1000 * R + N + 7 * K + E + (seed << 40))
        self.R, self.gated, self.E, self.N = R, gated, E, N
        # gated: sums of about 3, so that silu has its bend
        self.W = matrix(E * N, K, g, -round(0.5 * torch.tensor(float(K)).log2().item()) - 1 if gated else 0)
        self.off = counts(R, E, g) if E > 1 else None
        self.rows = torch.randint(0, max(1, R // 2), (R,), dtype=torch.int32, device="cuda", generator=g) if E > 1 and R % 4 == 1 else None
        self.X = matrix(max(1, R // 2) if self.rows is not None else R, K, g)

    def __call__(self, X=None, Y=None, ws=None, dtype=torch.float32):
        X = self.X if X is None else X
        if self.off is None:
            return B.hlq_mx4_gemm(self.W, X, Y, gated=self.gated, out_dtype=dtype, ws=ws)
        return B.hlq_expert_gemm(self.W, self.off, X, Y, rows=self.rows, gated=self.gated, out_dtype=dtype, ws=ws)

    def check(self, y):
        a = values(self.X)
        a = a if self.rows is None else a[self.rows.long()]
        if self.off is None:
            return check(y, a, values(self.W), self.gated)
        at = self.off.tolist()
        w = values(self.W)
        for e in range(self.E):
            if at[e + 1] > at[e]:
                check(y[at[e]:at[e + 1]], a[at[e]:at[e + 1]], w[e * self.N:(e + 1) * self.N], self.gated)

    def workspace(self):
        return B.alloc_mx4_workspace(self.W, self.X.rows, self.R, self.E)


@pytest.mark.parametrize("key", list(PLANS), ids=str)
def test_product(key):
    for i, shape in enumerate(PLANS[key]):
        print(key, shape, flush=True)
        c = Case(*shape, key[4])
        for dtype in (TYPES[i % 3], TYPES[(i + 1) % 3]):
            y = c(dtype=dtype)
            c.check(y)
        # quantized by a launch before it (a value's 4-bit form is itself): the same bits
        R, N, K, E = shape
        if not B.mx4_plan_query(N, K, R, E, c.X.rows, B.HLQ_F32, key[4]).quantizes:
            assert torch.equal(c(B.hlq_mx4_dequantize(c.X, dtype=TYPES[i % 3]), dtype=dtype), y)


@pytest.mark.parametrize("xtype", TYPES, ids=str)
@pytest.mark.parametrize("parts,gated", list(INSIDE))
def test_product_that_quantizes(parts, gated, xtype):
    for i, shape in enumerate(INSIDE[parts, gated]):
        c = Case(*shape, gated)
        c.check(c(B.hlq_mx4_dequantize(c.X, dtype=xtype), dtype=TYPES[i % 3]))


CUT = [(77, 5000, 11004, 1), (256, 4096, 14336, 1), (300, 700, 11004, 4), (300, 4096, 14336, 1), (100, 2000, 14336, 2), (33, 20, 37885, 1), (107, 8062, 26045, 1), (65, 18, 53835, 33)]


@pytest.mark.parametrize("gated", [False, True])
def test_cut_products_share_a_workspace(gated):
    # partial sums and counters of one product are not another's: what lies in the workspace is NaN to begin with, and the counters are 0 again after each
    cases = [Case(R, N, K, E, gated) for R, N, K, E in CUT]
    for c, (R, _, K, E) in zip(cases, CUT):
        p = B.mx4_plan_query(c.N, K, R, E, c.X.rows, B.HLQ_MX4, gated)
        assert p.kernel == 2 and p.k_parts > 1
    alone = []
    for c in cases:
        y = c(ws=c.workspace())
        c.check(y)
        alone.append(y)
    ws = max((c.workspace() for c in cases), key=lambda w: w.numel())
    ws[131072:] = 255
    for order in (range(len(cases)), reversed(range(len(cases)))):
        for i in order:
            for _ in range(2):
                assert torch.equal(cases[i](ws=ws), alone[i])
                assert not bool(ws[:COUNTERS].any())
        ws[131072:] = 255


@pytest.mark.parametrize("shape", [CUT[0], CUT[2], CUT[5]], ids=str)
def test_cut_products_in_a_graph(shape):
    R, N, K, E = shape
    c, ws = Case(R, N, K, E, False), None
    ws, y = c.workspace(), torch.zeros((R, N), device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c(Y=y, ws=ws)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        c(Y=y, ws=ws)
        c(Y=y, ws=ws)
    for i in range(4):
        c.X.blob.copy_(matrix(c.X.rows, K, torch.Generator("cuda").manual_seed(i)).blob)
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        c.check(y)
        replayed = y.clone()
        assert torch.equal(c(ws=c.workspace()), replayed)
        assert not bool(ws[:COUNTERS].any())
