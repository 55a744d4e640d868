"""Microscaled 4-bit matrices on the GPU against the 64-bit oracle: quantization bit for bit, products within the rounding of
their fp32 sums, which is derived here:

a block's sum of 32 products is exact, and each of the row's ceil(K / 32) block sums is added once to an fp32 sum (a few more
additions join shares of K), so with u = 2^-23 an addition (the matrix core may cut off instead of rounding) the error is at most
(blocks + 32) u times the sum of the products' magnitudes; the result is then rounded once to its type."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as O
from paper_2510_19482_amd import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
HALF_ULP = {"f16": 2.0**-11, "bf16": 2.0**-8, "f32": 2.0**-24}   # of 11, 8 and 24 significant bits
SMALLEST = {"f16": 2.0**-25, "bf16": 2.0**-126, "f32": 2.0**-126}


def rng(*key):
    return np.random.default_rng([ord(c) for c in repr(key)])


def activations(rows, K, *key):
    r = rng("x", rows, K, *key)
    x = r.normal(size=(rows, K))
    x[:, r.permutation(K)[:max(1, K // 100)]] *= 20
    return x


def on_gpu(x, dtype):
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(TYPES[dtype]).cuda()


def host(t):
    return t.double().cpu().numpy()


def stored(rows, K, *key):
    """Weights in the exchange form, with scales over many powers of two."""
    w = rng("w", rows, K, *key).normal(size=(rows, K)) * np.exp2(rng("s", *key).integers(-6, 7, size=(rows, 1)))
    return O.quantize(w)


def matrix(codes, scales, K):
    return B.hlq_mx4_pack(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), K)


def product_bound(a, w, gated, dtype):
    """Largest error of each result, and the results."""
    p, mag = a @ w.T, np.abs(a) @ np.abs(w).T
    e = (-(-a.shape[1] // 32) + 32) * 2.0**-23 * mag
    if gated:
        h = p.shape[1] // 2
        y = O.gate(p)
        g, u = np.abs(p[:, :h]), np.abs(p[:, h:])
        # |silu'| <= 1.1, |silu(g)| <= |g|; the exponential's argument and the four operations around it
        e = 1.1 * e[:, :h] * (u + e[:, h:]) + g * e[:, h:] + (16 + g) * 2.0**-23 * np.abs(y) + 2.0**-120
    else:
        y = p
    return y, e + HALF_ULP[dtype] * (np.abs(y) + e) + SMALLEST[dtype]


def check(got, a, w, gated, dtype):
    y, e = product_bound(a, w, gated, dtype)
    got = host(got)
    assert got.shape == y.shape
    # what is past the type's largest rounds to infinity
    limit = float(torch.finfo(TYPES[dtype]).max) * (1 + HALF_ULP[dtype])
    with np.errstate(invalid="ignore"):
        past = np.isinf(got) & (np.sign(got) == np.sign(y)) & (np.abs(y) + e >= limit)
        bad = ~(np.abs(got - y) <= e) & ~past
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, worst {np.max(np.abs(got - y) / e):.3g} times the bound at {np.argwhere(bad)[:3].tolist()}"


# ---- quantization ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,K", [(1, 1), (1, 32), (3, 31), (2, 33), (5, 255), (4, 256), (7, 257), (130, 1000), (33, 4096), (2, 11004)])
def test_quantize_is_the_oracles(rows, K, dtype):
    x = on_gpu(activations(rows, K), dtype)
    m = B.hlq_mx4_quantize(x)
    codes, scales = B.hlq_mx4_unpack(m)
    want = O.quantize(host(x))
    assert np.array_equal(scales.cpu().numpy(), want[1])
    assert np.array_equal(codes.cpu().numpy(), want[0])
    assert np.array_equal(host(B.hlq_mx4_dequantize(m)), O.dequantize(*want, K))


@pytest.mark.parametrize("dtype", list(TYPES))
def test_quantize_ties_extremes_and_what_is_not_a_number(dtype):
    info = torch.finfo(TYPES[dtype])
    rows = []
    for top in (4.0, 5.0, 6.0, 7.0, 7.96875):     # the block's largest: the scale stays, above 5 it is 6
        rows.append([top] + [s * v for v in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 0.2490234375, 0.25390625, 0.0) for s in (1, -1)])
    x = np.zeros((len(rows) + 8, 96))
    for i, r in enumerate(rows):
        x[i, 32:32 + len(r)] = r
    n = len(rows)
    x[n, 40] = info.max
    x[n + 1, :96] = info.min
    x[n + 2, 3] = info.tiny
    x[n + 3, 64:70] = info.smallest_normal / 2   # subnormal
    x[n + 3, 3] = info.smallest_normal * (info.eps if dtype != "bf16" else 1 / 64)
    x[n + 4, 5], x[n + 4, 6] = np.inf, 1.0
    x[n + 5, 33], x[n + 5, 34] = np.nan, 2.0
    x[n + 6, 95] = -np.inf
    x[n + 7, :] = -0.0
    t = on_gpu(x, dtype)
    m = B.hlq_mx4_quantize(t)
    codes, scales = (v.cpu().numpy() for v in B.hlq_mx4_unpack(m))
    want = O.quantize(host(t))
    assert np.array_equal(scales, want[1])
    values = O.dequantize(codes, scales, 96)
    assert np.array_equal(values, O.dequantize(*want, 96), equal_nan=True)
    got = host(B.hlq_mx4_dequantize(m, dtype=torch.float32))
    assert np.array_equal(got, values.astype(np.float32).astype(np.float64), equal_nan=True)
    assert np.isnan(got[n + 4, :32]).all() and not np.isnan(got[n + 4, 32:]).any()


@pytest.mark.parametrize("dtype", list(TYPES))
def test_quantize_strided_and_unaligned_rows(dtype):
    wide = on_gpu(activations(9, 700), dtype)
    for lo, hi in ((1, 602), (8, 520), (3, 36)):
        view = wide[::2, lo:hi]
        m = B.hlq_mx4_quantize(view)
        want = O.quantize(host(view))
        codes, scales = B.hlq_mx4_unpack(m)
        assert np.array_equal(codes.cpu().numpy(), want[0]) and np.array_equal(scales.cpu().numpy(), want[1])
        y = torch.full((5, 800), 7.0, dtype=TYPES[dtype], device="cuda")
        B.hlq_mx4_dequantize(m, y[:, 11:11 + hi - lo])
        assert (y[:, :11] == 7).all() and (y[:, 11 + hi - lo:] == 7).all()
        assert torch.equal(y[:, 11:11 + hi - lo].double().cpu(), torch.from_numpy(O.dequantize(*want, hi - lo)).to(TYPES[dtype]).double())


@pytest.mark.parametrize("rows,K", [(1, 1), (3, 33), (20, 300), (5, 512), (2, 777)])
def test_pack_and_unpack_are_inverse(rows, K):
    r = rng(rows, K)
    codes = r.integers(0, 256, size=(rows, (K + 1) // 2), dtype=np.uint8)
    if K % 2:
        codes[:, -1] &= 15
    scales = r.integers(0, 256, size=(rows, (K + 31) // 32), dtype=np.uint8)
    c, s = B.hlq_mx4_unpack(matrix(codes, scales, K))
    assert np.array_equal(c.cpu().numpy(), codes) and np.array_equal(s.cpu().numpy(), scales)


def test_pack_takes_rows_with_room_behind_them():
    rows, K = 7, 299
    codes, scales = stored(rows, K)
    wide = torch.full((rows, 200), 255, dtype=torch.uint8, device="cuda")
    wide[:, 5:5 + codes.shape[1]] = torch.from_numpy(codes).cuda()
    many = torch.full((rows, 16), 255, dtype=torch.uint8, device="cuda")
    many[:, :scales.shape[1]] = torch.from_numpy(scales).cuda()
    m = B.hlq_mx4_pack(wide[:, 5:5 + codes.shape[1]], many, K)
    assert torch.equal(m.blob, matrix(codes, scales, K).blob)
    whole = B.hlq_mx4_pack(wide[:, 5:], many, K)               # what stands past K is no value
    assert torch.equal(whole.blob, m.blob)


# ---- products -------------------------------------------------------------------------------------------------------

SHAPES = [(1, 1, 1), (1, 16, 32), (1, 70, 100), (2, 33, 257), (3, 256, 512), (5, 17, 4096), (16, 300, 1000), (17, 48, 288), (31, 129, 640),
          (33, 64, 256), (40, 130, 1056), (64, 256, 256), (65, 200, 300), (100, 513, 768), (128, 128, 1024), (129, 257, 2048), (200, 96, 11004),
          (255, 511, 320), (257, 520, 1300), (300, 1000, 256), (513, 300, 544), (700, 768, 512)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_product(M, N, K, dtype):
    x = on_gpu(activations(M, K), dtype)
    codes, scales = stored(N, K)
    y = B.hlq_mx4_gemm(matrix(codes, scales, K), x)
    assert y.dtype == TYPES[dtype]
    check(y, O.rounded(host(x)), O.dequantize(codes, scales, K), False, dtype)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("M,N,K", [(m, n + n % 2, k) for m, n, k in SHAPES])
def test_gated_product(M, N, K, dtype):
    x = on_gpu(activations(M, K) * 0.3, dtype)
    w = rng("gated", N, K).normal(size=(N, K)) * K**-0.5
    codes, scales = O.quantize(w)
    y = B.hlq_mx4_gemm(matrix(codes, scales, K), x, gated=True)
    check(y, O.rounded(host(x)), O.dequantize(codes, scales, K), True, dtype)


@pytest.mark.parametrize("M", [1, 4, 16, 17, 100, 300])
def test_types_meet_freely_and_a_quantized_operand_gives_the_same(M):
    K, N = 520, 144
    codes, scales = stored(N, K)
    W = matrix(codes, scales, K)
    for xt in TYPES:
        x = on_gpu(activations(M, K), xt)
        q = B.hlq_mx4_quantize(x)
        for yt in TYPES:
            y = B.hlq_mx4_gemm(W, x, out_dtype=TYPES[yt])
            assert torch.equal(y, B.hlq_mx4_gemm(W, q, out_dtype=TYPES[yt]))
            check(y, O.rounded(host(x)), O.dequantize(codes, scales, K), False, yt)


@pytest.mark.parametrize("M", [1, 7, 40, 300])
def test_strides_and_what_lies_beside_the_results(M):
    K, N = 332, 150
    codes, scales = stored(N, K)
    W = matrix(codes, scales, K)
    wide = on_gpu(activations(M, 3 * K), "bf16")
    for at in (1, 8):
        x = wide[:, at:at + K]
        for yt in TYPES:
            for gated in (False, True):
                cols = N // 2 if gated else N
                out = torch.full((M + 2, cols + 13), 5.0, dtype=TYPES[yt], device="cuda")
                B.hlq_mx4_gemm(W, x, out[1:1 + M, 3:3 + cols], gated=gated)
                check(out[1:1 + M, 3:3 + cols], O.rounded(host(x)), O.dequantize(codes, scales, K), gated, yt)
                out[1:1 + M, 3:3 + cols] = 5.0
                assert (out == 5).all()


@pytest.mark.parametrize("M", [1, 20, 300])
def test_infinities_and_nan_stay_in_their_rows_and_columns(M):
    K, N = 700, 300
    x = activations(M, K)
    x[0, 650] = np.inf
    x[M - 1, 3] = np.nan
    codes, scales = stored(N, K)
    scales[7, 2] = 255
    t = on_gpu(x, "f32")
    y = host(B.hlq_mx4_gemm(matrix(codes, scales, K), t))
    nan = np.zeros((M, N), bool)
    nan[[0, M - 1]] = True
    nan[:, 7] = True
    assert np.array_equal(np.isnan(y), nan)


def test_scales_far_apart():
    # a block 2^40 above another: what the smaller gives is still added as fp32 adds it
    K, N, M = 256, 64, 20
    x = activations(M, K)
    x[:, :32] *= 2.0**40
    codes, scales = stored(N, K)
    t = on_gpu(x, "f32")
    check(B.hlq_mx4_gemm(matrix(codes, scales, K), t), O.rounded(host(t)), O.dequantize(codes, scales, K), False, "f32")


def test_no_rows():
    W = matrix(*stored(40, 96), 96)
    assert B.hlq_mx4_gemm(W, torch.empty((0, 96), device="cuda")).shape == (0, 40)
    assert B.hlq_mx4_quantize(torch.empty((0, 96), device="cuda")).rows == 0
    off = torch.zeros(5, dtype=torch.int32, device="cuda")
    assert B.hlq_expert_gemm(W, off, torch.empty((0, 96), device="cuda")).shape == (0, 10)


# ---- products grouped by expert -------------------------------------------------------------------------------------

def group(counts):
    return torch.tensor(np.concatenate(([0], np.cumsum(counts))), dtype=torch.int32, device="cuda")


COUNTS = [[1], [0, 3], [2, 0, 0, 1], [1] * 8, [0, 0, 5, 0], [16, 17, 1, 0, 33], [64, 0, 65, 3, 128], [200, 1, 0, 57, 256, 300], [0, 700, 1, 1], [3] * 70]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("counts", COUNTS, ids=str)
def test_expert_product(counts, gather, gated):
    E, R = len(counts), sum(counts)
    N, K = 90, 300
    T = max(1, R // 2) if gather else R
    x = on_gpu(activations(T, K) * 0.3, "bf16")
    rows = torch.from_numpy(rng("rows", R, E).integers(0, T, size=R).astype(np.int32)).cuda() if gather else None
    codes, scales = O.quantize(rng("we", E).normal(size=(E * N, K)) * K**-0.5)
    y = B.hlq_expert_gemm(matrix(codes, scales, K), group(counts), x, rows=rows, gated=gated, out_dtype=torch.float32)
    a = O.rounded(host(x))
    a = a[rows.cpu().numpy()] if gather else a
    w = O.dequantize(codes, scales, K)
    at = 0
    for e, n in enumerate(counts):
        if n:
            check(y[at:at + n], a[at:at + n], w[e * N:(e + 1) * N], gated, "f32")
        at += n


@pytest.mark.parametrize("R", [6, 40, 900])
def test_rows_past_the_experts_are_not_written_and_bad_indexes_stay_inside(R):
    E, N, K, T = 3, 64, 128, 5
    used = R - R // 3
    counts = [used // 2, 0, used - used // 2]
    x = on_gpu(activations(T, K), "f32")
    rows = rng(R).integers(0, T, size=R).astype(np.int32)
    wild = rows.copy()
    rows[1], wild[1] = 0, -4
    rows[2], wild[2] = T - 1, 1 << 30
    wild[used:] = -1
    codes, scales = stored(E * N, K)
    out = torch.full((R, N), 3.0, device="cuda")
    B.hlq_expert_gemm(matrix(codes, scales, K), group(counts), x, out, rows=torch.from_numpy(wild).cuda())
    assert (out[used:] == 3).all()
    a, w = O.rounded(host(x))[rows], O.dequantize(codes, scales, K)
    check(out[:counts[0]], a[:counts[0]], w[:N], False, "f32")
    check(out[counts[0]:used], a[counts[0]:used], w[2 * N:], False, "f32")
    # offsets that point past the rows count as their end
    off = group(counts)
    off[3] = 1 << 30
    B.hlq_expert_gemm(matrix(codes, scales, K), off, x, out, rows=torch.from_numpy(rows).cuda())
    check(out[counts[0]:], a[counts[0]:], w[2 * N:], False, "f32")


@pytest.mark.parametrize("R,N,K", [(40, 64, 128), (700, 300, 256), (90, 200, 2000)])
def test_offsets_that_overlap_write_rows_only(R, N, K):
    # offsets are the caller's to keep ascending; whatever they hold, only the R rows of the result are written
    E = 9
    x = on_gpu(activations(R, K), "bf16")
    codes, scales = stored(E * N, K)
    W = matrix(codes, scales, K)
    out = torch.full((R + 8, N), 3.0, device="cuda")
    for off in ([0, R, 0, R, 0, R, 0, R, 0, R], [-5, R + 5, -5, 1 << 30, -(1 << 30), R, R, 0, 0, R], [R] * 10, [0] * 9 + [R]):
        B.hlq_expert_gemm(W, torch.tensor(off, dtype=torch.int32, device="cuda"), x, out[4:4 + R])
        torch.cuda.synchronize()
        assert (out[:4] == 3).all() and (out[4 + R:] == 3).all()
    # the last: everything is the last expert's
    check(out[4:4 + R], O.rounded(host(x)), O.dequantize(codes, scales, K)[-N:], False, "f32")


# ---- router and combination -----------------------------------------------------------------------------------------

def routed(r):
    return [v.cpu().numpy() for v in (r.ids, r.weights, r.offsets, r.rows, r.slots)]


def check_route(logits, k, renorm, dtype):
    t = on_gpu(logits, dtype)
    got = routed(B.hlq_route(t, k, renorm))
    want = O.route(host(t), k, renorm)
    for name, g, w in zip(("ids", "", "offsets", "rows", "slots"), got, want):
        if name:
            assert np.array_equal(g, w), name
    # fp32: the difference to the largest logit, the exponential (2 ulp), a sum of up to E terms
    x = host(t)
    span = np.nan_to_num(np.abs(np.where(np.isfinite(x), x, 0)).max(-1, keepdims=True) * 2, posinf=1e30)
    bound = want[1] * np.minimum(1.0, (span + x.shape[1] + 16) * 2.0**-23) + 2.0**-126
    assert (np.abs(got[1] - want[1]) <= bound).all()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 8, 2), (3, 4, 4), (32, 64, 6), (63, 65, 8), (64, 128, 1), (65, 60, 4), (200, 256, 8), (129, 384, 3),
                                   (70, 1024, 64), (1000, 7, 2)])
def test_route(T, E, k, renorm, dtype):
    check_route(rng("route", T, E, k).normal(size=(T, E)), k, renorm, dtype)


@pytest.mark.parametrize("T", [5, 300])
def test_route_ties_masks_and_infinities(T):
    E, k = 40, 6
    r = rng("masks", T)
    x = r.integers(-2, 3, size=(T, E)).astype(float)         # ties everywhere
    x[r.random((T, E)) < 0.3] = -np.inf
    x[0] = -np.inf                                           # a row that nothing is left of
    x[1] = -np.inf
    x[1, 7] = 2.0                                            # fewer than k
    x[2] = np.nan
    x[2, 3] = -1.0
    x[3, 5], x[3, 6] = np.inf, np.inf
    x[4] = float(np.finfo(np.float32).min)                   # the type's lowest value is a number
    x[4, 9] = 0.0
    x[4, 10] = -0.0
    check_route(x, k, True, "f32")
    check_route(x, k, False, "f32")
    x[4] = float(torch.finfo(torch.float16).min)
    check_route(x, k, True, "f16")


def test_route_many_chunks_and_strided_logits():
    # over 512 chunks of 32 tokens the counts are scanned by a kernel of their own
    T, E, k = 32 * 600 + 5, 10, 3
    wide = on_gpu(rng("many").normal(size=(T, E + 3)), "bf16")
    t = wide[:, 2:2 + E]
    ids, w, offsets, rows, slots = routed(B.hlq_route(t, k))
    x = host(t)
    want = np.argsort(-x, axis=1, kind="stable")[:, :k]
    assert np.array_equal(ids, want)
    order = np.argsort(want.ravel(), kind="stable")
    assert np.array_equal(rows, order // k)
    assert np.array_equal(offsets, np.concatenate(([0], np.cumsum(np.bincount(want.ravel(), minlength=E)))))
    assert np.array_equal(slots.ravel()[order], np.arange(T * k))
    assert B.hlq_route(torch.empty((0, 6), device="cuda"), 2).offsets.eq(0).all()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T,k,D", [(1, 1, 1), (1, 4, 64), (5, 8, 100), (64, 3, 4096), (33, 5, 1001), (3, 64, 8)])
def test_combine(T, k, D, dtype):
    r = rng("combine", T, k, D)
    y = on_gpu(r.normal(size=(T * k, D)), dtype)
    slots = r.permutation(T * k).reshape(T, k).astype(np.int32)
    slots[r.random((T, k)) < 0.2] = -1
    if T > 2:
        slots[1] = -1                                        # nothing to add: zeros
        slots[2, 0] = T * k + 5                              # outside: nothing
        y[0] = float("nan")                                  # in no token's sum unless chosen
        slots[slots == 0] = -1
    w = r.random((T, k)).astype(np.float32)
    out = host(B.hlq_expert_combine(y, torch.from_numpy(slots).cuda(), torch.from_numpy(w).cuda()))
    yy = np.where(np.isnan(host(y)), 0.0, host(y))
    ok = (slots >= 0) & (slots < T * k)
    terms = np.where(ok[..., None], w[..., None].astype(np.float64) * yy[np.where(ok, slots, 0)], 0.0)
    want, mag = terms.sum(1), np.abs(terms).sum(1)
    assert (np.abs(out - want) <= k * 2.0**-23 * mag + HALF_ULP[dtype] * np.abs(want) * 1.01 + SMALLEST[dtype]).all()


# ---- as a program runs them -----------------------------------------------------------------------------------------

@pytest.mark.parametrize("T", [1, 3, 40, 600])
def test_block_on_another_stream_and_in_a_graph(T):
    E, k, D, F = 12, 3, 320, 192
    x, logits = on_gpu(activations(T, D), "bf16"), on_gpu(rng("l", T).normal(size=(T, E)), "f32")
    up = matrix(*O.quantize(rng("up").normal(size=(E * 2 * F, D)) * D**-0.5), D)
    down = matrix(*O.quantize(rng("down").normal(size=(E * D, F)) * F**-0.5), F)
    route = B.alloc_route(T, E, k)
    h, y, out = (torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in ((T * k, F), (T * k, D), (T, D)))
    w1, w2 = B.alloc_mx4_workspace(up, T, T * k, E), B.alloc_mx4_workspace(down, T * k, T * k, E)

    def block():
        B.hlq_route(logits, k, out=route)
        B.hlq_expert_gemm(up, route.offsets, x, h, rows=route.rows, gated=True, ws=w1)
        B.hlq_expert_gemm(down, route.offsets, h, y, ws=w2)
        B.hlq_expert_combine(y, route.slots, route.weights, out)

    block()
    torch.cuda.synchronize()
    first = out.clone()
    assert torch.isfinite(first).all() and first.abs().max() > 0
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        out.zero_()
        block()
    s.synchronize()
    assert torch.equal(out, first)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        block()
    for i in range(4):
        x.copy_(on_gpu(activations(T, D, i), "bf16"))
        logits.copy_(on_gpu(rng("l", T, i).normal(size=(T, E)), "f32"))
        g.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        out.zero_()
        block()
        torch.cuda.synchronize()
        assert torch.equal(out, replayed)
