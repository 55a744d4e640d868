"""Sizes and refusals of the microscaled 4-bit matrices and the expert block: decided on the host, nothing is launched.  And the
oracle against the format's own table."""
import ctypes

import numpy as np
import pytest

from oracle import mx4_oracle as O
from paper_2510_19482_amd import binding as B

OK, NULL, DESC, UNSUPPORTED, SMALL, STRIDE = 0, 1, 2, 3, 4, 5
P = 0x10000     # never dereferenced
BIG = 1 << 40


def test_oracle_values_and_rounding():
    codes = np.arange(16, dtype=np.uint8)
    v = O.dequantize((codes[0::2] | codes[1::2] << 4)[None], np.array([[127]], np.uint8), 16)[0]
    assert v.tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6]
    x = np.array([[4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.01, 7.9, -0.26]])
    assert O.rounded(x)[0].tolist() == [4, 0, 1, 1, 2, 2, 4, 4, 6, 6, -0.5]
    assert O.quantize(np.array([[1.0]]))[1].tolist() == [[125]]
    assert O.quantize(np.array([[np.inf]]))[1].tolist() == [[255]]
    assert O.quantize(np.zeros((1, 33)))[1].tolist() == [[0, 0]]


def test_bytes():
    # 4.25 bits a value, rows padded to 128
    assert B.mx4_bytes(10, 256) == 10 * (128 + 8)
    assert B.mx4_bytes(10, 257) == 10 * 3 * (64 + 4)
    assert B.mx4_bytes(4096, 14336) == 4096 * 14336 * 17 // 32
    assert B.mx4_bytes(0, 5) == 0
    n = ctypes.c_size_t()
    assert B.lib.hlq_mx4_bytes(-1, 5, ctypes.byref(n)) == DESC
    assert B.lib.hlq_mx4_bytes(1, 0, ctypes.byref(n)) == DESC
    assert B.lib.hlq_mx4_bytes(1, (1 << 21) + 1, ctypes.byref(n)) == UNSUPPORTED
    assert B.lib.hlq_mx4_bytes((1 << 31) + 1, 32, ctypes.byref(n)) == UNSUPPORTED
    assert B.lib.hlq_mx4_bytes(1, 32, None) == NULL


def test_quantize_refusals():
    q = B.lib.hlq_mx4_quantize
    assert q(2, 64, None, 0, 64, P, BIG, None) == NULL
    assert q(2, 64, P, 0, 64, None, BIG, None) == NULL
    assert q(2, 64, P, 3, 64, P, BIG, None) == UNSUPPORTED
    assert q(2, 64, P, 7, 64, P, BIG, None) == UNSUPPORTED
    assert q(2, 64, P, 0, 63, P, BIG, None) == STRIDE
    assert q(2, 64, P + 1, 0, 64, P, BIG, None) == STRIDE
    assert q(2, 64, P + 2, 1, 64, P, BIG, None) == STRIDE
    assert q(2, 64, P, 0, 64, P + 8, BIG, None) == STRIDE
    assert q(2, 64, P, 0, 64, P, 2 * 68 - 1, None) == SMALL
    assert q(-1, 64, P, 0, 64, P, BIG, None) == DESC
    assert q(0, 64, None, 0, 64, None, 0, None) == OK
    d = B.lib.hlq_mx4_dequantize
    assert d(2, 64, None, P, 0, 64, None) == NULL
    assert d(2, 64, P, None, 0, 64, None) == NULL
    assert d(2, 64, P, P, 3, 64, None) == UNSUPPORTED
    assert d(2, 64, P, P, 0, 63, None) == STRIDE
    assert d(2, 64, P, P + 1, 0, 64, None) == STRIDE
    assert B.lib.hlq_mx4_pack(2, 64, None, 32, P, 2, P, BIG, None) == NULL
    assert B.lib.hlq_mx4_pack(2, 64, P, 32, None, 2, P, BIG, None) == NULL
    assert B.lib.hlq_mx4_pack(2, 64, P, 31, P, 2, P, BIG, None) == STRIDE
    assert B.lib.hlq_mx4_pack(2, 64, P, 32, P, 1, P, BIG, None) == STRIDE
    assert B.lib.hlq_mx4_pack(2, 64, P, 32, P, 2, P, 2 * 68 - 1, None) == SMALL
    assert B.lib.hlq_mx4_unpack(2, 64, None, P, P, None) == NULL
    assert B.lib.hlq_mx4_unpack(2, 64, P, None, None, None) == OK


def gemm(N=64, K=96, W=P, M=40, X=P, xt=0, ldx=96, Y=P, yt=0, ldy=64, ep=0, ws=P, wb=BIG):
    return B.lib.hlq_mx4_gemm(N, K, W, M, X, xt, ldx, Y, yt, ldy, ep, ws, wb, None)


def test_product_refusals():
    assert gemm(W=None) == NULL and gemm(X=None) == NULL and gemm(Y=None) == NULL and gemm(ws=None) == NULL
    assert gemm(N=0) == DESC and gemm(K=0) == DESC and gemm(M=-1) == DESC
    assert gemm(N=63, ep=1, ldy=63) == DESC
    assert gemm(ep=2) == UNSUPPORTED and gemm(xt=4) == UNSUPPORTED and gemm(yt=3) == UNSUPPORTED
    assert gemm(N=(1 << 20) + 1, ldy=1 << 21) == UNSUPPORTED and gemm(K=(1 << 21) + 1, ldx=1 << 22) == UNSUPPORTED
    assert gemm(M=1 << 31) == UNSUPPORTED
    assert gemm(ldx=95) == STRIDE and gemm(ldy=63) == STRIDE and gemm(ep=1, ldy=31) == STRIDE
    assert gemm(W=P + 8) == STRIDE and gemm(X=P + 1) == STRIDE and gemm(xt=1, X=P + 2) == STRIDE and gemm(Y=P + 1) == STRIDE
    assert gemm(xt=3, X=P + 8) == STRIDE and gemm(ws=P + 4) == STRIDE
    assert gemm(wb=B.mx4_workspace_bytes(64, 96, 1, 40, 40) - 257) == SMALL
    assert gemm(M=0, W=None, X=None, Y=None, ws=None) == OK
    n = ctypes.c_size_t()
    assert B.lib.hlq_mx4_workspace_bytes(0, 96, 1, 4, 4, ctypes.byref(n)) == DESC
    assert B.lib.hlq_mx4_workspace_bytes(64, 96, 0, 4, 4, ctypes.byref(n)) == DESC
    assert B.lib.hlq_mx4_workspace_bytes(64, 96, 1, -1, 4, ctypes.byref(n)) == DESC
    assert B.lib.hlq_mx4_workspace_bytes(64, 96, 1, 4, 4, None) == NULL


def experts(E=4, N=64, K=96, W=P, off=P, rows=P, R=40, T=20, X=P, xt=0, ldx=96, Y=P, yt=0, ldy=64, ep=0, ws=P, wb=BIG):
    return B.lib.hlq_expert_gemm(E, N, K, W, off, rows, R, T, X, xt, ldx, Y, yt, ldy, ep, ws, wb, None)


def test_expert_product_refusals():
    assert experts(off=None) == NULL and experts(W=None) == NULL and experts(X=None) == NULL and experts(Y=None) == NULL
    assert experts(E=0) == DESC and experts(R=-1) == DESC and experts(T=-1) == DESC
    assert experts(T=0) == DESC and experts(rows=None) == DESC          # fewer rows of x than of the result
    assert experts(E=1025) == UNSUPPORTED
    assert experts(off=P + 2) == STRIDE and experts(rows=P + 1) == STRIDE
    assert experts(R=0, W=None, X=None, Y=None, ws=None) == OK


def test_route_and_combine_refusals():
    def route(T=9, E=8, k=2, x=P, t=1, ld=8, ids=P, w=P, off=P, rows=P, slots=P, ws=P, wb=BIG):
        return B.lib.hlq_route(T, E, k, x, t, ld, 1, ids, w, off, rows, slots, ws, wb, None)
    assert route(k=9) == DESC and route(k=0) == DESC and route(E=0) == DESC and route(T=-1) == DESC
    assert route(E=1025, ld=2000) == UNSUPPORTED and route(E=100, k=65, ld=100) == UNSUPPORTED and route(t=3) == UNSUPPORTED
    assert route(T=1 << 30, ld=8) == UNSUPPORTED
    assert route(ld=7) == STRIDE and route(x=P + 2) == STRIDE and route(ids=P + 1) == STRIDE and route(off=P + 2) == STRIDE
    assert all(route(**{n: None}) == NULL for n in ("x", "ids", "w", "off", "rows", "slots"))
    assert route(T=1000, ws=None) == NULL and route(T=1000, wb=100) == SMALL and route(T=1000, ws=P + 4) == STRIDE

    def combine(T=9, k=2, D=8, R=18, y=P, t=0, ld=8, slots=P, w=P, out=P, ot=0, ldo=8):
        return B.lib.hlq_expert_combine(T, k, D, R, y, t, ld, slots, w, out, ot, ldo, None)
    assert combine(T=-1) == DESC and combine(k=0) == DESC and combine(D=0) == DESC and combine(R=-1) == DESC
    assert combine(k=65) == UNSUPPORTED and combine(t=3) == UNSUPPORTED and combine(ot=3) == UNSUPPORTED
    assert combine(ld=7) == STRIDE and combine(ldo=7) == STRIDE and combine(out=P + 1) == STRIDE and combine(slots=P + 2) == STRIDE
    assert all(combine(**{n: None}) == NULL for n in ("y", "slots", "w", "out"))
    assert combine(T=0, y=None, slots=None, w=None, out=None) == OK


def test_binding_refuses_what_it_cannot_hand_over():
    torch = pytest.importorskip("torch")
    m = B.Mx4(torch.empty(B.mx4_bytes(8, 64), dtype=torch.uint8), 8, 64)
    with pytest.raises(ValueError):
        B.Mx4(torch.empty(10, dtype=torch.uint8), 8, 64)
    with pytest.raises(ValueError):
        B.hlq_mx4_pack(torch.zeros((2, 32), dtype=torch.uint8), torch.zeros((2, 1), dtype=torch.uint8), 64)
    with pytest.raises(TypeError):
        B.hlq_mx4_quantize(torch.zeros((2, 64), dtype=torch.float64))
    with pytest.raises(ValueError):
        B.hlq_mx4_quantize(torch.zeros((64, 2)).T)
    with pytest.raises(ValueError):
        B.hlq_mx4_quantize(torch.zeros((2, 64)), m)
    with pytest.raises(ValueError):
        B.hlq_mx4_gemm(m, torch.zeros((2, 65)))
    with pytest.raises(ValueError):
        B.hlq_mx4_gemm(m, torch.zeros((2, 64)), torch.zeros((2, 7)))
    with pytest.raises(ValueError):
        B.hlq_expert_gemm(m, torch.zeros(4, dtype=torch.int32), torch.zeros((2, 64)))       # 8 rows are not 3 matrices
    with pytest.raises(ValueError):
        B.hlq_expert_gemm(m, torch.zeros(3, dtype=torch.int64), torch.zeros((2, 64)))
    with pytest.raises(ValueError):
        B.hlq_expert_combine(torch.zeros((4, 8)), torch.zeros((2, 2), dtype=torch.int64), torch.zeros((2, 2)))


@pytest.mark.parametrize("part", ["hlq_mx4_quantize_kernel", "hlq_mx4_dequantize_kernel", "hlq_mx4_few_kernel", "hlq_mx4_tile_kernel", "hlq_route_top_kernel",
                                  "hlq_route_place_kernel", "hlq_expert_combine_kernel"])
def test_no_scratch_memory(part):
    from test_kernel_resources import kernels
    mine = {n: k for n, k in kernels().items() if part in n}
    assert mine
    assert {n: k[".private_segment_fixed_size"] for n, k in mine.items() if k[".private_segment_fixed_size"]} == {}


def test_no_scratch_memory_in_large_products():
    from test_kernel_resources import kernels
    mine = {n: k for n, k in kernels().items() if "hlq_mx4_big_kernel" in n}
    assert len(mine) == 2 and all(k[".private_segment_fixed_size"] == 0 for k in mine.values())
