"""A matrix whose blob is replaced: products take the weights that stand there at the time of the call, and none that are not on the GPU."""
import pytest
import torch

from paper_2510_19482_amd import binding as B

pytestmark = pytest.mark.gpu


def test_products_follow_the_blob():
    N, K, M = 96, 160, 5
    first, second = (B.hlq_mx4_quantize(torch.randn(N, K, device="cuda")) for _ in range(2))
    x = torch.randn(M, K, device="cuda")
    want = B.hlq_mx4_gemm(second, x)
    assert not torch.equal(B.hlq_mx4_gemm(first, x), want)
    assign, data = B.Mx4(first.blob.clone(), N, K), B.Mx4(first.blob.clone(), N, K)
    assign.blob = second.blob.clone()
    data.blob.data = second.blob.clone()
    off = torch.tensor([0, 0, M], dtype=torch.int32, device="cuda")
    for m in (assign, data):
        assert torch.equal(B.hlq_mx4_gemm(m, x), want)
        assert torch.equal(B.hlq_mx4_dequantize(m), B.hlq_mx4_dequantize(second))
        assert torch.equal(B.hlq_expert_gemm(m, off, x), B.hlq_expert_gemm(second, off, x))
        assert torch.equal(B.hlq_mx4_unpack(m)[0], B.hlq_mx4_unpack(second)[0])
        m.blob = m.blob.cpu()
        for call in (lambda: B.hlq_mx4_gemm(m, x), lambda: B.hlq_mx4_dequantize(m), lambda: B.hlq_expert_gemm(m, off, x), lambda: B.hlq_mx4_unpack(m),
                     lambda: B.hlq_mx4_quantize(torch.zeros(N, K, device="cuda"), m)):
            with pytest.raises(ValueError):
                call()
        m.blob = m.blob.cuda()
        assert torch.equal(B.hlq_mx4_gemm(m, x), want)
