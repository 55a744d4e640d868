"""What packed scale bytes stand for at both ends: the lowest, which only types with small exponents hold, and the highest, whose larger values are past
every type.  All sixteen codes of each byte, in each type, against the format's definition rounded once."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as O
from paper_2510_19482_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=str)
def test_values_of_every_byte(dtype):
    K = 32
    codes = np.tile((np.arange(0, 16, 2) | np.arange(1, 16, 2) << 4).astype(np.uint8), (256, 2))
    scales = np.arange(256, dtype=np.uint8)[:, None]
    y = B.hlq_mx4_dequantize(B.hlq_mx4_pack(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), K), dtype=dtype).cpu()
    want = torch.from_numpy(O.dequantize(codes, scales, K))
    info = torch.finfo(dtype)
    past = want.abs() > info.max * (1 + info.eps / 4)
    rounded = torch.where(past, want.sign() * float("inf"), want.to(dtype).double())
    assert torch.equal(torch.isnan(y), torch.isnan(want))
    ok = ~torch.isnan(want)
    assert torch.equal(y.double()[ok], rounded[ok])
    # 2^-128 is there in f32 and bf16, what is past them is infinite from byte 253 on
    if dtype is not torch.float16:
        assert y[0, 1] == 2.0**-128 and not y[:253].isinf().any()
        assert y[253, 5:8].isinf().tolist() == [False, True, True] and y[254, 3:8].isinf().tolist() == [False] + [True] * 4
