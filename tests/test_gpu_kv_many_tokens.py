"""More tokens than one launch has wavefronts for: 2^26 and a few, rows of 8 values.  Rows at the ends of launches against calls of those rows alone."""
import pytest
import torch

from paper_2510_19482_amd import binding as B

pytestmark = pytest.mark.gpu


def test_rotary_write_and_read_of_many_tokens():
    T, D = (1 << 26) + 37, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty((T, 1, D), dtype=torch.bfloat16, device="cuda")
    for at in range(0, T, 1 << 24):
        part = x[at:at + (1 << 24)]
        part.copy_(torch.randn(part.shape, device="cuda", generator=g))
    positions = torch.arange(T, dtype=torch.int32, device="cuda")
    rotary = B.Rotary(B.rotary_frequencies(D))
    some = torch.tensor([0, 1, 4095, (1 << 26) - 6, (1 << 26) - 5, (1 << 26) - 4, (1 << 26) - 3, (1 << 26) - 1, 1 << 26, T - 2, T - 1], device="cuda")
    few, places = x[some].contiguous(), positions[some].contiguous()
    want = B.hlq_rotary(few, places, rotary)
    assert torch.equal(B.hlq_rotary(x, positions, rotary)[some], want)
    kv = B.alloc_kv_cache(-(-T // 1024), 1024, 1, D, torch.bfloat16)
    q = B.hlq_kv_write(kv, x, x, positions.long(), rotary, positions, q=x)
    assert torch.equal(q[some], want)
    del q
    k, v = B.hlq_kv_read(kv, positions.long(), dtype=torch.bfloat16)
    assert torch.equal(k[some], want) and torch.equal(v[some], few)
    assert torch.equal(v, x)
