"""The example that runs the expert block's operators together, against its plain form; and calls on a stream of their own."""
import importlib.util
import os

import pytest
import torch

from paper_2510_19482_amd import binding as B

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("expert_block", os.path.join(ROOT, "examples", "expert_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("T", [1, 7, 64, 700])
@pytest.mark.parametrize("E,k,D,F", [(8, 2, 256, 128), (20, 4, 320, 500)])
def test_block_is_the_plain_forms(E, k, D, F, T):
    # What differs: fp32 sums in another order, which can move a value of h or y by one bf16 step (2^-8 of it) and such a value of h
    # by one step of its 4-bit form (at most a third of it, for the few whose bf16 neighbours round apart: a 4-bit value has 2 bits, bf16
    # 8, so one such move in 64 crosses a border).  Per value of h at most 2^-8 / 64 of them move, by 1/3: far below a bf16 step a result.
    ex = example()
    block = ex.random_block(E, k, D, F)
    x = torch.randn((T, D), device="cuda", generator=torch.Generator(device="cuda").manual_seed(T)).bfloat16()
    out = block(x, block.buffers(T))
    assert ex.difference(block, x, out) <= 2.0**-7


def test_calls_on_a_stream_of_their_own():
    # no buffer given: what a call makes belongs to the stream it runs on, also while the current one is busy with other work
    M, N, K = 40, 300, 640
    x = torch.randn((M, K), device="cuda").bfloat16()
    W = B.hlq_mx4_quantize(torch.randn((N, K), device="cuda"))
    E = 6
    logits = torch.randn((M, E), device="cuda")
    torch.cuda.synchronize()

    def calls(stream):
        r = B.hlq_route(logits, 2, stream=stream)
        y = B.hlq_expert_gemm(W, r.offsets, x, rows=r.rows, stream=stream)
        return [B.hlq_mx4_gemm(W, x, stream=stream), B.hlq_mx4_dequantize(B.hlq_mx4_quantize(x, stream=stream), stream=stream), y,
                B.hlq_expert_combine(y, r.slots, r.weights, stream=stream)]

    want = calls(None)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(3):
        busy = torch.randn((2048, 2048), device="cuda")
        for _ in range(10):
            busy = busy @ busy
            junk = torch.full((1 << 20,), 7, dtype=torch.uint8, device="cuda")
            del junk
        got = calls(s)
        s.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, want))
    torch.cuda.synchronize()
