#!/usr/bin/env python3
"""The feed-forward part of a decoder layer with experts, in microscaled 4-bit weights and activations:

    route     logits = x Wr^T; the k experts of each token, their weights, tokens grouped by expert
    up        h = silu(gate) up for each token's experts, x gathered by token (gate and up are one matrix per expert)
    down      the experts' outputs, grouped
    combine   their weighted sum for each token

`python examples/expert_block.py` runs a prompt, and decoding from a captured graph, and compares both with the same block by
plain torch on the values that the 4-bit matrices stand for."""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2510_19482_amd import binding as hlq  # noqa: E402


class ExpertBlock:
    """Router weights [E, D] in f32; per expert gate|up [2 F, D] and down [D, F], quantized here."""

    def __init__(self, router, up, down, k: int):
        self.E, self.k = router.shape[0], k
        self.D, self.F = router.shape[1], down.shape[-1]
        self.router = router
        self.up = hlq.hlq_mx4_quantize(up.reshape(self.E * 2 * self.F, self.D))
        self.down = hlq.hlq_mx4_quantize(down.reshape(self.E * self.D, self.F))

    def buffers(self, T: int, dtype=torch.bfloat16):
        """What a call for T tokens writes: made once, so that calls allocate nothing and can be captured."""
        rows = T * self.k

        def new(*shape, dtype=dtype):
            return torch.empty(shape, dtype=dtype, device=self.router.device)

        return dict(logits=new(T, self.E, dtype=torch.float32), route=hlq.alloc_route(T, self.E, self.k), h=new(rows, self.F), y=new(rows, self.D), out=new(T, self.D),
                    up_ws=hlq.alloc_mx4_workspace(self.up, T, rows, self.E), down_ws=hlq.alloc_mx4_workspace(self.down, rows, rows, self.E))

    def __call__(self, x, b):
        torch.mm(x.float(), self.router.T, out=b["logits"])
        r = hlq.hlq_route(b["logits"], self.k, out=b["route"])
        hlq.hlq_expert_gemm(self.up, r.offsets, x, b["h"], rows=r.rows, gated=True, ws=b["up_ws"])
        hlq.hlq_expert_gemm(self.down, r.offsets, b["h"], b["y"], ws=b["down_ws"])
        return hlq.hlq_expert_combine(b["y"], r.slots, r.weights, b["out"])


def plain(block: ExpertBlock, x):
    """The block token by expert in f32, on the same 4-bit values; what is quantized there is quantized here."""
    def rounded(v):
        return hlq.hlq_mx4_dequantize(hlq.hlq_mx4_quantize(v))

    up = hlq.hlq_mx4_dequantize(block.up).view(block.E, 2 * block.F, block.D)
    down = hlq.hlq_mx4_dequantize(block.down).view(block.E, block.D, block.F)
    chosen, ids = torch.sort(x.float() @ block.router.T, dim=-1, descending=True, stable=True)
    weights = torch.softmax(chosen[:, :block.k], -1)
    out = torch.zeros((x.shape[0], block.D), device=x.device)
    a = rounded(x)
    for e in range(block.E):
        t, i = (ids[:, :block.k] == e).nonzero(as_tuple=True)
        if len(t):
            g, u = (a[t] @ up[e].T).chunk(2, -1)
            h = rounded((torch.nn.functional.silu(g) * u).to(x.dtype))
            out[t] += weights[t, i, None] * (h @ down[e].T).to(x.dtype).float()
    return out


def random_block(E: int, k: int, D: int, F: int, seed: int = 0) -> ExpertBlock:
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std):
        return torch.randn(shape, device="cuda", generator=g).mul_(std)

    return ExpertBlock(normal(E, D, std=D**-0.5), normal(E, 2 * F, D, std=D**-0.5).bfloat16(), normal(E, D, F, std=F**-0.5).bfloat16(), k)


def difference(block: ExpertBlock, x, out) -> float:
    """Norm of the difference to the plain form over the norm of its result."""
    want = plain(block, x)
    return float((out.float() - want).norm() / want.norm())


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("experts", 32), ("choices", 4), ("hidden", 4096), ("ffn", 2048), ("prompt", 2048), ("batch", 8)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args()
    block = random_block(a.experts, a.choices, a.hidden, a.ffn)

    x = torch.randn((a.prompt, a.hidden), device="cuda").bfloat16()
    b = block.buffers(a.prompt)
    print(f"prompt of {a.prompt} tokens: {microseconds(lambda: block(x, b)):.0f} us, difference to the plain form {difference(block, x, block(x, b)):.1e}")

    x = torch.randn((a.batch, a.hidden), device="cuda").bfloat16()
    b = block.buffers(a.batch)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        block(x, b)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = block(x, b)
    graph.replay()
    torch.cuda.synchronize()
    print(f"decoding {a.batch} tokens from a graph: {microseconds(graph.replay):.0f} us, difference to the plain form {difference(block, x, out):.1e}")


def microseconds(call, n: int = 20) -> float:
    for _ in range(3):
        call()
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    for _ in range(n):
        call()
    end.record()
    end.synchronize()
    return start.elapsed_time(end) / n * 1e3


if __name__ == "__main__":
    main()
