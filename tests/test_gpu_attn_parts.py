"""Inputs and outputs that are parts of one buffer, side by side in each token's row, head by head, or every other token: the same bits as with buffers of their own."""
import pytest
import torch

from attn_util import TYPES, rng, rounded
from paper_2510_19482_amd import binding as B

pytestmark = pytest.mark.gpu


def room(layout, T, H, D, dtype):
    """Two arrays [T, H, D] in one buffer."""
    n = lambda *s: torch.full(s, 7.0, dtype=TYPES[dtype], device="cuda")   # noqa: E731
    if layout == "side by side":
        both = n(T, 2 * H, D)
        return both[:, :H], both[:, H:]
    if layout == "heads in turn":
        both = n(T, H, 2, D)
        return both[:, :, 0], both[:, :, 1]
    if layout == "tokens in turn":
        both = n(T, 2, H, D)
        return both[:, 0], both[:, 1]
    both = n(2, H, T, D)           # head by head
    return both[0].transpose(0, 1), both[1].transpose(0, 1)


LAYOUTS = ["side by side", "heads in turn", "tokens in turn", "head by head"]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,dims,interleaved", [(64, 64, False), (72, 20, False), (64, 6, True)])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_rotary_and_write(layout, D, dims, interleaved, dtype):
    T, H, r = 83, 3, rng("parts", layout, D, dims, dtype)
    rotary, at = B.Rotary(B.rotary_frequencies(dims), interleaved), torch.arange(T, dtype=torch.int32, device="cuda")
    q, k, v = (rounded(r.normal(size=(T, H, D)), dtype)[0].cuda() for _ in range(3))
    want_q, want_k = B.hlq_rotary(q, at, rotary), B.hlq_rotary(k, at, rotary)
    x, y = room(layout, T, H, D, dtype)
    x.copy_(q)
    assert torch.equal(B.hlq_rotary(x, at, rotary, out=y), want_q) and torch.equal(x, q)
    kv = B.alloc_kv_cache(6, 16, H, D, TYPES[dtype] if dtype != "f32" else torch.float16)
    k_in, k_out = room(layout, T, H, D, dtype)
    k_in.copy_(k)
    y.fill_(0)
    B.hlq_kv_write(kv, k_in, v, torch.arange(T, device="cuda"), rotary, at, q=x, q_out=y, k_out=k_out)
    assert torch.equal(y, want_q) and torch.equal(k_out, want_k) and torch.equal(x, q) and torch.equal(k_in, k)
    keys, values = room(layout, T, H, D, dtype)
    B.hlq_kv_read(kv, torch.arange(T, device="cuda"), keys, values)
    one, two = B.hlq_kv_read(kv, torch.arange(T, device="cuda"), dtype=TYPES[dtype])
    assert torch.equal(keys, one) and torch.equal(values, two)


@pytest.mark.parametrize("layout", LAYOUTS)
def test_attention(layout):
    T, H, D, r = 140, 2, 64, rng("attention parts", layout)
    q, k, v = (rounded(r.normal(size=(T, H, D)), "bf16")[0].cuda() for _ in range(3))
    at = torch.tensor([0, 100, T], dtype=torch.int32, device="cuda")
    want = B.hlq_attn_prompt(q, k, v, at)
    x, y = room(layout, T, H, D, "bf16")
    x.copy_(q)
    assert torch.equal(B.hlq_attn_prompt(x, k, v, at, out=y), want) and torch.equal(x, q)
    y.copy_(k)
    assert torch.equal(B.hlq_attn_prompt(x, y, v, at, out=x), want)       # results in the queries' place
    kv = B.alloc_kv_cache(9, 16, H, D, torch.bfloat16)
    B.hlq_kv_write(kv, k, v, torch.arange(T, device="cuda"))
    table = torch.arange(9, dtype=torch.int32, device="cuda").expand(T, -1).contiguous()
    lengths = torch.arange(1, T + 1, dtype=torch.int32, device="cuda")
    want = B.hlq_attn_decode(kv, q, table, lengths)
    x.copy_(q)
    assert torch.equal(B.hlq_attn_decode(kv, x, table, lengths, out=y), want)
    assert torch.equal(B.hlq_attn_decode(kv, x, table, lengths, out=x), want)


def test_overlaps_are_refused():
    buffer = torch.zeros((9, 5, 64), dtype=torch.bfloat16, device="cuda")
    rotary, at = B.Rotary(B.rotary_frequencies(64)), torch.arange(9, dtype=torch.int32, device="cuda")
    with pytest.raises(B.HlqError):
        B.hlq_rotary(buffer[:, :3], at, rotary, out=buffer[:, 1:4])
    kv = B.alloc_kv_cache(1, 16, 2, 64, torch.bfloat16)
    with pytest.raises(B.HlqError):
        B.hlq_kv_read(kv, torch.arange(9, device="cuda"), buffer[:, :2], buffer[:, 1:3])
    assert (buffer == 0).all()
