"""Keys alone and values alone out of the cache: the same bits as both together, in 16, 8 and 4 bits, whole tokens and tokens whose heads are cut over wavefronts."""
import pytest
import torch

from attn_util import KINDS, TYPES
from paper_2510_19482_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("kind,H,D", [("bf16", 5, 40), ("f16", 3, 256), ("bf16", 16, 128), ("mx8", 7, 96), ("mx8", 1, 32), ("mx4", 13, 64), ("mx4", 8, 160)])
@pytest.mark.parametrize("T", [1, 70, 5000])
def test_one_side(T, kind, H, D, out):
    pages = -(-T // 16) + 1
    kv = B.alloc_kv_cache(pages, 16, H, D, KINDS[kind])
    g = torch.Generator(device="cuda").manual_seed(T + H)
    k, v = (torch.randn((T, H, D), device="cuda", generator=g).to(TYPES["f16" if kind == "f16" else "bf16"]) for _ in range(2))
    slots = torch.randperm(pages * 16, device="cuda", generator=g)[:T]
    B.hlq_kv_write(kv, k, v, slots)
    slots[T // 2] = -1
    both = [torch.full((T, H, D), 3.0, dtype=TYPES[out], device="cuda") for _ in range(2)]
    B.hlq_kv_read(kv, slots, *both)
    assert (both[0][T // 2] == 3).all() and not torch.equal(both[0], both[1]) or T == 1
    for only, want in zip("kv", both):
        alone = torch.full((T, H, D + 8), 3.0, dtype=TYPES[out], device="cuda")
        got = B.hlq_kv_read(kv, slots, **{only: alone[:, :, :D]}, only=only)
        assert got["vk".index(only)] is None and torch.equal(alone[:, :, :D], want) and (alone[:, :, D:] == 3).all()
        keep = torch.arange(T, device="cuda") != T // 2
        new = B.hlq_kv_read(kv, slots, dtype=TYPES[out], only=only)
        assert torch.equal(new["kv".index(only)][keep], want[keep]) and new["vk".index(only)] is None
