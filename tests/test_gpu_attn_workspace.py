"""Workspaces on the GPU: one that is made for the largest prompt serves smaller ones that are cut otherwise, and a call without one takes memory only if its launch is cut."""
import pytest
import torch

from paper_2510_19482_amd import binding as B

pytestmark = pytest.mark.gpu

HQ, H, D = 8, 2, 64


def prompt(n_q, n_k, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, k, v = (torch.randn((n, h, D), device="cuda", generator=g).bfloat16() for n, h in ((n_q, HQ), (n_k, H), (n_k, H)))
    return q, k, v, *(torch.tensor([0, n // 3, n], dtype=torch.int32, device="cuda") for n in (n_q, n_k))


def test_a_large_workspace_serves_smaller_prompts():
    most = (700, 20000, 5)
    ws = B.alloc_prompt_workspace(*most, HQ, H, D)
    ws[131072:].fill_(255)                       # what parts leave is not read by later calls
    for n_q, n_k in ((700, 20000), (1, 20000), (3, 300), (64, 9000), (700, 600), (33, 4097), (200, 20000), (1, 1)):
        args = prompt(n_q, n_k, n_q)
        own = B.alloc_prompt_workspace(n_q, n_k, 2, HQ, H, D)
        assert own.numel() <= ws.numel()
        want = B.hlq_attn_prompt(*args, ws=own)
        for _ in range(2):
            assert torch.equal(B.hlq_attn_prompt(*args, ws=ws), want)
        assert torch.equal(B.hlq_attn_prompt(*args), want)
        assert (ws[:131072] == 0).all() and (own[:131072] == 0).all()


def taken(call):
    torch.cuda.synchronize()
    before = torch.cuda.memory_stats()["allocation.all.allocated"]
    call()
    return torch.cuda.memory_stats()["allocation.all.allocated"] - before


def test_a_call_without_one():
    q, k, v, q_at, k_at = prompt(20000, 20000)   # more workgroups than a launch that is cut has
    out = torch.empty_like(q)
    assert taken(lambda: B.hlq_attn_prompt(q, k, v, q_at, k_at, out=out)) == 0
    q, k, v, q_at, k_at = prompt(3, 20000)
    out = torch.empty_like(q)
    assert taken(lambda: B.hlq_attn_prompt(q, k, v, q_at, k_at, out=out)) > 0
    kv = B.alloc_kv_cache(512, 64, H, D, torch.bfloat16)
    kv.blob.zero_()
    q = torch.ones((512, HQ, D), dtype=torch.bfloat16, device="cuda")
    table, lengths = torch.arange(512, dtype=torch.int32, device="cuda")[:, None], torch.full((512,), 64, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    assert taken(lambda: B.hlq_attn_decode(kv, q, table, lengths, out=out)) == 0
    assert (out == 0).all()
    one, n = table.view(1, -1).contiguous(), lengths[:1] * 512
    assert taken(lambda: B.hlq_attn_decode(kv, q[:1], one, n, out=out[:1])) > 0
    assert (out == 0).all()
