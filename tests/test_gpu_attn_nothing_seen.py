"""A query none of whose scores is above -infinity has 0, whatever the values are that it sees: infinite, NaN, in whole tiles or at the edge of what is seen, cut or not."""
import pytest
import torch

from attn_util import KINDS, TYPES
from paper_2510_19482_amd import binding as B

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def odd(v):
    """Some of the rows' values are no numbers."""
    v[3], v[5:, :, 1], v[-1, :, 2], v[-1, :, 3] = INF, -INF, NAN, INF
    return v


@pytest.mark.parametrize("out_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [7, 33, 300, 9000])
@pytest.mark.parametrize("kind,qtype", [("bf16", "bf16"), ("f16", "f16"), ("mx8", "bf16"), ("mx8", "f16"), ("mx4", "bf16")])
@pytest.mark.parametrize("D", [32, 128, 256])
def test_decode(kind, qtype, D, n, out_dtype):
    # (an 8- or 4-bit block with an infinity is NaN, so there it is the query that makes the scores)
    page = 64
    pages = -(-n // page)
    kv = B.alloc_kv_cache(pages, page, 2, D, KINDS[kind])
    k = torch.full((n, 2, D), -1.0, dtype=TYPES[qtype], device="cuda")
    q = torch.ones((1, 6, D), dtype=TYPES[qtype], device="cuda")
    q[:, :, 4] = INF
    B.hlq_kv_write(kv, k, odd(torch.ones((n, 2, D), dtype=TYPES[qtype], device="cuda")), torch.arange(n, device="cuda"))
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    got = B.hlq_attn_decode(kv, q, table, torch.full((1,), n, dtype=torch.int32, device="cuda"), out_dtype=TYPES[out_dtype])
    assert (got == 0).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n_q,n_k,causal", [(200, 200, True), (70, 3000, True), (40, 100, False), (3, 9000, True)])
def test_prompt(n_q, n_k, causal, D, dtype):
    q = torch.ones((n_q, 2, D), dtype=TYPES[dtype], device="cuda")
    k = torch.ones((n_k, 1, D), dtype=TYPES[dtype], device="cuda")
    k[:, :, 7] = -INF
    v = odd(torch.ones((n_k, 1, D), dtype=TYPES[dtype], device="cuda"))
    q_at, k_at = (torch.tensor([0, n], dtype=torch.int32, device="cuda") for n in (n_q, n_k))
    assert (B.hlq_attn_prompt(q, k, v, q_at, k_at, causal=causal) == 0).all()
