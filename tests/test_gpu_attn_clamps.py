"""Lengths and pages out of range by value: a length counts as at most the table's tokens and at least 0, a page as the nearest one inside the cache."""
import numpy as np
import pytest
import torch

from attn_util import KINDS, TYPES, bound, host, rng, rounded, stored
from oracle import attn_oracle as O
from paper_2510_19482_amd import binding as B

pytestmark = pytest.mark.gpu

LOW, HIGH = -(2**31), 2**31 - 1


@pytest.mark.parametrize("kind,qtype,weight", [("bf16", "bf16", 2.0**-16), ("f16", "f16", 2.0**-22), ("mx8", "bf16", 2.0**-16), ("mx4", "f16", 2.0**-16)])
@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_values(D, page, kind, qtype, weight):
    pages, width, H, Hq = 7, 5, 2, 4
    r = rng("clamps", D, page, kind, qtype)
    k, v = (rounded(r.normal(size=(pages * page, H, D)), qtype)[1] for _ in range(2))
    kv = B.alloc_kv_cache(pages, page, H, D, KINDS[kind])
    B.hlq_kv_write(kv, *(torch.from_numpy(x).to(TYPES[qtype]).cuda() for x in (k, v)), torch.arange(pages * page, device="cuda"))
    k, v = stored(k, kind), stored(v, kind)
    # page numbers below, above and next to the cache's, within the tokens that count; the first and the last page among them
    table = np.array([[-7, 3, HIGH, 0, 6], [LOW, pages, pages - 1, -1, 7], [2, 5, 1, 4, 0], [HIGH, LOW, HIGH, LOW, 3]], np.int32)
    lengths = np.array([HIGH, width * page + 1, -5, width * page - 3], np.int32)
    clamped, counted = table.clip(0, pages - 1), lengths.clip(0, width * page)
    q_host, q = rounded(r.normal(size=(4, Hq, D)), qtype)
    on_gpu = lambda t, n: (q_host.cuda(), torch.from_numpy(t).cuda(), torch.from_numpy(n).cuda())   # noqa: E731
    for window in (0, page + 5):
        got = B.hlq_attn_decode(kv, *on_gpu(table, lengths), window=window, out_dtype=torch.float32)
        assert torch.equal(got, B.hlq_attn_decode(kv, *on_gpu(clamped, counted.astype(np.int32)), window=window, out_dtype=torch.float32))
        got = host(got)
        for b in range(4):
            n = int(counted[b])
            t = np.arange(max(0, n - window) if window else 0, n)
            at = clamped[b, t // page] * page + t % page
            for h in range(Hq):
                y, size, products = O.attend(q[b, h:h + 1], k[at, h // 2], v[at, h // 2], np.ones((1, len(at)), bool), np.float32(D**-0.5))
                e = bound(size[0], products[0], len(at), D, np.abs(v).max(), weight, "f32", y[0])
                assert (np.abs(got[b, h] - y[0]) <= e).all(), (b, h)
        assert (got[2] == 0).all()
