"""A value that is infinite or NaN is its column's result for every query that sees it, however small its weight and wherever it stands; a key whose score is -infinity counts as
one that is not seen, so its value does not show.  All other columns have the bits that they have without it.

Scores: one channel of the queries is 1, the keys' is the score, the others are small numbers."""
import pytest
import torch

from attn_util import KINDS, TYPES, rng, rounded
from paper_2510_19482_amd import binding as B
from test_gpu_attn_corners import shifted

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def inputs(r, n_q, n_k, Hq, D, dtype, low):
    """The key at 40 has a score of 0, the others one about `low`."""
    q, k, v = (r.normal(size=s) for s in ((n_q, Hq, D), (n_k, 1, D), (n_k, 1, D)))
    q, k = q * 0.01, k * 0.01
    q[:, :, 0] = 1
    k[:, :, 0] = low + r.normal(size=(n_k, 1))
    k[40] = 0
    return [rounded(x, dtype)[0].cuda() for x in (q, k, v)]


def expected(clean, seen_by, v, column_only=True):
    """The result with the values at {row: (column, number)}, of queries seen_by[row]."""
    want = clean.clone()
    for row, (column, number) in v.items():
        at = want[seen_by(row)]
        at[..., column] = at[..., column] + number if number == number else NAN
        want[seen_by(row)] = at
    return want


def same(got, want):
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got[~torch.isnan(got)], want[~torch.isnan(want)])


# in whole tiles, at the edge of what is seen, beside the largest score, both infinities in one column
ODD = {3: (1, INF), 40: (2, -INF), 70: (3, INF), 130: (3, -INF), 131: (4, NAN), 190: (5, -INF), 199: (6, INF), 64: (7, INF)}


def clear(v, odd):
    """Without them: where an infinity is added to a column its finite part does not show."""
    v = v.clone()
    for row, (column, number) in odd.items():
        v[row, 0, column] = 0
    return v


def put(v, odd):
    v = v.clone()
    for row, (column, number) in odd.items():
        v[row, 0, column] = number
    return v


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("low", [-3.0, -25.0, -300.0])
@pytest.mark.parametrize("before,Hq", [(0, 2), (0, 4), (2600, 1)])
def test_prompt(before, Hq, low, D, dtype):
    # the odd rows among the last 200 keys, the queries are these tokens; with 2600 keys before, the launch is cut
    n = 200
    q, k, v = inputs(rng("infinite", before, Hq, low, D, dtype), n, before + n, Hq, D, dtype, low)
    odd = {row + before: x for row, x in ODD.items()}
    q_at, k_at = (torch.tensor([0, x], dtype=torch.int32, device="cuda") for x in (n, before + n))
    clean = B.hlq_attn_prompt(q, k, clear(v, odd), q_at, k_at)
    got = B.hlq_attn_prompt(q, k, put(v, odd), q_at, k_at)
    same(got, expected(clean, lambda row: torch.arange(n, device="cuda") >= row - before, odd))
    # every query sees every key; a window
    clean = B.hlq_attn_prompt(q, k, clear(v, odd), q_at, k_at, causal=False)
    got = B.hlq_attn_prompt(q, k, put(v, odd), q_at, k_at, causal=False)
    same(got, expected(clean, lambda row: torch.arange(n, device="cuda") >= 0, odd))
    i = torch.arange(n, device="cuda")
    clean = B.hlq_attn_prompt(q, k, clear(v, odd), q_at, k_at, window=90)
    got = B.hlq_attn_prompt(q, k, put(v, odd), q_at, k_at, window=90)
    same(got, expected(clean, lambda row: (i >= row - before) & (i < row - before + 90), odd))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 72, 128, 256])
@pytest.mark.parametrize("before,causal", [(0, True), (0, False), (2600, True)])
def test_prompt_of_rows_at_any_alignment(before, causal, D, dtype):
    n = 200
    q, k, v = inputs(rng("infinite, any", before, causal, D, dtype), n, before + n, 2, D, dtype, -25.0)
    odd = {row + before: x for row, x in ODD.items()}
    q_at, k_at = (torch.tensor([0, x], dtype=torch.int32, device="cuda") for x in (n, before + n))
    want = B.hlq_attn_prompt(q, k, put(v, odd), q_at, k_at, causal=causal)
    clean = B.hlq_attn_prompt(q, k, clear(v, odd), q_at, k_at, causal=causal)
    same(want, expected(clean, lambda row: torch.arange(n, device="cuda") >= (row - before if causal else 0), odd))
    same(B.hlq_attn_prompt(shifted(q), shifted(k, 3), shifted(put(v, odd)), q_at, k_at, causal=causal), want)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n_k", [200, 2800])
def test_prompt_keys_whose_score_is_minus_infinity(n_k, D, dtype):
    n = 200
    q, k, v = inputs(rng("hidden", n_k, D, dtype), n, n_k, 2, D, dtype, -2.0)
    hidden = list(range(50)) + [70, 100, 131, n_k - 1]
    q[:, :, 1], k[:, :, 1] = 1, 0
    k[hidden, :, 1] = -INF
    q_at, k_at = (torch.tensor([0, x], dtype=torch.int32, device="cuda") for x in (n, n_k))
    for causal in (True, False):
        clean = B.hlq_attn_prompt(q, k, v, q_at, k_at, causal=causal)
        w = v.clone()
        for i, row in enumerate(hidden):
            w[row, 0, i % 9] = (INF, -INF, NAN)[i % 3]
        got = B.hlq_attn_prompt(q, k, w, q_at, k_at, causal=causal)
        assert torch.isfinite(got).all() and torch.equal(got, clean)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_prompt_infinity_before_larger_scores(D, dtype):
    # what was summed is multiplied by less than the smallest number when larger scores come
    n = 400
    q, k, v = inputs(rng("later", D, dtype), n, n, 2, D, dtype, -2.0)
    k[150:, :, 0] = 250
    k[300:, :, 0] = 600
    v[5, 0, 2], v[200, 0, 3] = INF, -INF
    at = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    got = B.hlq_attn_prompt(q, k, v, at, at)
    assert (got[5:, :, 2] == INF).all() and (got[200:, :, 3] == -INF).all()
    assert torch.isfinite(got[:5]).all() and torch.isfinite(got[:, :, 4:]).all() and torch.isfinite(got[:200, :, 3]).all()


def decode(kv, q, lengths, pages, **kw):
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None].expand(len(lengths), -1).contiguous()
    return B.hlq_attn_decode(kv, q, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), **kw)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("low", [-3.0, -25.0, -300.0])
@pytest.mark.parametrize("n", [200, 9000])
@pytest.mark.parametrize("out", ["f32", "f16"])
def test_decode(n, low, D, dtype, out):
    lengths = [n, 65, 132, 1]
    q, k, v = inputs(rng("one", n, low, D, dtype), 4, n, 5, D, dtype, low)
    odd = dict(ODD)
    if n > 200:
        odd[n - 700] = (8, INF)
    pages = -(-n // 64)
    results = []
    for values in (clear(v, odd), put(v, odd)):
        kv = B.alloc_kv_cache(pages, 64, 1, D, TYPES[dtype])
        kv.blob.fill_(255)
        B.hlq_kv_write(kv, k, values, torch.arange(n, device="cuda"))
        results += [decode(kv, q, lengths, pages, out_dtype=TYPES[out]), decode(kv, q, lengths, pages, window=50, out_dtype=TYPES[out])]
    m = torch.tensor(lengths, device="cuda")
    same(results[2], expected(results[0], lambda row: m > row, odd))
    same(results[3], expected(results[1], lambda row: (m > row) & (m - 50 <= row), odd))


@pytest.mark.parametrize("kind,qtype", [("mx8", "bf16"), ("mx8", "f16"), ("mx4", "bf16"), ("mx4", "f16")])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("low", [-3.0, -300.0])
def test_decode_blocks_that_are_nan(low, D, kind, qtype):
    n, lengths = 3000, [3000, 130, 1]
    r = rng("blocks", low, D, kind, qtype)
    _, k, v = inputs(r, 3, n, 4, D, qtype, low)
    k[:, :, 1:] = 0          # so that a block of keys is its score
    q = torch.zeros((3, 4, D), dtype=TYPES[qtype], device="cuda")
    q[:, :, 0] = 1
    results = []
    for bad in (False, True):
        w = v.clone()
        if bad:
            w[100, 0, 5], w[2999, 0, D - 1] = NAN, INF
        kv = B.alloc_kv_cache(-(-n // 64), 64, 1, D, KINDS[kind])
        B.hlq_kv_write(kv, k, w, torch.arange(n, device="cuda"))
        results.append(decode(kv, q, lengths, -(-n // 64), out_dtype=torch.float32))
    want = results[0].clone()
    want[:2, :, :32] = NAN
    want[0, :, D - 32:] = NAN
    same(results[1], want)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n", [200, 9000])
def test_decode_keys_whose_score_is_minus_infinity(n, D, dtype):
    q, k, v = inputs(rng("one hidden", n, D, dtype), 2, n, 3, D, dtype, -2.0)
    q[:, :, 1], k[:, :, 1] = 1, 0
    hidden = list(range(35)) + [77, 150, n - 1]
    k[hidden, :, 1] = -INF
    pages = -(-n // 64)
    results = []
    for bad in (False, True):
        w = v.clone()
        if bad:
            for i, row in enumerate(hidden):
                w[row, 0, i % 9] = (INF, -INF, NAN)[i % 3]
        kv = B.alloc_kv_cache(pages, 64, 1, D, TYPES[dtype])
        B.hlq_kv_write(kv, k, w, torch.arange(n, device="cuda"))
        results.append(decode(kv, q, [n, 60], pages, out_dtype=torch.float32))
    assert torch.isfinite(results[1]).all() and torch.equal(results[0], results[1])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n", [400, 9000])
def test_decode_infinity_before_larger_scores(n, dtype):
    q, k, v = inputs(rng("one later", n, dtype), 1, n, 2, 128, dtype, -2.0)
    k[n // 3:, :, 0] = 250
    k[n // 2:, :, 0] = 600
    v[5, 0, 2], v[n // 3 + 4, 0, 3] = INF, -INF
    pages = -(-n // 64)
    kv = B.alloc_kv_cache(pages, 64, 1, 128, TYPES[dtype])
    B.hlq_kv_write(kv, k, v, torch.arange(n, device="cuda"))
    got = decode(kv, q, [n], pages)
    assert (got[0, :, 2] == INF).all() and (got[0, :, 3] == -INF).all() and torch.isfinite(got[0, :, 4:]).all() and torch.isfinite(got[0, :, :2]).all()
