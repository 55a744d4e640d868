"""Attention where paths meet: keys that a launch is cut over with windows, with values that are no numbers and with rows at any alignment; many sequences; numbers
near the ends of their types; rows turned in place.  Bounds as in attn_util."""
import numpy as np
import pytest
import torch

from attn_util import HALF_STEP, TYPES, bound, host, rng, rounded
from oracle import attn_oracle as O
from paper_2510_19482_amd import binding as B
from test_gpu_attn_decode import WEIGHT, Batch
from test_gpu_attn_prompt import Packed, same

pytestmark = pytest.mark.gpu


def shifted(t, by=1):
    """The same numbers, `by` elements past a multiple of 16 bytes."""
    room = torch.zeros(t.numel() + by, dtype=t.dtype, device="cuda")
    room[by:].copy_(t.reshape(-1))
    return room[by:].view(t.shape)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [8, 64, 72, 128, 136, 256])
@pytest.mark.parametrize("lengths", [same(1, 40, 200), [(70, 1500), (3, 300)]], ids=["whole", "cut"])
def test_rows_at_any_alignment(lengths, D, dtype):
    p = Packed(lengths, 4, 2, D, dtype, key=("aligned",))
    q_at, k_at = p.offsets()
    want = p.run()
    p.check(want)
    got = B.hlq_attn_prompt(shifted(p.q_host), shifted(p.k_host), shifted(p.v_host, 3), q_at, k_at)
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("case", [([(100, 3000)], 4, 2, 128, True, 900), ([(33, 2000), (70, 900), (5, 0)], 2, 1, 64, True, 257), ([(64, 2500)], 2, 2, 256, False, 700), ([(64, 2500)], 4, 1, 96, True, 3)],
                         ids=lambda c: f"{c[3]}-w{c[5]}")
def test_cut_with_a_window(case, dtype):
    lengths, Hq, H, D, causal, window = case
    p = Packed(lengths, Hq, H, D, dtype, causal, window, key=("cut window",))
    out = p.run()
    p.check(out)
    assert torch.equal(p.run(), out)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("by", [0, 1])
def test_cut_with_values_that_are_no_numbers(D, dtype, by):
    n_q, n_k = 90, 2000
    p = Packed([(n_q, n_k)], 2, 1, D, dtype, key=("cut odd",))
    q_at, k_at = p.offsets()
    k, v = p.k_host.cuda(), p.v_host.cuda().clone()
    want = p.run().cpu()
    first = n_k - n_q
    v[first + 5, 0, 3], v[first + 60, 0, 9], v[first + 89, 0, 1], v[7, 0, 0] = float("inf"), float("nan"), float("-inf"), float("-inf")
    got = B.hlq_attn_prompt(p.q_host.cuda(), shifted(k, by), shifted(v, by), q_at, k_at).cpu()
    changed = torch.zeros((n_q, 2, D), dtype=torch.bool)
    changed[5:, :, 3] = changed[60:, :, 9] = changed[89:, :, 1] = changed[:, :, 0] = True
    assert torch.equal(got[~changed], want[~changed])
    assert (got[5:, :, 3] == float("inf")).all() and torch.isnan(got[60:, :, 9]).all() and (got[89:, :, 1] == float("-inf")).all()


def test_one_packed_launch_is_its_sequences_one_by_one():
    # sequences neither see nor disturb each other, whatever stands in the others
    p = Packed(same(130, 77, 300), 4, 2, 64, "bf16", key=("alone",))
    out = p.run()
    q_at, k_at = p.offsets()
    v = p.v_host.cuda()
    v[130:207] = float("nan")
    got = B.hlq_attn_prompt(p.q_host.cuda(), p.k_host.cuda(), v, q_at, k_at)
    assert torch.equal(got[:130], out[:130]) and torch.equal(got[207:], out[207:]) and torch.isnan(got[130:207]).all()


@pytest.mark.parametrize("H,Hq,B_", [(8, 32, 150), (1, 16, 40), (4, 4, 1500)])
def test_many_sequences(H, Hq, B_):
    r = rng("many", H, Hq, B_)
    lengths = r.integers(0, 200, size=B_).tolist()
    batch = Batch(lengths, Hq, H, 64, 16, "bf16", "bf16", key=("many",))
    cache, q, table, lengths = batch.gpu()
    out = B.hlq_attn_decode(cache, q, table, lengths)
    some = r.permutation(B_)[:12]
    for b in some:
        one = B.hlq_attn_decode(cache, q[b:b + 1], table[b:b + 1], lengths[b:b + 1])
        at = batch.slots[b]
        for h in range(Hq):
            k, v = (batch.cache.values[i][at][:, h // (Hq // H)] for i in (0, 1))
            y, size, products = O.attend(batch.q[b, h:h + 1], k, v, np.ones((1, len(at)), bool), np.float32(64**-0.5))
            e = bound(size[0], products[0], len(at), 64, np.abs(v).max() if len(at) else 0, WEIGHT["bf16"], "bf16", y[0])
            for got in (out[b, h], one[0, h]):
                assert (np.abs(host(got) - y[0]) <= e).all()


@pytest.mark.parametrize("kind,qtype", [("mx8", "bf16"), ("mx4", "bf16"), ("mx8", "f16"), ("mx4", "f16"), ("bf16", "bf16")])
@pytest.mark.parametrize("k_power,v_power", [(-110, 0), (110, 0), (0, -100), (0, 100), (-90, 90)])
def test_numbers_of_any_size(kind, qtype, k_power, v_power):
    # keys and values that only their scale bytes, or bf16's exponent, hold; the scale brings scores back
    n, H, D = 70, 2, 64
    r = rng("sizes", kind, qtype, k_power, v_power)
    pages = -(-n // 16)
    kv = B.alloc_kv_cache(pages, 16, H, D, TYPES[kind] if kind in TYPES else {"mx8": B.HLQ_MX8, "mx4": B.HLQ_MX4}[kind])
    k, v = (torch.from_numpy(r.normal(size=(n, H, D)) * 2.0**p).to(torch.bfloat16) for p in (k_power, v_power))
    slots = torch.arange(n, device="cuda")
    B.hlq_kv_write(kv, k.cuda(), v.cuda(), slots)
    held = [x.double().cpu().numpy() for x in B.hlq_kv_read(kv, slots)]
    q_host, q = rounded(r.normal(size=(1, H, D)), qtype)
    scale = float(np.float32(2.0**-k_power * D**-0.5))
    got = host(B.hlq_attn_decode(kv, q_host.cuda(), torch.arange(pages, dtype=torch.int32, device="cuda")[None], torch.tensor([n], dtype=torch.int32, device="cuda"), scale=scale,
                                 out_dtype=torch.float32))
    for h in range(H):
        y, size, products = O.attend(q[0, h:h + 1], held[0][:, h], held[1][:, h], np.ones((1, n), bool), np.float32(scale))
        e = bound(size[0], products[0], n, D, np.abs(held[1]).max(), WEIGHT["bf16"], "f32", y[0])
        assert (np.abs(got[0, h] - y[0]) <= e).all()


def test_an_infinite_query_over_an_8_bit_cache():
    # scores of -infinity only: nothing is seen; a head with a number among them is that key's value
    kv = B.alloc_kv_cache(1, 16, 1, 32, B.HLQ_MX8)
    k = torch.full((2, 1, 32), 0.0, dtype=torch.float16, device="cuda")
    v = torch.ones((2, 1, 32), dtype=torch.float16, device="cuda")
    k[:, 0, :] = -1.0
    B.hlq_kv_write(kv, k, v, torch.arange(2, device="cuda"))
    q = torch.ones((1, 1, 32), dtype=torch.float16, device="cuda")
    q[0, 0, 4] = float("inf")
    table, n = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.full((1,), 2, dtype=torch.int32, device="cuda")
    assert (B.hlq_attn_decode(kv, q, table, n) == 0).all()
    assert (B.hlq_attn_decode(kv, q.bfloat16(), table, n) == 0).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("D,dims,interleaved", [(128, 128, False), (64, 48, False), (40, 20, False), (96, 12, False), (72, 70, True), (256, 256, True)])
def test_in_place(D, dims, interleaved, dtype):
    r = rng("place", D, dims, interleaved, dtype)
    T, Hq, H = 300, 9, 5
    rotary = B.Rotary(B.rotary_frequencies(dims), interleaved)
    at = torch.from_numpy(r.integers(0, 100000, size=T).astype(np.int32)).cuda()
    q, k, v = (rounded(r.normal(size=(T, h, D)), dtype)[0].cuda() for h in (Hq, H, H))
    want_q, want_k = B.hlq_rotary(q, at, rotary), B.hlq_rotary(k, at, rotary)
    one, two = q.clone(), k.clone()
    assert B.hlq_rotary(one, at, rotary, out=one) is one and torch.equal(one, want_q)
    kv = B.alloc_kv_cache(-(-T // 16), 16, H, D, torch.bfloat16)
    one = q.clone()
    B.hlq_kv_write(kv, two, v, torch.arange(T, device="cuda"), rotary, at, q=one, q_out=one, k_out=two)
    assert torch.equal(one, want_q) and torch.equal(two, want_k)
    assert torch.equal(B.hlq_kv_read(kv, torch.arange(T, device="cuda"), dtype=torch.float32)[0], want_k.to(torch.bfloat16).float())


def test_a_cache_that_one_call_writes_and_the_next_reads_in_a_graph_beside_an_eager_one():
    # a captured step replayed while eager steps on another workspace run between its replays
    batch = Batch([3000, 50], 8, 2, 128, 64, "bf16", "bf16", key=("beside",))
    cache, q, table, lengths = batch.gpu()
    want = B.hlq_attn_decode(cache, q, table, lengths)
    ws = B.alloc_decode_workspace(cache, 8, 2, table.shape[1])
    out = torch.empty_like(want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.hlq_attn_decode(cache, q, table, lengths, out=out, ws=ws)
    for _ in range(4):
        out.zero_()
        graph.replay()
        assert torch.equal(B.hlq_attn_decode(cache, q, table, lengths), want)
        assert torch.equal(out, want)
