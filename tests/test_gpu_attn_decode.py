"""One new token over the paged cache, against the 64-bit oracle; the bounds are derived in attn_util."""
import numpy as np
import pytest
import torch

from attn_util import TYPES, Cache, bound, host, rng, rounded
from oracle import attn_oracle as O
from paper_2510_19482_amd import binding as B

pytestmark = pytest.mark.gpu

WEIGHT = {"f16": 2.0**-22, "bf16": 2.0**-16}   # two terms, each off by half a step


class Batch:
    """Sequences of these lengths in a cache with nothing else in it, and tables whose unused entries are no pages."""

    def __init__(self, lengths, Hq, H, D, page, kind, qtype, window=0, width=None, spread=1.0, key=()):
        r = rng("decode", lengths, Hq, H, D, page, kind, qtype, window, *key)
        self.lengths, self.window, self.kind, self.qtype = lengths, window, kind, qtype
        B_, need = len(lengths), [-(-n // page) for n in lengths]
        width = max(1, max(need)) if width is None else width
        pages = sum(need) + 3
        order = r.permutation(pages)
        self.table = np.where(r.integers(0, 2, size=(B_, width)), 2**31 - 1, -7).astype(np.int32)
        self.cache = Cache(pages, page, H, D, kind)
        at = 0
        slots = []
        for b, n in enumerate(lengths):
            mine = order[at:at + need[b]]
            at += need[b]
            self.table[b, :need[b]] = mine
            t = np.arange(n)
            first = max(0, n - window) if window else 0
            slots.append((mine[t // page] * page + t % page)[first:] if n else np.zeros(0, np.int64))
        every = np.concatenate(slots).astype(np.int64)
        self.slots = slots
        kvtype = kind if kind in TYPES else "bf16"
        k, v = (rounded(r.normal(size=(len(every), H, D)), kvtype)[1] for _ in range(2))
        k[:, :, :: max(1, D // 3)] *= 4
        k = rounded(k, kvtype)[1]
        if len(every):
            self.cache.put(every, k, v, kvtype)
        self.q_host, self.q = rounded(r.normal(size=(B_, Hq, D)) * spread, qtype)

    def gpu(self):
        return self.cache.kv, self.q_host.cuda(), torch.from_numpy(self.table).cuda(), torch.tensor(self.lengths, dtype=torch.int32, device="cuda")

    def check(self, got, dtype, scale=None):
        got = host(got)
        Bn, Hq, D = self.q.shape
        H = self.cache.heads
        scale = np.float32(D**-0.5 if scale is None else scale)
        compute = "f16" if self.kind == "f16" else "bf16"
        for b in range(Bn):
            at = self.slots[b]
            for h in range(Hq):
                k, v = (self.cache.values[i][at][:, h // (Hq // H)] for i in (0, 1))
                y, size, products = O.attend(self.q[b, h:h + 1], k, v, np.ones((1, len(at)), bool), scale)
                e = bound(size[0], products[0], len(at), D, np.abs(v).max() if len(at) else 0, WEIGHT[compute], dtype, y[0])
                bad = ~(np.abs(got[b, h] - y[0]) <= e)
                assert not bad.any(), f"sequence {b} of {len(at)}, head {h}: worst {np.nanmax(np.abs(got[b, h] - y[0]) / e):.3g} times the bound, {bad.sum()} values"


CASES = [
    # lengths about the edges of tiles, pages and workgroups; one empty
    ([0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 161], 8, 2, 128, 16, "bf16", "bf16", 0),
    ([0, 1, 15, 16, 17, 31, 33, 64, 127, 128, 129, 300], 4, 1, 64, 32, "f16", "f16", 0),
    ([1, 16, 33, 100, 257, 700], 12, 4, 32, 64, "bf16", "bf16", 0),
    ([5, 130, 513], 5, 5, 96, 16, "f16", "f16", 0),
    ([1, 77, 400], 16, 1, 40, 16, "bf16", "bf16", 0),
    ([3, 129, 260], 17, 1, 72, 128, "f16", "f16", 0),          # more heads than one product has
    ([60, 1], 40, 1, 8, 16, "bf16", "bf16", 0),
    ([0, 31, 161, 290], 6, 2, 256, 16, "bf16", "bf16", 0),
    ([7, 200], 4, 2, 160, 64, "f16", "f16", 0),
    ([33, 400], 8, 8, 192, 32, "bf16", "bf16", 0),
    ([0, 1, 15, 17, 32, 65, 129, 513], 8, 2, 128, 16, "mx8", "bf16", 0),
    ([1, 31, 200], 6, 3, 96, 32, "mx8", "f16", 0),
    ([1, 100, 333], 4, 1, 32, 16, "mx8", "f16", 0),
    ([65, 290], 3, 1, 256, 64, "mx8", "bf16", 0),
    ([0, 1, 15, 17, 32, 65, 129, 513], 8, 2, 128, 16, "mx4", "bf16", 0),
    ([1, 31, 200], 6, 3, 64, 32, "mx4", "f16", 0),
    ([40, 333], 20, 1, 160, 16, "mx4", "f16", 0),
    ([65, 290], 4, 4, 256, 128, "mx4", "bf16", 0),
    ([64, 290], 4, 4, 32, 1024, "mx4", "bf16", 0),
    # a window
    ([0, 1, 16, 40, 41, 100, 500], 8, 2, 128, 16, "bf16", "bf16", 40),
    ([1, 33, 300, 1025], 4, 1, 64, 64, "f16", "f16", 1),
    ([31, 300, 777], 4, 2, 128, 16, "mx4", "f16", 129),
    ([31, 300, 777], 2, 2, 96, 16, "mx8", "bf16", 33),
    # several workgroups a sequence
    ([20000, 3, 9000], 8, 1, 128, 64, "bf16", "bf16", 0),
    ([9999], 5, 1, 64, 16, "f16", "f16", 0),
    ([12345, 0], 4, 1, 256, 128, "mx8", "bf16", 0),
    ([16400], 16, 1, 128, 16, "mx4", "f16", 5000),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[3]}-{c[5]}-{c[6]}-{max(c[0])}-{c[1]}x{c[2]}-w{c[7]}")
def test_against_the_oracle(case):
    batch = Batch(*case)
    cache, q, table, lengths = batch.gpu()
    for dtype in ("f32", case[6]):
        out = B.hlq_attn_decode(cache, q, table, lengths, window=case[7], out_dtype=TYPES[dtype])
        batch.check(out, dtype)
    # again, the same bits: no order of workgroups shows
    ws = B.alloc_decode_workspace(cache, q.shape[1], q.shape[0], table.shape[1])
    for _ in range(3):
        again = B.hlq_attn_decode(cache, q, table, lengths, window=case[7], ws=ws)
        assert torch.equal(again, out)
    assert (ws[:131072] == 0).all()


def test_peaked_and_shifted_scores():
    # one key takes nearly all of the weight, scores far from 0, scale negative and 0
    batch = Batch([500, 33], 4, 2, 128, 16, "bf16", "bf16", spread=30.0, key=("peaked",))
    cache, q, table, lengths = batch.gpu()
    for scale in (None, 0.01, -0.1, 0.0):
        batch.check(B.hlq_attn_decode(cache, q, table, lengths, scale=scale, out_dtype=torch.float32), "f32", scale)


def test_strides_and_tables_wider_than_needed():
    batch = Batch([70, 0, 129], 6, 2, 64, 16, "f16", "f16", width=40, key=("strides",))
    cache, q, table, lengths = batch.gpu()
    want = B.hlq_attn_decode(cache, q, table, lengths)
    batch.check(want, "f16")
    fused = torch.zeros((3, 10 * 64 + 5), dtype=torch.float16, device="cuda")
    view = fused.as_strided((3, 6, 64), (645, 64, 1), 3)
    view.copy_(q)
    out = torch.full((6, 3, 66), 9.0, dtype=torch.float16, device="cuda")
    wide = torch.full((3, 50), -1, dtype=torch.int32, device="cuda")
    wide[:, :40] = table
    B.hlq_attn_decode(cache, view, wide[:, :40], lengths, out=out[:, :, 1:65].transpose(0, 1))
    assert torch.equal(out[:, :, 1:65].transpose(0, 1), want)
    assert (out[:, :, 0] == 9).all() and (out[:, :, 65] == 9).all()


def test_lengths_and_pages_out_of_range_stay_inside():
    # only that nothing outside is read or written, and that what is in range is right
    batch = Batch([40, 48, 16], 4, 2, 64, 16, "bf16", "bf16", key=("range",))
    cache, q, table, lengths = batch.gpu()
    want = B.hlq_attn_decode(cache, q, table, lengths)
    odd = lengths.clone()
    odd[0], odd[2] = -5, 2**31 - 1       # as 0, as all 48 of the table
    got = B.hlq_attn_decode(cache, q, table, odd)
    assert (got[0] == 0).all() and torch.equal(got[1], want[1])


def test_an_empty_table():
    batch = Batch([0, 0], 4, 2, 64, 16, "bf16", "bf16")
    cache, q, _, lengths = batch.gpu()
    out = B.hlq_attn_decode(cache, q, torch.empty((2, 0), dtype=torch.int32, device="cuda"), lengths + 3)
    assert (out == 0).all()
    assert B.hlq_attn_decode(cache, q[:0], torch.empty((0, 4), dtype=torch.int32, device="cuda"), lengths[:0]).shape == (0, 4, 64)


def test_infinite_scores_and_values():
    batch = Batch([40], 2, 1, 64, 16, "bf16", "bf16", key=("inf",))
    cache, q, table, lengths = batch.gpu()
    rows = cache.rows
    page = int(table[0, 0])
    plain = B.hlq_attn_decode(cache, q, table, lengths, out_dtype=torch.float32)
    # a key that no query head can choose: its value, whatever it is, has weight 0 times itself, as in the formula
    rows[page, 0, 0, 3] = (-q[0, 0].sign() * float("inf")).to(torch.bfloat16)
    rows[page, 0, 0, 3][q[0, 0] == 0] = 0
    out = B.hlq_attn_decode(cache, q, table, lengths, out_dtype=torch.float32)
    assert torch.isfinite(out[0, 0]).all() and not torch.equal(out, plain)
    # an infinite value is its column's result, and no other's
    rows[page, 1, 0, 5, 7] = float("inf")
    out = B.hlq_attn_decode(cache, q, table, lengths, out_dtype=torch.float32)
    assert out[0, 0, 7] == float("inf") and torch.isfinite(out[0, 0, torch.arange(64) != 7]).all()
    # a key that is NaN makes its heads' results NaN
    rows[page, 0, 0, 9, 0] = float("nan")
    assert torch.isnan(B.hlq_attn_decode(cache, q, table, lengths)).all()


def test_a_workspace_serves_smaller_calls_and_one_after_the_other():
    big = Batch([9000, 4000, 100], 8, 2, 128, 64, "bf16", "bf16", key=("ws",))
    small = Batch([3000], 8, 2, 128, 64, "bf16", "bf16", key=("ws",))
    cache, q, table, lengths = big.gpu()
    ws = B.alloc_decode_workspace(cache, 8, 3, table.shape[1])
    want = [B.hlq_attn_decode(*x.gpu()) for x in (big, small)]
    for _ in range(5):
        for x, y in zip((big, small), want):
            assert torch.equal(B.hlq_attn_decode(*x.gpu(), ws=ws), y)


def test_pages_past_32_bits():
    pages, page, H, D = 18000, 128, 8, 128
    kv = B.alloc_kv_cache(pages, page, H, D, torch.bfloat16)
    n = 300
    r = rng("far pages")
    k, v = (rounded(r.normal(size=(n, H, D)), "bf16")[0] for _ in range(2))
    table = torch.tensor([[17999, 9000, 16384]], dtype=torch.int32)
    t = torch.arange(n)
    B.hlq_kv_write(kv, k.cuda(), v.cuda(), (table[0, t // page].long() * page + t % page).cuda())
    q = rounded(r.normal(size=(1, H, D)), "bf16")[0]
    out = B.hlq_attn_decode(kv, q.cuda(), table.cuda(), torch.tensor([n], dtype=torch.int32, device="cuda"), out_dtype=torch.float32)
    for h in range(H):
        y, size, products = O.attend(q[0, h:h + 1].double().numpy(), k[:, h].double().numpy(), v[:, h].double().numpy(), np.ones((1, n), bool), np.float32(D**-0.5))
        assert (np.abs(host(out)[0, h] - y[0]) <= bound(size[0], products[0], n, D, 5.0, WEIGHT["bf16"], "f32", y[0])).all()
