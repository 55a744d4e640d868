"""Attention of packed prompts against the 64-bit oracle; the bounds are derived in attn_util."""
import numpy as np
import pytest
import torch

from attn_util import HALF_STEP, TYPES, bound, host, rng, rounded
from oracle import attn_oracle as O
from paper_2510_19482_amd import binding as B

pytestmark = pytest.mark.gpu


def seen(n_q, n_k, causal, window):
    place, j = (n_k - n_q + np.arange(n_q))[:, None], np.arange(n_k)[None]
    s = np.ones((n_q, n_k), bool)
    if causal:
        s &= j <= place
    if window:
        s &= j > place - window
    return s


class Packed:
    def __init__(self, lengths, Hq, H, D, dtype, causal=True, window=0, before=0, spread=1.0, key=()):
        r = rng("prompt", lengths, Hq, H, D, dtype, causal, window, before, *key)
        self.lengths, self.causal, self.window, self.dtype = lengths, causal, window, dtype
        at = np.array([[0, 0]] + [list(n) for n in lengths]).cumsum(0) + before   # (queries, keys) of each sequence
        self.q_at, self.k_at = at[:, 0], at[:, 1]
        self.Tq, self.Tk = int(at[-1, 0]) + before, int(at[-1, 1]) + before
        self.q_host, self.q = rounded(r.normal(size=(self.Tq, Hq, D)) * spread, dtype)
        k = r.normal(size=(self.Tk, H, D))
        k[:, :, :: max(1, D // 3)] *= 4
        self.k_host, self.k = rounded(k, dtype)
        self.v_host, self.v = rounded(r.normal(size=(self.Tk, H, D)), dtype)

    def offsets(self):
        return [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (self.q_at, self.k_at)]

    def run(self, **kw):
        q_at, k_at = self.offsets()
        return B.hlq_attn_prompt(self.q_host.cuda(), self.k_host.cuda(), self.v_host.cuda(), q_at, k_at, causal=self.causal, window=self.window, **kw)

    def check(self, got, scale=None, heads=None):
        got = host(got)
        Hq, D = self.q.shape[1:]
        H = self.k.shape[1]
        scale = np.float32(D**-0.5 if scale is None else scale)
        for b, (n_q, n_k) in enumerate(self.lengths):
            s = seen(n_q, n_k, self.causal, self.window)
            n = np.maximum(s.sum(1), 1)[:, None]
            rows, keys = slice(self.q_at[b], self.q_at[b + 1]), slice(self.k_at[b], self.k_at[b + 1])
            for h in range(Hq) if heads is None else heads:
                v = self.v[keys, h // (Hq // H)]
                y, size, products = O.attend(self.q[rows, h], self.k[keys, h // (Hq // H)], v, s, scale)
                e = bound(size, products[:, None], n, D, np.abs(v).max() if n_k else 0, 2 * HALF_STEP[self.dtype], self.dtype, y)
                bad = ~(np.abs(got[rows, h] - y) <= e)
                assert not bad.any(), f"sequence {b} ({n_q}, {n_k}), head {h}: worst {np.nanmax(np.abs(got[rows, h] - y) / e):.3g} times the bound, rows {np.nonzero(bad.any(1))[0][:5]}"
                assert (got[rows, h][~s.any(1)] == 0).all()


def same(*n):
    return [(x, x) for x in n]


CASES = [
    (same(1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200), 4, 2, 128, "bf16", True, 0),
    (same(0, 5, 0, 0, 130, 1, 0), 4, 1, 64, "f16", True, 0),
    (same(300, 17), 3, 1, 128, "f16", True, 0),
    (same(150, 64), 2, 2, 32, "bf16", True, 0),
    (same(33, 140), 5, 1, 96, "f16", True, 0),
    (same(100, 131), 2, 1, 256, "bf16", True, 0),
    (same(70), 2, 1, 160, "f16", True, 0),
    (same(257), 4, 4, 8, "f16", True, 0),
    (same(90, 40), 2, 1, 72, "bf16", True, 0),
    (same(90, 40, 129), 2, 1, 128, "bf16", False, 0),
    # keys from before, of a cached piece of the prompt; single tokens; no keys; fewer keys than queries, so that the first queries see nothing
    ([(5, 100), (64, 300), (1, 77), (1, 1), (130, 131), (17, 513)], 4, 2, 128, "bf16", True, 0),
    ([(5, 0), (40, 33), (130, 2), (3, 3), (200, 129)], 2, 1, 64, "f16", True, 0),
    ([(5, 0), (40, 33), (130, 2), (0, 50), (3, 200)], 2, 1, 128, "bf16", False, 0),
    # a window
    (same(200, 31, 65), 2, 1, 128, "bf16", True, 1),
    (same(300, 64, 129), 4, 2, 64, "f16", True, 40),
    ([(64, 500), (130, 300), (9, 9)], 2, 1, 128, "f16", True, 100),
    ([(64, 500), (130, 60)], 2, 1, 96, "bf16", False, 33),
    ([(200, 200)], 1, 1, 256, "f16", True, 2**31 - 1),
    ([(100, 40)], 1, 1, 64, "bf16", True, 7),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[3]}-{c[4]}-{len(c[0])}-{c[1]}x{c[2]}-{'causal' if c[5] else 'all'}-w{c[6]}")
def test_against_the_oracle(case):
    p = Packed(*case)
    out = p.run()
    p.check(out)
    assert torch.equal(p.run(), out)


def test_many_short_sequences():
    # more sequences than a wavefront has lanes
    lengths = [(i % 7, i % 7 + (i % 3) * 20) for i in range(150)]
    p = Packed(lengths, 2, 1, 64, "bf16")
    p.check(p.run())


def test_long_prompts():
    p = Packed(same(2100, 900), 2, 1, 128, "bf16", key=("long",))
    p.check(p.run())
    p = Packed([(40, 6000)], 4, 1, 64, "f16", key=("long",))
    p.check(p.run())


def test_peaked_and_shifted_scores():
    p = Packed(same(200), 2, 1, 128, "f16", spread=20.0)
    for scale in (None, -0.05, 0.0):
        p.check(p.run(scale=scale), scale)


def test_strides_offsets_and_rows_of_no_sequence():
    p = Packed(same(37, 100), 4, 2, 64, "bf16", before=5, key=("strides",))
    q_at, k_at = p.offsets()
    want = torch.full((p.Tq, 4, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    p.run(out=want)
    p.check(want)
    assert (want[:5] == 3).all() and (want[-5:] == 3).all()
    # parts of a projection's rows that begin at any element; head by head
    fused = torch.zeros((p.Tq, 8 * 64 + 3), dtype=torch.bfloat16, device="cuda")
    q, k, v = (fused.as_strided((p.Tq, h, 64), (8 * 64 + 3, 64, 1), 1 + at * 64) for at, h in ((0, 4), (4, 2), (6, 2)))
    for t, x in ((q, p.q_host), (k, p.k_host), (v, p.v_host)):
        t.copy_(x)
    out = torch.full((4, p.Tq, 68), 3.0, dtype=torch.bfloat16, device="cuda")
    B.hlq_attn_prompt(q, k, v, q_at, k_at, out=out[:, :, 1:65].transpose(0, 1))
    assert torch.equal(out[:, :, 1:65].transpose(0, 1), want)
    assert (out[:, :, 0] == 3).all() and (out[:, :, 65:] == 3).all()
    heads = [x.transpose(0, 1).contiguous().cuda().transpose(0, 1) for x in (p.q_host, p.k_host, p.v_host)]
    assert torch.equal(B.hlq_attn_prompt(*heads, q_at, k_at)[5:-5], want[5:-5])


def test_offsets_out_of_range_stay_inside():
    p = Packed(same(40, 40), 2, 1, 64, "bf16", key=("range",))
    want = p.run()
    q_at = torch.tensor([-9, 40, 2**31 - 1], dtype=torch.int32, device="cuda")
    k_at = torch.tensor([-(2**31), 40, 99], dtype=torch.int32, device="cuda")
    got = B.hlq_attn_prompt(p.q_host.cuda(), p.k_host.cuda(), p.v_host.cuda(), q_at, k_at)
    assert torch.equal(got, want)
    down = torch.tensor([80, 40, 0], dtype=torch.int32, device="cuda")
    out = torch.full_like(got, 3.0)
    B.hlq_attn_prompt(p.q_host.cuda(), p.k_host.cuda(), p.v_host.cuda(), down, down, out=out)
    assert (out == 3).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_what_is_not_seen_does_not_show(D, dtype):
    # keys and values that are infinite or NaN in places that a query does not see; those who see them have them
    n = 200
    p = Packed(same(n), 2, 1, D, dtype, key=("odd",))
    q_at, k_at = p.offsets()
    k, v = p.k_host.cuda(), p.v_host.cuda()
    want = p.run()
    v[70, 0, 3], v[150, 0, 5], v[151, 0, 5], v[180, 0, 7] = float("inf"), float("inf"), float("-inf"), float("nan")
    got = B.hlq_attn_prompt(p.q_host.cuda(), k, v, q_at, k_at)
    changed = torch.zeros((n, 2, D), dtype=torch.bool)
    changed[70:, :, 3] = changed[150:, :, 5] = changed[180:, :, 7] = True
    assert torch.equal(got.cpu()[~changed], want.cpu()[~changed])
    assert (got[70:, :, 3] == float("inf")).all() and (got[150, :, 5] == float("inf")).all() and torch.isnan(got[151:, :, 5]).all() and torch.isnan(got[180:, :, 7]).all()
    # a window that has left them behind, and the end of the sequence's keys
    got = B.hlq_attn_prompt(p.q_host.cuda(), k, v, q_at, k_at, window=10)
    p.window = 10
    clean = p.run()
    changed[:] = False
    changed[70:80, :, 3] = changed[150:161, :, 5] = changed[180:190, :, 7] = True
    assert torch.equal(got.cpu()[~changed], clean.cpu()[~changed])
    cut = torch.tensor([0, 60], dtype=torch.int32, device="cuda")
    p.window = 0
    assert torch.isfinite(B.hlq_attn_prompt(p.q_host.cuda(), k, v, cut, cut)[:60]).all()
    k[:, 0, 0] = float("nan")
    k[:50] = p.k_host[:50].cuda()
    got = B.hlq_attn_prompt(p.q_host.cuda(), k, p.v_host.cuda(), q_at, k_at)
    assert torch.equal(got[:50], want[:50]) and torch.isnan(got[50:]).all()


def test_nothing_to_do():
    q = torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    k = torch.ones((9, 2, 64), dtype=torch.bfloat16, device="cuda")
    assert B.hlq_attn_prompt(q, k, k, torch.tensor([0, 0], dtype=torch.int32, device="cuda"), torch.tensor([0, 9], dtype=torch.int32, device="cuda")).shape == (0, 4, 64)
    out = torch.full((3, 4, 64), 2.0, dtype=torch.bfloat16, device="cuda")
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.hlq_attn_prompt(out, k, k, one, one, out=out)
    assert (out == 2).all()
    # queries without any key
    at, none = torch.tensor([0, 3], dtype=torch.int32, device="cuda"), torch.tensor([0, 0], dtype=torch.int32, device="cuda")
    got = B.hlq_attn_prompt(out, k[:0], k[:0], at, none)
    assert (got == 0).all()
