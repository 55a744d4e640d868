"""Outputs that share memory with an input, or with each other, are refused; parts of one projection's rows, of which one is turned into another, are not.

Addresses are made up, so what is not refused must not run: these tests are for machines without a GPU, where a launch is an error of its own."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2510_19482_amd import binding as B
from test_attn_host import A, DECODE, PROMPT, READ, ROTARY, STRIDE, WRITE

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses")


def status(name, args):
    return getattr(B.lib, name)(*args.values(), None)


def places(at, T, heads, ts, hs, dim, size):
    """The bytes of an array."""
    t, h, d = np.ogrid[:T, :heads, :dim * size]
    return set((at + (t * ts + h * hs) * size + d).reshape(-1).tolist())


@pytest.mark.parametrize("seed", range(40))
def test_rotary_into_any_layout(seed):
    # against the sets of their bytes; arrays of unlike token strides may be refused without sharing a byte
    r = np.random.default_rng(seed)
    seen = set()
    for _ in range(60):
        T, heads, dim = int(r.integers(1, 7)), int(r.integers(1, 5)), 8 * int(r.integers(1, 3))
        pad, gap = 8 * int(r.integers(0, 3)), int(r.integers(0, 3)) * dim
        token = heads * (dim + gap) + pad
        layouts = [(token + 8 * int(r.integers(0, 2)) * heads, dim + gap), (dim, T * dim + pad), (2 * token, dim), (token, dim + gap)]
        (xt, xh), (yt, yh) = layouts[r.integers(4)], layouts[r.integers(4)]
        kind, size = ((0, 2), (1, 4))[r.integers(2)]
        x = A + 4 * int(r.integers(0, 400))
        y = x if r.random() < 0.1 else A + 4 * int(r.integers(0, 400))
        got = status("hlq_rotary", {**ROTARY, "r": B.HlqRotaryDesc(dim, 0, 1.0, A), "T": T, "heads": heads, "dim": dim, "type": kind, "x": x, "x_ts": xt, "x_hs": xh, "y": y, "y_ts": yt, "y_hs": yh})
        own = len(places(y, T, heads, yt, yh, dim, size)) == T * heads * dim * size
        if not own:
            assert got == STRIDE
            continue
        one = x == y and (T == 1 or xt == yt) and (heads == 1 or xh == yh)
        share = bool(places(x, T, heads, xt, xh, dim, size) & places(y, T, heads, yt, yh, dim, size)) and not one
        if share:
            assert got == STRIDE
        elif xt == yt or T == 1:
            assert got != STRIDE
        seen.add((share, got == STRIDE))
    assert (True, True) in seen and (False, False) in seen


FUSED = 8 * 64 + 16   # q (4 heads), k (2) and v (2) of 64 in a row, and something behind


@pytest.mark.parametrize("change,refused", [
    (dict(), False), (dict(k_out=A + 256 * 2), False), (dict(q_out=A, k_out=None), False), (dict(k_out=A + 256 * 2 + 2), True), (dict(k_out=A + 384 * 2), True), (dict(k_out=A), True),
    (dict(q_out=A + 64 * 2), True), (dict(q_out=A + 256 * 2), True), (dict(q_out=A + FUSED * 2), True), (dict(q_out=A + 3 * FUSED * 2), False), (dict(q_out=1 << 30, k_out=(1 << 30) + 64 * 2), True),
    (dict(q_out=1 << 30, k_out=(1 << 30) + 256 * 2), False)], ids=str)
def test_write(change, refused):
    places = dict(k=A + 256 * 2, v=A + 384 * 2, q=A, k_ts=FUSED, v_ts=FUSED, q_ts=FUSED, ko_ts=FUSED, qo_ts=FUSED, k_out=1 << 28, q_out=1 << 29)
    assert (status("hlq_kv_write", {**WRITE, **places, **change}) == STRIDE) == refused


def test_read_decode_and_prompt():
    assert status("hlq_kv_read", READ) == STRIDE
    assert status("hlq_kv_read", {**READ, "v": A + 64 * 2}) == STRIDE
    assert status("hlq_kv_read", {**READ, "v": A + 3 * 128 * 2}) != STRIDE
    assert status("hlq_kv_read", {**READ, "k_ts": 256, "v_ts": 256, "v": A + 128 * 2}) != STRIDE
    assert status("hlq_kv_read", {**READ, "v": None}) != STRIDE
    assert status("hlq_attn_decode", DECODE) != STRIDE
    assert status("hlq_attn_decode", {**DECODE, "otype": B.HLQ_F32}) == STRIDE
    assert status("hlq_attn_decode", {**DECODE, "out": A + 64 * 2}) == STRIDE
    far = dict(k=1 << 28, v=1 << 29)
    assert status("hlq_attn_prompt", {**PROMPT, **far}) != STRIDE
    assert status("hlq_attn_prompt", PROMPT) == STRIDE
    assert status("hlq_attn_prompt", {**PROMPT, **far, "out": (1 << 28) + 8 * 128 * 2}) == STRIDE
    assert status("hlq_attn_prompt", {**PROMPT, **far, "out": (1 << 29) - 9 * 256 * 2}) != STRIDE
    assert status("hlq_attn_prompt", {**PROMPT, **far, "o_ts": 264}) == STRIDE


def test_addresses_and_strides_at_their_ends():
    top = (1 << 64) - (1 << 20)
    huge = {**ROTARY, "T": 2**31 - 1, "x_ts": 1 << 40, "y_ts": 1 << 40, "x": A, "y": A + 256}
    assert status("hlq_rotary", huge) != STRIDE
    assert status("hlq_rotary", {**huge, "y": A + 128}) == STRIDE
    assert status("hlq_rotary", {**ROTARY, "x": ctypes.c_void_p(top), "y": A}) != STRIDE
    assert status("hlq_rotary", {**ROTARY, "x": ctypes.c_void_p(top), "y": ctypes.c_void_p(top + 128)}) == STRIDE
