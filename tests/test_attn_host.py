"""Attention and its cache without a GPU: sizes, what is refused and how, frequencies of rotary positions.  No call here launches anything: addresses are
made up, and every one of these calls is refused (or has nothing to do) before the library would look behind them."""
import copy
import ctypes
import math
import pickle

import numpy as np
import pytest
import torch

from oracle import attn_oracle as O
from paper_2510_19482_amd import binding as B

NULL, DESC, UNSUPPORTED, SMALL, STRIDE = 1, 2, 3, 4, 5
A = 0x10000   # an address


def desc(pages=10, page=16, heads=2, dim=64, kind=B.HLQ_BF16):
    return B.HlqKvDesc(pages, page, heads, dim, kind)


def rotary(dims=64, turns=A):
    return B.HlqRotaryDesc(dims, 0, 1.0, turns)


@pytest.mark.parametrize("kind,bits", [(torch.float16, 16), (torch.bfloat16, 16), (B.HLQ_MX8, 8.25), (B.HLQ_MX4, 4.25)])
def test_sizes(kind, bits):
    for pages, page, heads, dim in ((1, 16, 1, 32), (7, 64, 8, 128), (3, 1024, 5, 256), (2**31 - 1, 128, 8, 128)):
        assert B.kv_bytes(pages, page, heads, dim, kind) == int(pages * page * heads * dim * 2 * bits) // 8


@pytest.mark.parametrize("change,status", [
    (dict(pages=0), DESC), (dict(pages=-1), DESC), (dict(page=8), DESC), (dict(page=24), DESC), (dict(page=2048), DESC), (dict(heads=0), DESC), (dict(dim=0), DESC), (dict(dim=4), DESC),
    (dict(dim=60), DESC), (dict(dim=40, kind=B.HLQ_MX8), DESC), (dict(dim=72, kind=B.HLQ_MX4), DESC), (dict(pages=2**31), UNSUPPORTED), (dict(heads=1025), UNSUPPORTED),
    (dict(dim=264), UNSUPPORTED), (dict(kind=B.HLQ_F32), UNSUPPORTED), (dict(kind=5), UNSUPPORTED), (dict(kind=-1), UNSUPPORTED)])
def test_caches_that_are_refused(change, status):
    n = ctypes.c_size_t()
    d = desc(**change)
    assert B.lib.hlq_kv_bytes(d, ctypes.byref(n)) == status
    assert B.lib.hlq_attn_decode_workspace_bytes(d, 2, 1, 1, ctypes.byref(n)) == status
    assert B.lib.hlq_kv_read(d, A, 1 << 40, 1, A, 0, A, 128, 64, A, 128, 64, None) == status
    assert B.lib.hlq_kv_bytes(None, ctypes.byref(n)) == NULL and B.lib.hlq_kv_bytes(desc(), None) == NULL


ROTARY = dict(r=rotary(), T=3, heads=2, dim=64, type=0, positions=A, x=A, x_ts=128, x_hs=64, y=A, y_ts=128, y_hs=64)
WRITE = dict(c=desc(), cache=A, bytes=1 << 30, T=3, type=0, k=A, k_ts=128, k_hs=64, v=A, v_ts=128, v_hs=64, slots=A, r=rotary(), positions=A, k_out=A, ko_ts=128, ko_hs=64, q_heads=4,
             q=A, q_ts=256, q_hs=64, q_out=A, qo_ts=256, qo_hs=64)
READ = dict(c=desc(), cache=A, bytes=1 << 30, T=3, slots=A, type=0, k=A, k_ts=128, k_hs=64, v=A, v_ts=128, v_hs=64)
DECODE = dict(c=desc(), cache=A, bytes=1 << 30, q_heads=4, B=3, type=B.HLQ_BF16, q=A, q_ts=256, q_hs=64, table=A, ld=100, width=100, lengths=A, window=0, scale=1.0, out=A, otype=B.HLQ_BF16,
              o_ts=256, o_hs=64, ws=A, ws_bytes=1 << 30)
PROMPT = dict(B=2, q_heads=4, heads=2, dim=64, type=0, Tq=9, q=A, q_ts=256, q_hs=64, Tk=9, k=A, k_ts=128, k_hs=64, v=A, v_ts=128, v_hs=64, q_offsets=A, k_offsets=A, causal=1, window=0,
              scale=1.0, out=A, o_ts=256, o_hs=64, ws=A, ws_bytes=1 << 30)

REFUSED = [
    ("hlq_rotary", ROTARY, [
        (dict(r=None), NULL), (dict(r=rotary(0)), DESC), (dict(r=rotary(7)), DESC), (dict(r=rotary(66)), DESC), (dict(r=rotary(turns=None)), NULL), (dict(r=rotary(turns=A + 4)), STRIDE),
        (dict(positions=None), NULL), (dict(positions=A + 2), STRIDE), (dict(x=None), NULL), (dict(y=None), NULL), (dict(x=A + 1), STRIDE), (dict(type=1, y=A + 2), STRIDE), (dict(T=-1), DESC),
        (dict(T=2**31), UNSUPPORTED), (dict(heads=0), DESC), (dict(heads=1025), UNSUPPORTED), (dict(dim=60), DESC), (dict(dim=264), UNSUPPORTED), (dict(type=3), UNSUPPORTED), (dict(type=4), UNSUPPORTED),
        (dict(x_ts=-1), STRIDE), (dict(y_ts=127), STRIDE), (dict(y_hs=63), STRIDE), (dict(y_ts=0, y_hs=64), STRIDE), (dict(y_ts=64, y_hs=128), STRIDE), (dict(x_ts=1 << 41), STRIDE)]),
    ("hlq_kv_write", WRITE, [
        (dict(c=None), NULL), (dict(cache=None), NULL), (dict(cache=A + 8), STRIDE), (dict(bytes=10 * 16 * 2 * 64 * 4 - 1), SMALL), (dict(T=-1), DESC), (dict(T=2**31), UNSUPPORTED), (dict(type=3), UNSUPPORTED),
        (dict(k=None), NULL), (dict(v=None), NULL), (dict(slots=None), NULL), (dict(slots=A + 4), STRIDE), (dict(k_ts=-1), STRIDE), (dict(v_hs=-1), STRIDE), (dict(r=rotary(80)), DESC),
        (dict(positions=None), NULL), (dict(r=None), DESC), (dict(r=None, q_heads=0), DESC), (dict(r=None, k_out=None), DESC), (dict(ko_ts=100), STRIDE), (dict(q_heads=-1), DESC), (dict(q_heads=2000), UNSUPPORTED),
        (dict(q=None), NULL), (dict(q_out=None), NULL), (dict(qo_hs=32), STRIDE), (dict(q=A + 1), STRIDE)]),
    ("hlq_kv_read", READ, [
        (dict(cache=None), NULL), (dict(cache=A + 8), STRIDE), (dict(bytes=100), SMALL), (dict(slots=None), NULL), (dict(slots=A + 4), STRIDE), (dict(type=4), UNSUPPORTED), (dict(T=-1), DESC),
        (dict(k_ts=0), STRIDE), (dict(v_hs=0), STRIDE), (dict(k=A + 1), STRIDE)]),
    ("hlq_attn_decode", DECODE, [
        (dict(c=None), NULL), (dict(cache=None), NULL), (dict(cache=A + 8), STRIDE), (dict(bytes=100), SMALL), (dict(q_heads=3), DESC), (dict(q_heads=0), DESC), (dict(q_heads=1026), UNSUPPORTED), (dict(B=-1), DESC),
        (dict(B=1 << 24), UNSUPPORTED), (dict(type=B.HLQ_F16), UNSUPPORTED), (dict(type=B.HLQ_F32), UNSUPPORTED), (dict(otype=3), UNSUPPORTED), (dict(q=None), NULL), (dict(q_ts=-1), STRIDE), (dict(table=None), NULL),
        (dict(table=A + 2), STRIDE), (dict(ld=99), STRIDE), (dict(width=-1), DESC), (dict(width=2**27), UNSUPPORTED), (dict(lengths=None), NULL), (dict(lengths=A + 1), STRIDE), (dict(window=-1), DESC),
        (dict(out=None), NULL), (dict(o_ts=0), STRIDE), (dict(ws=None), NULL), (dict(ws=A + 8), STRIDE), (dict(ws_bytes=131072), SMALL)]),
    ("hlq_attn_prompt", PROMPT, [
        (dict(B=-1), DESC), (dict(q_heads=3), DESC), (dict(heads=0), DESC), (dict(dim=60), DESC), (dict(dim=264), UNSUPPORTED), (dict(q_heads=2048), UNSUPPORTED), (dict(type=1), UNSUPPORTED), (dict(type=3), UNSUPPORTED),
        (dict(Tq=-1), DESC), (dict(Tk=-1), DESC), (dict(Tq=2**31), UNSUPPORTED), (dict(Tk=2**31), UNSUPPORTED), (dict(q=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(out=None), NULL),
        (dict(q_offsets=None), NULL), (dict(k_offsets=None), NULL), (dict(q_offsets=A + 2), STRIDE), (dict(window=-1), DESC), (dict(o_ts=255), STRIDE), (dict(k_ts=-4), STRIDE), (dict(v=A + 1), STRIDE)]),
]


@pytest.mark.parametrize("name,args,change,status", [(n, a, c, s) for n, a, every in REFUSED for c, s in every], ids=lambda v: "-".join(v) if isinstance(v, dict) and len(v) < 4 else v if isinstance(v, str) else "")
def test_calls_that_are_refused(name, args, change, status):
    assert set(change) <= set(args)
    assert getattr(B.lib, name)(*{**args, **change}.values(), None) == status


@pytest.mark.parametrize("name,args,change", [("hlq_rotary", ROTARY, dict(T=0)), ("hlq_kv_write", WRITE, dict(T=0)), ("hlq_kv_read", READ, dict(T=0)), ("hlq_kv_read", READ, dict(k=None, v=None)),
                                              ("hlq_attn_decode", DECODE, dict(B=0)), ("hlq_attn_prompt", PROMPT, dict(Tq=0)), ("hlq_attn_prompt", PROMPT, dict(B=0))])
def test_nothing_to_do(name, args, change):
    assert getattr(B.lib, name)(*{**args, **change}.values(), None) == 0


def test_workspaces_serve_smaller_calls():
    n = ctypes.c_size_t()

    def need(heads, q_heads, batch, width, dim=128, page=64):
        assert B.lib.hlq_attn_decode_workspace_bytes(desc(10, page, heads, dim), q_heads, batch, width, ctypes.byref(n)) == 0
        return n.value

    for heads, q_heads in ((8, 32), (1, 16), (8, 8), (1, 64)):
        for batch in (1, 3, 17, 100, 1000):
            for width in (1, 5, 40, 300, 2048):
                most = need(heads, q_heads, batch, width)
                assert 131072 <= most < 1 << 31
                for b in {1, 2, batch // 3, batch // 2, batch - 1} & set(range(1, batch + 1)):
                    for w in {0, 1, 2, width // 7, width // 2, width - 1} & set(range(width + 1)):
                        assert need(heads, q_heads, b, w) <= most


def test_turns_of_frequencies():
    f = [1.0, 1e-4, 0.0, 2 * math.pi, 1e9, -1.0, 5e-324]
    got = (ctypes.c_uint64 * len(f))()
    assert B.lib.hlq_rotary_turns(len(f), (ctypes.c_double * len(f))(*f), got) == 0
    for x, t in zip(f, got):
        turn = np.longdouble(x) / (2 * np.longdouble("3.14159265358979323846264338327950288"))
        off = abs(float((np.longdouble(t) / np.longdouble(2)**64 - turn) % 1))
        assert min(off, 1 - off) <= 2.0**-64 * (2 + abs(x))
    for bad in (math.inf, -math.inf, math.nan, 2.0**32, -2.0**40):
        assert B.lib.hlq_rotary_turns(2, (ctypes.c_double * 2)(1.0, bad), got) == DESC
    assert B.lib.hlq_rotary_turns(0, (ctypes.c_double * 1)(1.0), got) == DESC and B.lib.hlq_rotary_turns(129, (ctypes.c_double * 1)(1.0), got) == DESC
    assert B.lib.hlq_rotary_turns(1, None, got) == NULL


def test_frequencies():
    assert B.rotary_frequencies(4, 100.0) == [1.0, 0.1]
    assert B.rotary_frequencies(4, 100.0, 4.0) == [0.25, 0.025]
    f = B.rotary_frequencies(128, 500000.0)
    g = B.rotary_frequencies(128, 500000.0, 8.0, 8192)
    for a, b in zip(f, g):
        turns = 8192 * a / (2 * math.pi)
        assert b == a if turns >= 4 else b == a / 8 if turns <= 1 else a / 8 < b < a
    for bad in (dict(dims=3), dict(dims=0), dict(dims=4, base=0.0), dict(dims=4, factor=0.0), dict(dims=4, keep=(2.0, 2.0))):
        with pytest.raises(ValueError):
            B.rotary_frequencies(**bad)


def test_a_cache_and_a_rotation_stay_as_they_were_made_and_can_be_copied():
    kv = B.alloc_kv_cache(3, 16, 2, 32, torch.bfloat16, device="cpu")
    kv.blob.copy_(torch.arange(kv.blob.numel()) % 251)
    for again in (copy.deepcopy(kv), pickle.loads(pickle.dumps(kv))):
        assert torch.equal(again.blob, kv.blob) and again.blob.data_ptr() != kv.blob.data_ptr()
        assert (again.pages, again.page, again.heads, again.dim, again.type) == (3, 16, 2, 32, B.HLQ_BF16)
    assert kv.rows.shape == (3, 2, 2, 16, 32) and kv.rows.data_ptr() == kv.blob.data_ptr()
    r = B.Rotary(B.rotary_frequencies(32), True, 1.5, device="cpu")
    for again in (copy.deepcopy(r), pickle.loads(pickle.dumps(r))):
        assert torch.equal(again.turns, r.turns) and again.frequencies == r.frequencies and again.interleaved and again.magnitude == 1.5
        assert again._desc.turns == again.turns.data_ptr()
    for thing, name in ((kv, "blob"), (kv, "pages"), (r, "turns"), (r, "magnitude")):
        with pytest.raises(AttributeError):
            setattr(thing, name, 1)
    with pytest.raises(ValueError):
        B.alloc_kv_cache(3, 16, 2, 32, B.HLQ_MX4, device="cpu").rows
    with pytest.raises(ValueError):
        B.KvCache(kv.blob[:-1], 3, 16, 2, 32, torch.bfloat16)
    with pytest.raises(ValueError):
        B.KvCache(kv.blob.view(torch.int8), 3, 16, 2, 32, torch.bfloat16)
    with pytest.raises(B.HlqError):
        B.alloc_kv_cache(3, 16, 2, 32, torch.float32, device="cpu")


def test_the_oracles_formats():
    # every code's value is its own code again, halves between neighbours go to the even one
    values = O.E4M3
    assert values[126] == 448 and values[1] == 2.0**-9 and (np.diff(values) > 0).all()
    x = np.concatenate([values, np.full(-len(values) % 31, 0.0)]).reshape(-1, 31)
    x = np.concatenate([x, np.full((len(x), 1), 448.0)], 1)
    codes, scales = O.mx8_quantize(x)
    assert (scales == 127).all() and (codes[:, :31].reshape(-1)[:127] == np.arange(127)).all()
    mid = (values[1:] + values[:-1]) / 2
    x = np.concatenate([mid, np.zeros(-len(mid) % 31)]).reshape(-1, 31)
    codes, _ = O.mx8_quantize(np.concatenate([x, np.full((len(x), 1), 448.0)], 1))
    assert (codes[:, :31].reshape(-1)[:126] == np.arange(126) + np.arange(126) % 2).all()


def tensors(**change):
    """Arguments of each operator on the CPU, with some of them changed."""
    T = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype)   # noqa: E731
    a = dict(cache=B.alloc_kv_cache(3, 16, 2, 32, torch.bfloat16, device="cpu"), rotary=B.Rotary(B.rotary_frequencies(32), device="cpu"), q=T(5, 4, 32), k=T(5, 2, 32), v=T(5, 2, 32),
             slots=T(5, dtype=torch.int64), positions=T(5, dtype=torch.int32), table=T(5, 2, dtype=torch.int32), lengths=T(5, dtype=torch.int32), q_offsets=T(3, dtype=torch.int32),
             k_offsets=T(3, dtype=torch.int32), out=T(5, 4, 32), k_out=T(5, 2, 32), ws=T(1 << 20, dtype=torch.uint8))
    return {**a, **change}


CALLS = {
    "rotary": lambda a: B.hlq_rotary(a["q"], a["positions"], a["rotary"], a["out"]),
    "write": lambda a: B.hlq_kv_write(a["cache"], a["k"], a["v"], a["slots"], a["rotary"], a["positions"], a["q"], a["out"], a["k_out"]),
    "read": lambda a: B.hlq_kv_read(a["cache"], a["slots"], a["k"], a["v"]),
    "decode": lambda a: B.hlq_attn_decode(a["cache"], a["q"], a["table"], a["lengths"], a["out"], ws=a["ws"]),
    "prompt": lambda a: B.hlq_attn_prompt(a["q"], a["k"], a["v"], a["q_offsets"], a["k_offsets"], a["out"], ws=a["ws"]),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_tensors_that_are_not_on_a_gpu_are_refused(name):
    with pytest.raises(ValueError, match="one GPU"):
        CALLS[name](tensors())


Z = torch.zeros
BF = torch.bfloat16


@pytest.mark.parametrize("name,change,error", [
    ("rotary", dict(q=Z(5, 4, 32, dtype=torch.float64)), TypeError), ("rotary", dict(q=Z(5, 128, dtype=BF)), ValueError), ("rotary", dict(out=Z(5, 4, 32)), ValueError),
    ("rotary", dict(q=Z(5, 32, 4, dtype=BF).transpose(1, 2)), ValueError), ("rotary", dict(positions=Z(5, dtype=torch.int64)), ValueError), ("rotary", dict(positions=Z(4, dtype=torch.int32)), ValueError),
    ("rotary", dict(positions=Z(10, dtype=torch.int32)[::2]), ValueError),
    ("write", dict(k=Z(5, 1, 32, dtype=BF)), ValueError), ("write", dict(k=Z(5, 2, 64, dtype=BF)), ValueError), ("write", dict(v=Z(4, 2, 32, dtype=BF)), ValueError), ("write", dict(v=Z(5, 2, 32)), ValueError),
    ("write", dict(slots=Z(5, dtype=torch.int32)), ValueError), ("write", dict(rotary=None), ValueError), ("write", dict(rotary=None, q=None, k_out=None), ValueError), ("write", dict(positions=None), ValueError),
    ("write", dict(q=Z(5, 4, 64, dtype=BF)), ValueError), ("write", dict(q=Z(4, 4, 32, dtype=BF)), ValueError), ("write", dict(out=Z(5, 3, 32, dtype=BF)), ValueError), ("write", dict(q=None), ValueError),
    ("write", dict(k_out=Z(5, 2, 32)), ValueError),
    ("read", dict(k=Z(5, 2, 32)), ValueError), ("read", dict(v=Z(5, 3, 32, dtype=BF)), ValueError), ("read", dict(slots=Z(5, 1, dtype=torch.int64)), ValueError),
    ("decode", dict(q=Z(5, 4, 64, dtype=BF)), ValueError), ("decode", dict(out=Z(5, 4, 32, dtype=torch.int32)), TypeError), ("decode", dict(out=Z(4, 4, 32)), ValueError),
    ("decode", dict(table=Z(4, 2, dtype=torch.int32)), ValueError), ("decode", dict(table=Z(5, 2, dtype=torch.int64)), ValueError), ("decode", dict(table=Z(2, 5, dtype=torch.int32).T), ValueError),
    ("decode", dict(lengths=Z(4, dtype=torch.int32)), ValueError),
    ("prompt", dict(q=Z(5, 4, 64, dtype=BF)), ValueError), ("prompt", dict(k=Z(5, 2, 32, dtype=torch.float16)), ValueError), ("prompt", dict(v=Z(6, 2, 32, dtype=BF)), ValueError),
    ("prompt", dict(out=Z(5, 4, 32)), ValueError), ("prompt", dict(k_offsets=Z(2, dtype=torch.int32)), ValueError), ("prompt", dict(q_offsets=Z(0, dtype=torch.int32), k_offsets=None), ValueError)])
def test_tensors_that_do_not_fit_are_refused(name, change, error):
    with pytest.raises(error):
        CALLS[name](tensors(**change))


def test_a_workspace_for_many_sequences_serves_a_few():
    # more than there are counters for: those calls are not cut, calls of fewer sequences on the same workspace are
    n = ctypes.c_size_t()
    d = desc(10, 64, 8, 128)
    assert B.lib.hlq_attn_decode_workspace_bytes(d, 8, 5000, 40, ctypes.byref(n)) == 0
    many = n.value
    for batch in (1, 7, 100, 1000, 4095, 4096):
        assert B.lib.hlq_attn_decode_workspace_bytes(d, 8, batch, 40, ctypes.byref(n)) == 0
        assert n.value <= many


@pytest.mark.parametrize("rows", [dict(Tq=2**30), dict(Tk=2**30), dict(B=2**30)])
def test_prompts_past_the_limit_are_refused(rows):
    assert B.lib.hlq_attn_prompt(*{**PROMPT, **rows}.values(), None) == UNSUPPORTED


def test_numbers_past_32_bits_are_refused():
    with pytest.raises(ValueError, match="32 bits"):
        B.alloc_kv_cache(3, 16 + 2**32, 2, 32, torch.bfloat16, device="cpu")
    with pytest.raises(ValueError, match="32 bits"):
        B.kv_bytes(3, 16, 2 + 2**32, 32, torch.bfloat16)
    a = tensors()
    for window in (2**31, 2**32 + 5):
        with pytest.raises(ValueError, match="window"):
            B.hlq_attn_decode(a["cache"], a["q"], a["table"], a["lengths"], window=window, ws=a["ws"])
        with pytest.raises(ValueError, match="window"):
            B.hlq_attn_prompt(a["q"], a["k"], a["v"], a["q_offsets"], a["k_offsets"], window=window, ws=a["ws"])
    with pytest.raises(ValueError, match="32 bits"):
        B.decode_workspace_bytes(a["cache"], 4, 1, 2**32)
    with pytest.raises(ValueError, match="32 bits"):
        B.prompt_workspace_bytes(5, 5, 2**32, 4, 2, 32)


def test_an_array_of_nothing_may_have_any_strides():
    # as one made of an empty numpy array has
    nothing = torch.from_numpy(np.zeros((0, 2, 32))).to(torch.bfloat16)
    empty = nothing.as_strided((0, 2, 32), (0, 0, 0))
    with pytest.raises(ValueError, match="one GPU"):
        CALLS["prompt"](tensors(k=empty, v=empty))
