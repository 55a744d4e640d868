"""Workspaces of attention: a call without one makes one only where its launch is cut over the keys, and one made for more rows, sequences or pages serves fewer.  Without a GPU."""
import ctypes

import pytest
import torch

from paper_2510_19482_amd import binding as B
from test_attn_devices import cache, ints, rows, two_devices   # noqa: F401
from test_mx4_devices import Tensor, machine   # noqa: F401

NULL = 1

CALLS = {
    "hlq_attn_decode": lambda ws=None: B.hlq_attn_decode(cache(0), rows(0, 5, 4), ints(0, 5, 3), ints(0, 5), rows(0, 5, 4), ws=ws),
    "hlq_attn_prompt": lambda ws=None: B.hlq_attn_prompt(rows(0, 5, 4), rows(0, 5, 2), rows(0, 5, 2), ints(0, 3), ints(0, 3), rows(0, 5, 4), ws=ws),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_none_is_made_where_none_is_needed(two_devices, name, monkeypatch):   # noqa: F811
    monkeypatch.setattr(B, "_empty", lambda *a: pytest.fail("memory was asked for"))
    CALLS[name]()
    assert [call for call, *_ in two_devices] == [name]


@pytest.mark.parametrize("name", list(CALLS))
def test_one_is_made_where_the_launch_is_cut(two_devices, name, monkeypatch):   # noqa: F811
    made, given = [], []

    def launch(*args):
        given.append(args[-3:-1])
        two_devices.append((name, 0, args[-1]))
        return NULL if args[-3] is None else 0

    def empty(shape, dtype, device, stream):
        made.append(shape)
        return Tensor(0, shape, dtype=dtype)

    setattr(B.lib, name, launch)
    monkeypatch.setattr(B, "_empty", empty)
    monkeypatch.setattr(B, "_ptr", lambda t: t.data_ptr())
    CALLS[name]()
    assert [call for call, *_ in two_devices] == [name, "hlq_workspace_init", name]
    assert given == [(None, 0), (0x1000, made[0])] and len(made) == 1
    # an error of a call that was given one is its own
    monkeypatch.setattr(B, "status_string", str)
    setattr(B.lib, name, lambda *args: NULL)
    with pytest.raises(B.HlqError):
        CALLS[name](Tensor(0, 1 << 20, dtype=torch.uint8))


def test_a_prompts_workspace_serves_smaller_calls():
    n = ctypes.c_size_t()

    def need(Tq, Tk, batch, q_heads, heads, dim):
        assert B.lib.hlq_attn_prompt_workspace_bytes(Tq, Tk, batch, q_heads, heads, dim, ctypes.byref(n)) == 0
        return n.value

    sizes = (0, 1, 31, 32, 33, 100, 511, 512, 1000, 4096, 20000)
    for q_heads, heads, dim in ((32, 8, 128), (8, 8, 64), (16, 1, 256), (6, 2, 96), (40, 40, 64), (12, 4, 136)):
        table = {(q, k, b): need(q, k, b, q_heads, heads, dim) for q in sizes for k in sizes + (131072,) for b in (0, 1, 2, 7, 64, 5000)}
        for (q, k, b), most in table.items():
            for i in range(3):      # one size at a time made smaller, which leads to every smaller call
                at = [sizes + (131072,), sizes + (131072,), (0, 1, 2, 7, 64, 5000)][i]
                below = [x for x in at if x < (q, k, b)[i]]
                if below:
                    less = [q, k, b]
                    less[i] = below[-1]
                    if tuple(less) in table:
                        assert table[tuple(less)] <= most


def test_a_workspace_is_on_a_gpu():
    with pytest.raises(ValueError, match="on a GPU"):
        B.alloc_prompt_workspace(5, 5, 1, 4, 2, 64, device="cpu")
