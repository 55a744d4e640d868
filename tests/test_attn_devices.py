"""Attention and its cache: operands on several devices are refused, and a call runs on the device that its operands are on, whichever is current, on the stream given
or that device's current one.  Without a GPU: stand-ins for tensors of devices that are not here, and for the library, which note what a call does."""
import pytest
import torch

from paper_2510_19482_amd import binding as B
from test_mx4_devices import Stream, Tensor, machine   # noqa: F401


class Rows(Tensor):
    """[tokens, heads, dim], contiguous."""

    def stride(self, i=None):
        s, n = [], 1
        for size in reversed(self.shape):
            s.insert(0, n)
            n *= size
        return tuple(s) if i is None else s[i]


def rows(device, T, H):
    return Rows(device, T, H, 64, dtype=torch.bfloat16)


def ints(device, *shape, dtype=torch.int32):
    return Rows(device, *shape, dtype=dtype)


def cache(device):
    return B.KvCache(Tensor(device, B.kv_bytes(3, 16, 2, 64, torch.bfloat16), dtype=torch.uint8), 3, 16, 2, 64, torch.bfloat16)


def rotary(device):
    r = B.Rotary(B.rotary_frequencies(64), device="cpu")
    object.__setattr__(r, "turns", Tensor(device, 32, dtype=torch.int64))
    object.__setattr__(r, "_device", device)
    return r


def calls(d, stream=None):
    """Each operator with its operands on devices d(0), d(1), ..."""
    long = torch.int64
    return {
        "hlq_rotary": (4, lambda: B.hlq_rotary(rows(d(0), 5, 4), ints(d(1), 5), rotary(d(2)), rows(d(3), 5, 4), stream=stream)),
        "hlq_kv_write": (4, lambda: B.hlq_kv_write(cache(d(0)), rows(d(1), 5, 2), rows(d(2), 5, 2), ints(d(3), 5, dtype=long), stream=stream)),
        "hlq_kv_write turned": (9, lambda: B.hlq_kv_write(cache(d(0)), rows(d(1), 5, 2), rows(d(2), 5, 2), ints(d(3), 5, dtype=long), rotary(d(4)), ints(d(5), 5), rows(d(6), 5, 4), rows(d(7), 5, 4),
                                                          rows(d(8), 5, 2), stream=stream)),
        "hlq_kv_read": (4, lambda: B.hlq_kv_read(cache(d(0)), ints(d(1), 5, dtype=long), rows(d(2), 5, 2), rows(d(3), 5, 2), stream=stream)),
        "hlq_attn_decode": (6, lambda: B.hlq_attn_decode(cache(d(0)), rows(d(1), 5, 4), ints(d(2), 5, 3), ints(d(3), 5), rows(d(4), 5, 4), ws=Tensor(d(5), 1 << 20, dtype=torch.uint8), stream=stream)),
        "hlq_attn_prompt": (7, lambda: B.hlq_attn_prompt(rows(d(0), 5, 4), rows(d(1), 5, 2), rows(d(2), 5, 2), ints(d(3), 3), ints(d(4), 3), rows(d(5), 5, 4),
                                                         ws=Tensor(d(6), 1 << 20, dtype=torch.uint8), stream=stream)),
    }


@pytest.fixture
def two_devices(machine, monkeypatch):   # noqa: F811
    for name in ("hlq_kv_bytes", "hlq_rotary_turns", "hlq_attn_decode_workspace_bytes", "hlq_attn_prompt_workspace_bytes"):
        setattr(B.lib, name, getattr(B._load(), name))
    return machine


@pytest.mark.parametrize("name", list(calls(lambda i: 0)))
def test_a_call_runs_where_its_operands_are(two_devices, name):
    for device in (0, 1):
        del two_devices[:]
        calls(lambda i: device)[name][1]()
        assert two_devices == [(name.split()[0], device, 100 + device)]
        del two_devices[:]
        calls(lambda i: device, Stream(device))[name][1]()
        assert two_devices == [(name.split()[0], device, 1000 + device)]


@pytest.mark.parametrize("name", list(calls(lambda i: 0)))
def test_operands_on_two_devices_and_streams_of_another_are_refused(two_devices, name):
    for odd in range(calls(lambda i: 0)[name][0]):
        for here, there in ((0, 1), (1, 0)):
            with pytest.raises(ValueError, match="one GPU"):
                calls(lambda i: there if i == odd else here)[name][1]()
    with pytest.raises(ValueError, match="stream"):
        calls(lambda i: 1, Stream(0))[name][1]()
    assert two_devices == []
