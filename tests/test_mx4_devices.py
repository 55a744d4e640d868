"""Operands on several devices are refused, and a call runs on the device that its operands are on, whichever is current.  Without a GPU:
stand-ins for tensors of devices that are not here, and for the library, which note what a call does."""
import contextlib

import pytest
import torch

from paper_2510_19482_amd import binding as B


class Tensor:
    """A matrix or vector on a device."""

    def __init__(self, device, *shape, dtype=torch.float32):
        self.index, self.shape, self.dtype, self.device, self.is_cuda = device, torch.Size(shape), dtype, torch.device("cuda", device), True

    def get_device(self):
        return self.index

    def stride(self, i=None):
        s = (self.shape[1], 1) if len(self.shape) == 2 else (1,)
        return s if i is None else s[i]

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x1000

    def detach(self):
        return self


class Stream:
    def __init__(self, device):
        self.device_index, self.cuda_stream = device, 1000 + device


@pytest.fixture
def machine(monkeypatch):
    """Two devices, the first current; the list of what was launched: name, device that was current, stream."""
    launched, current = [], [0]

    class Library:
        def __getattr__(self, name):
            def call(*args):
                launched.append((name, current[0], args[-1]))
                return 0
            return call

    @contextlib.contextmanager
    def on(device):
        before, current[0] = current[0], torch.device("cuda", device).index if isinstance(device, int) else device.index
        yield
        current[0] = before

    sizes = B.lib
    library = Library()
    for name in ("hlq_mx4_bytes", "hlq_mx4_workspace_bytes", "hlq_route_workspace_bytes"):
        setattr(library, name, getattr(sizes, name))
    monkeypatch.setattr(B, "lib", library)
    monkeypatch.setattr(torch.cuda, "device", on)
    monkeypatch.setattr(B, "_current_device", lambda: current[0])
    monkeypatch.setattr(B, "_current_stream", lambda device: 100 + device)
    return launched


def matrix(device, rows=8, K=64):
    return B.Mx4(Tensor(device, B.mx4_bytes(rows, K), dtype=torch.uint8), rows, K)


def calls(d, stream=None):
    """Each operator with its operands on devices d(0), d(1), ..."""
    u8, i32 = torch.uint8, torch.int32
    ws = 1 << 20

    def route(device):
        r = B.alloc_route(5, 8, 2, device="cpu")
        object.__setattr__(r, "_device", device)
        return r

    return {
        "hlq_mx4_quantize": (2, lambda: B.hlq_mx4_quantize(Tensor(d(0), 8, 64), matrix(d(1)), stream=stream)),
        "hlq_mx4_dequantize": (2, lambda: B.hlq_mx4_dequantize(matrix(d(0)), Tensor(d(1), 8, 64), stream=stream)),
        "hlq_mx4_pack": (3, lambda: B.hlq_mx4_pack(Tensor(d(0), 8, 32, dtype=u8), Tensor(d(1), 8, 2, dtype=u8), 64, matrix(d(2)), stream=stream)),
        "hlq_mx4_gemm": (4, lambda: B.hlq_mx4_gemm(matrix(d(0)), Tensor(d(1), 5, 64), Tensor(d(2), 5, 8), ws=Tensor(d(3), ws, dtype=u8), stream=stream)),
        "hlq_mx4_gemm of a matrix": (4, lambda: B.hlq_mx4_gemm(matrix(d(0)), matrix(d(1), 5), Tensor(d(2), 5, 8), ws=Tensor(d(3), ws, dtype=u8), stream=stream)),
        "hlq_expert_gemm": (6, lambda: B.hlq_expert_gemm(matrix(d(0)), Tensor(d(1), 3, dtype=i32), Tensor(d(2), 5, 64), Tensor(d(3), 5, 4), ws=Tensor(d(4), ws, dtype=u8),
                                                         rows=Tensor(d(5), 5, dtype=i32), stream=stream)),
        "hlq_route": (2, lambda: B.hlq_route(Tensor(d(0), 5, 8), 2, out=route(d(1)), stream=stream)),
        "hlq_expert_combine": (4, lambda: B.hlq_expert_combine(Tensor(d(0), 10, 8), Tensor(d(1), 5, 2, dtype=i32), Tensor(d(2), 5, 2), Tensor(d(3), 5, 8), stream=stream)),
    }


@pytest.mark.parametrize("name", list(calls(lambda i: 0)))
def test_a_call_runs_where_its_operands_are(machine, name):
    for device in (0, 1):
        del machine[:]
        calls(lambda i: device)[name][1]()
        assert machine == [(name.split()[0], device, 100 + device)]
        del machine[:]
        calls(lambda i: device, Stream(device))[name][1]()
        assert machine == [(name.split()[0], device, 1000 + device)]


@pytest.mark.parametrize("name", list(calls(lambda i: 0)))
def test_operands_on_two_devices_and_streams_of_another_are_refused(machine, name):
    for odd in range(calls(lambda i: 0)[name][0]):
        for here, there in ((0, 1), (1, 0)):
            with pytest.raises(ValueError, match="one GPU"):
                calls(lambda i: there if i == odd else here)[name][1]()
    with pytest.raises(ValueError, match="stream"):
        calls(lambda i: 1, Stream(0))[name][1]()
    assert machine == []
