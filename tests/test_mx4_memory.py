"""Whose memory a call is handed: a matrix's is what stands in its blob at the time of the call, a route's is its own for as long as it lives.
Without a GPU: the library's entry points are replaced by ones that note their arguments."""
import copy
import pickle

import pytest
import torch

from paper_2510_19482_amd import binding as B


def matrix(rows=8, K=64):
    return B.Mx4(torch.zeros(B.mx4_bytes(rows, K), dtype=torch.uint8), rows, K)


def test_a_matrix_is_where_its_blob_is():
    m = matrix()
    other = torch.ones_like(m.blob)
    m.blob = other
    assert B._blob(m) == (other.data_ptr(), other.numel(), -1)
    third = torch.ones_like(other)
    m.blob.data = third
    assert B._blob(m) == (third.data_ptr(), third.numel(), -1)
    assert not m.is_cuda and m.device == third.device


def test_memory_that_a_call_was_handed_is_not_anothers():
    # while the matrix still has the address of its last call, nothing else can lie there
    m = matrix()
    at = m.blob.data_ptr()
    m.blob.data = torch.zeros_like(m.blob)
    assert all(torch.zeros(m._need, dtype=torch.uint8).data_ptr() != at for _ in range(100))
    assert B._blob(m)[0] == m.blob.data_ptr() != at
    m.blob.untyped_storage().resize_(0)
    with pytest.raises(ValueError):
        B._blob(m)


def test_a_blob_that_does_not_hold_the_matrix_is_refused():
    m = matrix()
    for bad in (torch.zeros(m.blob.numel() - 1, dtype=torch.uint8), torch.zeros(2 * m.blob.numel(), dtype=torch.uint8)[::2], torch.zeros(m.blob.numel(), dtype=torch.int8)):
        with pytest.raises(ValueError):
            m.blob = bad
        with pytest.raises(ValueError):
            B.Mx4(bad, 8, 64)
    for name in ("rows", "K"):
        with pytest.raises(AttributeError):
            setattr(m, name, 1 << 20)
    # past the assignment's check
    for bad in (torch.zeros(m.blob.numel() - 1, dtype=torch.uint8), torch.zeros(1, dtype=torch.uint8).expand(m.blob.numel())):
        m = matrix()
        m.blob.data = bad
        for call in (lambda: B._blob(m), lambda: B.hlq_mx4_dequantize(m, torch.zeros(8, 64)), lambda: B.hlq_mx4_gemm(m, torch.zeros(2, 64)),
                     lambda: B.hlq_mx4_unpack(m), lambda: B.hlq_mx4_quantize(torch.zeros(8, 64), m)):
            with pytest.raises(ValueError):
                call()


def test_a_matrix_moved_to_the_host_is_refused():
    m = matrix()
    m.blob = m.blob.cpu()
    with pytest.raises(ValueError, match="on the GPU"):
        B.hlq_mx4_gemm(m, torch.zeros(2, 64), torch.zeros(2, 8), ws=torch.zeros(1 << 18, dtype=torch.uint8))


def test_a_route_keeps_the_memory_that_it_writes():
    T, E, k = 300, 10, 3
    r = B.alloc_route(T, E, k, device="cpu")
    parts = [r.ids, r.weights, r.offsets, r.rows, r.slots, r.ws]
    assert [tuple(p.shape) for p in parts[:5]] == [(T, k), (T, k), (E + 1,), (T * k,), (T, k)]
    assert [p.dtype for p in parts] == [torch.int32, torch.float32, torch.int32, torch.int32, torch.int32, torch.uint8]
    assert r._args[:6] == tuple(p.data_ptr() for p in parts) and r._args[6] == r.ws.numel() and r.ws.data_ptr() % 16 == 0
    lo, hi = r._memory.data_ptr(), r._memory.data_ptr() + r._memory.numel()
    spans = sorted((p.data_ptr(), p.data_ptr() + p.nbytes) for p in parts)
    assert lo <= spans[0][0] and spans[-1][1] <= hi and all(a[1] <= b[0] for a, b in zip(spans, spans[1:]))
    with pytest.raises(AttributeError):
        r.ids = torch.zeros_like(r.ids)
    r.ids.data = torch.zeros((T, k), dtype=torch.int32)      # the caller's tensor is another now; what is written is still there
    del parts
    assert r._memory.data_ptr() == lo and r._args[0] >= lo and r._args[0] + 4 * T * k <= hi


def test_copies_have_memory_of_their_own():
    m = matrix()
    m.blob.random_(0, 255)
    r = B.alloc_route(300, 10, 3, device="cpu")
    r.ids.random_(0, 9)
    for again in (copy.deepcopy, lambda v: pickle.loads(pickle.dumps(v))):
        c = again(m)
        assert (c.rows, c.K) == (m.rows, m.K) and torch.equal(c.blob, m.blob)
        assert B._blob(c)[0] == c.blob.data_ptr() != m.blob.data_ptr()
        c = again(r)
        assert (c.T, c.E, c.k) == (r.T, r.E, r.k) and torch.equal(c.ids, r.ids)
        assert c._args[0] == c.ids.data_ptr() != r.ids.data_ptr() and c._args[5] == c.ws.data_ptr()
