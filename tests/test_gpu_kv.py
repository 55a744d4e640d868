"""Rotary positions and rows into and out of the paged cache, against the 64-bit oracle.

A turned value is made in 64 bits, where angles are off by 2^-33 turns at most, rounded to f32 and then to its type: half a step of f32 and half a step of
the type, and 2^-30 of the pair's magnitudes for the angle.  What the cache holds is exact by definition."""
import numpy as np
import pytest
import torch

from attn_util import HALF_STEP, KINDS, SMALLEST, TYPES, Cache, host, rng, rounded, stored
from oracle import attn_oracle as O
from paper_2510_19482_amd import binding as B

pytestmark = pytest.mark.gpu


def frequencies(dims):
    return B.rotary_frequencies(dims)


def check_turned(got, x, positions, f, interleaved, magnitude, dtype):
    y = O.turned(x, positions, f, interleaved, np.float32(magnitude))
    n = 2 * len(f)
    a = np.abs(x[..., :n])
    pair = np.zeros_like(x)
    pair[..., :n] = np.repeat(a[..., 0::2] + a[..., 1::2], 2, -1) if interleaved else np.tile(a[..., :n // 2] + a[..., n // 2:], 2)
    e = 2.0**-30 * abs(magnitude) * pair
    e = e + 2.0**-24 * (np.abs(y) + e)
    if dtype != "f32":
        e = e + HALF_STEP[dtype] * (np.abs(y) + e)
    e = e + SMALLEST[dtype]
    assert not (~(np.abs(got - y) <= e)).any(), f"worst {np.max(np.abs(got - y) / e):.3g} times the bound"
    np.testing.assert_array_equal(got[..., n:], x[..., n:])


SHAPES = [(1, 1, 8, 2), (3, 5, 128, 128), (7, 2, 64, 32), (33, 3, 96, 48), (5, 4, 40, 20), (2, 9, 256, 256), (130, 40, 128, 64), (9, 1, 120, 6), (4, 3, 72, 72), (1, 80, 16, 16), (600, 2, 24, 10)]


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,H,D,dims", SHAPES)
def test_rotary(T, H, D, dims, interleaved, dtype):
    r = rng("rotary", T, H, D, dims)
    t, x = rounded(r.normal(size=(T, H, D)), dtype)
    positions = r.integers(0, 1 << 20, size=T).astype(np.int32)
    positions[:4] = [0, 2**31 - 1, -1, 131071][:min(T, 4)]
    f = frequencies(dims)
    rotary = B.Rotary(f, interleaved, 1.25)
    x_gpu, at = t.cuda(), torch.from_numpy(positions).cuda()
    out = B.hlq_rotary(x_gpu, at, rotary)
    check_turned(host(out), x, positions, f, interleaved, 1.25, dtype)
    np.testing.assert_array_equal(host(x_gpu), x)
    # in place, a part of wider rows that begins anywhere, and head by head
    wide = torch.full((T, H * D + 3), 7.0, dtype=TYPES[dtype], device="cuda")
    part = wide.as_strided((T, H, D), (H * D + 3, D, 1), 1)
    part.copy_(x_gpu)
    B.hlq_rotary(part, at, rotary, out=part)
    assert torch.equal(part, out)
    assert (wide[:, 0] == 7).all() and (wide[:, 1 + H * D:] == 7).all()
    by_head = torch.empty((H, T, D), dtype=TYPES[dtype], device="cuda").transpose(0, 1)
    assert torch.equal(B.hlq_rotary(x_gpu, at, rotary, out=by_head), out)


def test_rotary_of_stretched_positions_and_other_frequencies():
    r = rng("stretched")
    for f in (B.rotary_frequencies(64, 500000.0, 8.0, 8192), B.rotary_frequencies(64, factor=4.0), [0.0, 1e-9, 3.0, 12345.678, -0.5]):
        t, x = rounded(r.normal(size=(50, 2, 64)), "f32")
        positions = r.integers(-(1 << 17), 1 << 17, size=50).astype(np.int32)
        out = B.hlq_rotary(t.cuda(), torch.from_numpy(positions).cuda(), B.Rotary(f))
        check_turned(host(out), x, positions, f, False, 1.0, "f32")


def test_rotary_of_infinities_and_nan():
    x = torch.ones((1, 1, 16), dtype=torch.bfloat16)
    x[0, 0, 3], x[0, 0, 5], x[0, 0, 15] = float("inf"), float("nan"), float("-inf")
    out = B.hlq_rotary(x.cuda(), torch.tensor([3], dtype=torch.int32, device="cuda"), B.Rotary(frequencies(8)))[0, 0].cpu()
    assert (~torch.isfinite(out)).nonzero().flatten().tolist() == [1, 3, 5, 7, 15]   # 5's partner is 1, 3's is 7
    assert torch.isnan(out[1]) and torch.isnan(out[5]) and out[15] == float("-inf")


CACHES = [("f16", 8), ("f16", 64), ("bf16", 128), ("bf16", 40), ("bf16", 256), ("mx8", 32), ("mx8", 96), ("mx8", 128), ("mx4", 64), ("mx4", 160), ("mx4", 128), ("mx4", 256)]


def rows(r, T, H, D):
    x = r.normal(size=(T, H, D)) * np.exp2(r.integers(-12, 12, size=(T, H, 1)))
    x[:, :, ::17] *= 20
    x.reshape(-1)[r.integers(0, x.size, size=3)] = 0
    return x


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("kind,D", CACHES)
def test_write_and_read(kind, D, dtype):
    H, page, pages = 3, 32, 5
    for T in (1, 9, 100):
        r = rng("write", kind, D, dtype, T)
        cache = Cache(pages, page, H, D, kind)
        k, v = (rounded(rows(r, T, H, D), dtype)[1] for _ in range(2))
        slots = r.permutation(pages * page)[:T]
        skipped = np.array(slots)
        skipped[T // 2] = -1 if T % 2 else pages * page     # a row of padding
        B.hlq_kv_write(cache.kv, *(torch.from_numpy(x).to(TYPES[dtype]).cuda() for x in (k, v)), torch.from_numpy(skipped).cuda())
        expected = np.full((2, pages * page, H, D), np.nan)
        for t, s in enumerate(skipped):
            if 0 <= s < pages * page:
                expected[0, s], expected[1, s] = stored(k[t], kind), stored(v[t], kind)
        every = torch.arange(pages * page, device="cuda")
        for out in ("f32", "f16", "bf16"):
            got = B.hlq_kv_read(cache.kv, every, dtype=TYPES[out])
            for g, want in zip(got, expected):
                np.testing.assert_array_equal(host(g), rounded(want, out)[1])
        # bytes beside the written ones are as they were
        if kind in ("f16", "bf16"):
            raw = cache.kv.rows.view(torch.int16).permute(1, 0, 3, 2, 4).reshape(2, pages * page, H, D)
            untouched = np.setdiff1d(np.arange(pages * page), skipped)
            assert (raw[:, torch.from_numpy(untouched).cuda()] == -1).all()


@pytest.mark.parametrize("kind", ["mx8", "mx4"])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_codes_of_every_grid_point_tie_and_neighbour(kind, dtype):
    grid = O.E4M3 if kind == "mx8" else np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    points = np.concatenate([grid, (grid[1:] + grid[:-1]) / 2])
    points = np.concatenate([points, points * (1 + 2.0**-8), points * (1 - 2.0**-8), [grid[-1] * 1.06, grid[-1] * 1.12]])
    points = np.concatenate([points, -points])
    points = np.concatenate([points, np.zeros(-len(points) % 31)]).reshape(-1, 31)
    x = np.concatenate([points, np.full((len(points), 1), grid[-1])], 1)        # the largest sets the scale
    scales = {"f16": (-14, -3, 0, 4), "bf16": (-126, -120, -9, 0, 60, 118), "f32": (-140, -126, -9, 0, 60, 118)}[dtype]
    x = np.concatenate([np.ldexp(x, s) for s in scales])[:, None, :]
    x = rounded(x, dtype)[1]
    cache = Cache((len(x) + 15) // 16, 16, 1, 32, kind)
    cache.put(np.arange(len(x)), x, -x[::-1].copy(), dtype)
    k, v = B.hlq_kv_read(cache.kv, torch.arange(len(x), device="cuda"))
    with np.errstate(over="ignore"):
        np.testing.assert_array_equal(host(k), cache.values[0, :len(x)])
        np.testing.assert_array_equal(host(v), cache.values[1, :len(x)])


@pytest.mark.parametrize("kind", ["mx8", "mx4", "bf16"])
def test_infinities_and_nan_are_kept_to_their_block(kind):
    x = np.ones((3, 2, 64))
    x[0, 0, 5], x[1, 1, 40], x[2, 0, 0] = np.inf, np.nan, -np.inf
    cache = Cache(1, 16, 2, 64, kind)
    cache.put([3, 0, 15], x, x + 1, "bf16")
    for g, want in zip(B.hlq_kv_read(cache.kv, torch.tensor([3, 0, 15], device="cuda")), cache.values):
        np.testing.assert_array_equal(host(g), want[[3, 0, 15]])


@pytest.mark.parametrize("kind", ["mx8", "mx4"])
def test_every_scale_byte_and_code_reads_as_its_value(kind):
    cache = B.alloc_kv_cache(16, 16, 1, 32, KINDS[kind])
    n, row = 256, 32 if kind == "mx8" else 16
    codes = np.array([c for c in range(256) if kind == "mx4" or c & 127 != 127], dtype=np.uint8)
    codes = codes[(np.arange(2 * n * row) * 7 % len(codes))].reshape(16, 2, 1, 16, row)
    scales = np.broadcast_to(np.arange(n, dtype=np.uint8).reshape(16, 1, 1, 1, 16), (16, 2, 1, 1, 16))
    cache.blob.copy_(torch.from_numpy(np.concatenate([codes.reshape(-1), scales.reshape(-1)])))
    got = B.hlq_kv_read(cache, torch.arange(n, device="cuda"))
    for i, g in enumerate(got):
        want = O.mx_values(codes[:, i].reshape(n, row), np.arange(n, dtype=np.uint8)[:, None], kind)
        with np.errstate(over="ignore"):
            np.testing.assert_array_equal(host(g).reshape(n, 32), want.astype(np.float32).astype(np.float64))


@pytest.mark.parametrize("kind,dtype,D,dims", [("bf16", "bf16", 128, 128), ("mx4", "bf16", 128, 64), ("mx8", "f16", 96, 96), ("f16", "f16", 40, 20), ("mx4", "f32", 64, 48), ("bf16", "f32", 256, 256)])
@pytest.mark.parametrize("T", [1, 37, 700])
def test_write_with_rotary_is_rotary_and_write(kind, dtype, D, dims, T):
    H, Hq, page, pages = 2, 6, 16, 50
    r = rng("fused", kind, D, T)
    qkv = rounded(r.normal(size=(T, (Hq + 2 * H) * D)), dtype)[0].cuda()
    q, k, v = qkv.view(T, -1, D).split([Hq, H, H], 1)
    rotary = B.Rotary(frequencies(dims), interleaved=T == 37, magnitude=0.75)
    positions = torch.from_numpy(r.integers(0, 1 << 18, size=T).astype(np.int32)).cuda()
    slots = torch.from_numpy(r.permutation(pages * page)[:T]).cuda()
    one, two = (Cache(pages, page, H, D, kind) for _ in range(2))
    q1, k1 = B.hlq_rotary(q, positions, rotary), B.hlq_rotary(k, positions, rotary)
    B.hlq_kv_write(one.kv, k1, v, slots)
    k2 = torch.empty_like(k1)
    q2 = B.hlq_kv_write(two.kv, k, v, slots, rotary=rotary, positions=positions, q=q, k_out=k2)
    assert torch.equal(q1, q2) and torch.equal(k1, k2) and torch.equal(one.kv.blob, two.kv.blob)
    # only the keys; then all in place
    three = Cache(pages, page, H, D, kind)
    assert B.hlq_kv_write(three.kv, k, v, slots, rotary=rotary, positions=positions) is None
    assert torch.equal(one.kv.blob, three.kv.blob)
    three.kv.blob.fill_(255)
    B.hlq_kv_write(three.kv, k, v, slots, rotary=rotary, positions=positions, q=q, q_out=q, k_out=k)
    assert torch.equal(q1, q) and torch.equal(k1, k) and torch.equal(one.kv.blob, three.kv.blob)


def test_read_leaves_rows_whose_slot_is_outside():
    cache = Cache(2, 16, 2, 64, "bf16")
    x = rng("outside").normal(size=(32, 2, 64))
    x = rounded(x, "bf16")[1]
    cache.put(np.arange(32), x, x + 1, "bf16")
    k, v = (torch.full((4, 2, 64), 5.0, device="cuda") for _ in range(2))
    B.hlq_kv_read(cache.kv, torch.tensor([31, -1, 32, 1 << 40], device="cuda"), k, v)
    assert (k[1:] == 5).all() and (v[1:] == 5).all()
    np.testing.assert_array_equal(host(k[0]), x[31])


def test_no_tokens():
    cache = Cache(2, 16, 2, 64, "mx4")
    empty = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    at = torch.empty(0, dtype=torch.int32, device="cuda")
    B.hlq_kv_write(cache.kv, empty, empty, none, rotary=B.Rotary(frequencies(64)), positions=at, q=empty)
    B.hlq_rotary(empty, at, B.Rotary(frequencies(64)))
    assert B.hlq_kv_read(cache.kv, none)[0].shape == (0, 2, 64)
    assert (cache.kv.blob == 255).all()


def test_slots_past_32_bits():
    # 2^32 values and more: pages at both ends of a cache of 9 GB
    pages, page, H, D = 18000, 128, 8, 128
    kv = B.alloc_kv_cache(pages, page, H, D, torch.bfloat16)
    assert kv.blob.numel() > 2 << 32
    x = rounded(rng("far").normal(size=(4, H, D)), "bf16")[0].cuda()
    slots = torch.tensor([0, pages * page - 1, 8191 * page + 3, 8192 * page], device="cuda")
    B.hlq_kv_write(kv, x, -x, slots)
    k, v = B.hlq_kv_read(kv, slots, dtype=torch.bfloat16)
    assert torch.equal(k, x) and torch.equal(v, -x)
    assert torch.equal(kv.rows[8192, 0, :, 0], x[3])
