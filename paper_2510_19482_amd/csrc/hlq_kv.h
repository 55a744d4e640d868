// The paged cache of keys and values as the kernels see it; its layout stands in hlq.h.
#pragma once

#include "hlq_mx4.h"

constexpr int KV_MOST_DIM = 256, KV_MOST_HEADS = 1024, KV_BLOCK = 32;

struct KvDims {
    int64_t pages;
    int H, D, type;
    int log_page;            // of the tokens of a page
    int row_bytes, blocks;   // of a token and head: bytes of codes, scale bytes (0: 16-bit values)
    size_t code_bytes, total;
};
hlq_status hlq_kv_check(const hlq_kv_desc *c, KvDims *out);

struct KvView {
    uint8_t *codes, *scales;
    int64_t pages;
    int H, log_page, row_bytes, blocks;

    // where the page's keys (what = 0) or values (1) of a head are
    __device__ __forceinline__ int64_t piece(int64_t page, int what, int h) const { return (page * 2 + what) * H + h; }
    __device__ __forceinline__ uint8_t *rows(int64_t page, int what, int h) const { return codes + (piece(page, what, h) << log_page) * row_bytes; }
    __device__ __forceinline__ uint8_t *bytes(int64_t page, int what, int h) const { return scales + (piece(page, what, h) << log_page) * blocks; }
};
static inline KvView hlq_kv_view(const KvDims &d, const void *cache)
{
    uint8_t *p = (uint8_t *)const_cast<void *>(cache);
    return KvView{p, p + d.code_bytes, d.pages, d.H, d.log_page, d.row_bytes, d.blocks};
}

// rows of heads: strides in elements
struct KvRows {
    void *p;
    int64_t ts, hs;
};
// What an array [T, heads, dim] may be.  An output's rows have to stand apart: token by token or head by head.
static inline hlq_status hlq_check_rows(const void *p, int64_t T, int heads, int dim, int64_t ts, int64_t hs, hlq_dtype type, bool output)
{
    constexpr int64_t MOST = (int64_t)1 << 40;
    if (ts < 0 || hs < 0 || ts > MOST || hs > MOST) return HLQ_ERR_BAD_STRIDE;
    if (output && (T > 1 || heads > 1)) {
        const bool by_token = (heads == 1 || hs >= dim) && (T == 1 || ts >= (heads - 1) * hs + dim);
        const bool by_head = (T == 1 || ts >= dim) && (heads == 1 || hs >= (T - 1) * (__int128)ts + dim);
        if (!by_token && !by_head) return HLQ_ERR_BAD_STRIDE;
    }
    if (!p) return HLQ_ERR_NULL;
    return (uintptr_t)p % (unsigned)hlq_dtype_bytes(type) ? HLQ_ERR_BAD_STRIDE : HLQ_OK;
}

// An array [T, heads, dim] whose elements have `bytes`.
struct KvSpan {
    KvRows x;
    int64_t T;
    int heads, bytes;
};
static inline KvSpan hlq_span(const void *p, int64_t T, int heads, int64_t ts, int64_t hs, hlq_dtype type)
{
    return KvSpan{KvRows{const_cast<void *>(p), ts, hs}, T, heads, hlq_dtype_bytes(type)};
}
// Whether two of them share memory.  Exact where strides from token to token are the same, so that parts of one projection's rows stand apart; else a head's rows are taken as one
// piece if strides from head to head are the same, or all of an array.
static inline bool hlq_rows_overlap(const KvSpan &a, const KvSpan &b, int dim)
{
    if (a.T < 1 || b.T < 1 || !a.x.p || !b.x.p) return false;
    const int64_t far = (int64_t)((uintptr_t)b.x.p - (uintptr_t)a.x.p);
    const int64_t ats = a.x.ts * a.bytes, bts = b.x.ts * b.bytes, ahs = a.x.hs * a.bytes, bhs = b.x.hs * b.bytes, arow = (int64_t)dim * a.bytes, brow = (int64_t)dim * b.bytes;
    // [at, at + n), moved by some of low .. high periods, and [bt, bt + m)
    const auto meet = [](int64_t at, int64_t n, int64_t bt, int64_t m, int64_t period, int64_t low, int64_t high) {
        int64_t k = 0;
        if (period > 0) {
            const int64_t room = bt + m - 1 - at;   // the furthest that it begins before [bt, bt + m) ends
            k = room / period - (room % period < 0);
            k = k > high ? high : k;
            if (k < low) return false;
        }
        return at + k * period < bt + m && bt < at + k * period + n;
    };
    typedef __int128 Wide;
    const Wide aend = (Wide)(a.T - 1) * ats + (a.heads - 1) * ahs + arow, bend = (Wide)(b.T - 1) * bts + (b.heads - 1) * bhs + brow;
    if (far >= aend || -(Wide)far >= bend) return false;
    const int64_t period = a.T > 1 ? ats : bts;
    if (a.T == 1 || b.T == 1 || ats == bts) {
        const auto rows = [&](int64_t at, int64_t n, int64_t bt, int64_t m) { return meet(at, n, bt, m, period, 1 - b.T, a.T - 1); };
        if (!rows(0, (a.heads - 1) * ahs + arow, far, (b.heads - 1) * bhs + brow)) return false;
        for (int i = 0; i < a.heads; ++i)
            for (int j = 0; j < b.heads; ++j)
                if (rows(i * ahs, arow, far + j * bhs, brow)) return true;
        return false;
    }
    return ahs != bhs || meet(0, (a.T - 1) * ats + arow, far, (b.T - 1) * bts + brow, ahs, 1 - b.heads, a.heads - 1);
}
// An output may be where the input is that it is made of, row for row, or where nothing of it is.
static inline bool hlq_rows_in_the_way(const KvSpan &in, const KvSpan &out, int dim)
{
    const bool same = in.x.p == out.x.p && in.T == out.T && in.heads == out.heads && in.bytes == out.bytes && (in.T == 1 || in.x.ts == out.x.ts) && (in.heads == 1 || in.x.hs == out.x.hs);
    return !same && hlq_rows_overlap(in, out, dim);
}

// By value: a bit cast of a vector's element reads the vector's first.
__device__ __forceinline__ float as_float(uint32_t v) { return __builtin_bit_cast(float, v); }
__device__ __forceinline__ uint32_t as_bits(float v) { return __builtin_bit_cast(uint32_t, v); }

// Softmax of both attention kernels.  What sums are multiplied by: not 0, so that an infinite sum stays one; what 2^-126 leaves of a finite one is far below a rounding
__device__ __forceinline__ float exp2_above_0(float v) { return fmaxf(__builtin_amdgcn_exp2f(v), 0x1p-126f); }
// A base is the largest product with the scale, rounded.  From 2^22 on that rounding is felt, later it is more than an exponential holds: there the other products are rounded
// likewise before the base is taken away, so that the largest has its weight.  (At most 2^15.9, which f16 holds: the allowance of 2^8 is itself rounded there.)
constexpr float LARGE = 0x1p22f;
__device__ __forceinline__ float above_base(float x, float scale, float base)
{
#pragma clang fp contract(off)
    const float product = x * scale, far = product - base, v = fabsf(base) < LARGE ? __builtin_fmaf(x, scale, -base) : far;
    return v > 15.9f ? 15.9f : v;   // (a NaN stays)
}

// storage type of a cache's values
template <int T> struct KvType { using type = uint8_t; };
template <> struct KvType<HLQ_F16> { using type = _Float16; };
template <> struct KvType<HLQ_BF16> { using type = __bf16; };
