// Microscaled 4-bit matrices (MX4): values of a row in blocks of 32 along k, a value = e2m1 code x 2^(scale byte - 127).
//
// Layout of a matrix [rows, K] in one blob, panels of 128 k:
//
//   codes   [panels][rows][64]   two codes a byte, the even k in the low half; zero past K
//   scales  [panels][rows][4]    byte (b % 2) * 2 + b / 2 is that of block b of the panel's four; zero past K
//
// so that what a tile of rows needs of a panel is one contiguous piece of memory.  The matrix cores take 32 successive k of a
// row from one lane, which also gives the block's scale byte, chosen from a register by the instruction:
//   32x32x64   lane l: row l % 32, block 2 s + l / 32 of step s = 0, 1: its scale bytes are the 16 bits l / 32 of the row's four
//   16x16x128  lane l: row l % 16, block l / 16
// Scale byte 255 is NaN and makes the results NaN that its block enters; products and the sum over a block are exact, the
// accumulation is fp32.
#pragma once

#include "hlq_internal.h"

typedef int mx4_int4 __attribute__((ext_vector_type(4)));
typedef int mx4_int8 __attribute__((ext_vector_type(8)));
typedef float mx4_float4 __attribute__((ext_vector_type(4)));
typedef float mx4_float8 __attribute__((ext_vector_type(8)));
typedef float mx4_float16 __attribute__((ext_vector_type(16)));
typedef _Float16 mx4_half2 __attribute__((ext_vector_type(2)));
typedef _Float16 mx4_half8 __attribute__((ext_vector_type(8)));
typedef __bf16 mx4_bf2 __attribute__((ext_vector_type(2)));
typedef __bf16 mx4_bf8 __attribute__((ext_vector_type(8)));

#define MX4_PANEL_K 128
#define MX4_MAX_ROWS ((int64_t)1 << 31)
#define MX4_FP4 4   // the instruction's number of the e2m1 format

struct Mx4Dims {
    int64_t rows;
    int K, panels;
    size_t code_bytes, total;
};

// what the kernels see of a matrix
struct Mx4View {
    const uint8_t *codes, *scales;
    int64_t rows;           // a row's place in panel p is p * rows + row
};

hlq_status hlq_mx4_check(int64_t rows, int32_t K, Mx4Dims *out);
static inline Mx4View hlq_mx4_view(const Mx4Dims &d, const void *blob)
{
    return Mx4View{(const uint8_t *)blob, (const uint8_t *)blob + d.code_bytes, d.rows};
}
hlq_status hlq_mx4_launch_quantize(const Mx4Dims &d, const void *x, hlq_dtype t, int64_t ldx, void *blob, hipStream_t st);

// place of the scale byte of block b (0..3) of a panel
__host__ __device__ __forceinline__ int mx4_scale_byte(int b) { return (b & 1) * 2 + (b >> 1); }

static inline int hlq_dtype_bytes(hlq_dtype t) { return t == HLQ_F32 ? 4 : 2; }
static inline bool hlq_is_float(int t) { return t == HLQ_F16 || t == HLQ_F32 || t == HLQ_BF16; }

// storage type of a dtype
template <int T> struct Mx4Type;
template <> struct Mx4Type<HLQ_F16> { using type = _Float16; };
template <> struct Mx4Type<HLQ_BF16> { using type = __bf16; };
template <> struct Mx4Type<HLQ_F32> { using type = float; };

// Eight successive values of a row, quantized: what one lane holds of a block of 32 that four lanes share.
// `top` is the largest magnitude as a float's bits (infinities and NaN: exponent 255).
__device__ __forceinline__ uint32_t mx4_top_bits(const _Float16 (&v)[8])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t b = __builtin_bit_cast(uint16_t, v[i]) & 0x7fffu;
        m = b > m ? b : m;
    }
    return m >= 0x7c00u ? 0x7f800000u : __builtin_bit_cast(uint32_t, (float)__builtin_bit_cast(_Float16, (uint16_t)m));
}
__device__ __forceinline__ uint32_t mx4_top_bits(const __bf16 (&v)[8])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t b = __builtin_bit_cast(uint16_t, v[i]) & 0x7fffu;
        m = b > m ? b : m;
    }
    return m << 16;
}
__device__ __forceinline__ uint32_t mx4_top_bits(const float (&v)[8])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t b = __builtin_bit_cast(uint32_t, v[i]) & 0x7fffffffu;
        m = b > m ? b : m;
    }
    return m;
}
// Scale byte of a block whose largest magnitude has these bits: floor(log2) - 2 and the bias, at least 0.  Zero and
// subnormal floats have exponent field 0; a block that holds an infinity or a NaN gets 255.
__device__ __forceinline__ uint32_t mx4_scale_of(uint32_t top)
{
    const uint32_t e = top >> 23;
    return e == 255u ? 255u : e > 2u ? e - 2u : 0u;
}
// the largest of four neighbouring lanes
__device__ __forceinline__ uint32_t mx4_quad_max(uint32_t v)
{
    uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xf, 0xf, true);   // lanes 1 0 3 2
    v = o > v ? o : v;
    o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xf, 0xf, true);            // lanes 2 3 0 1
    return o > v ? o : v;
}
// Codes of eight values under a scale byte, the first in the lowest four bits: to nearest, ties to the even code, above 5 it
// is 6.  The conversion takes the scale's exponent field, so 2^-127 (byte 0) is given as +0.  (All finite f16 and bf16 values
// and f32 grids and ties against a 64-bit reference at scale bytes 0..252: no difference.)
__device__ __forceinline__ uint32_t mx4_codes(const _Float16 (&v)[8], uint32_t byte)
{
    const float s = __builtin_bit_cast(float, byte << 23);
    uint32_t r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(0u, (mx4_half2){v[0], v[1]}, s, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, (mx4_half2){v[2], v[3]}, s, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, (mx4_half2){v[4], v[5]}, s, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, (mx4_half2){v[6], v[7]}, s, 3);
}
__device__ __forceinline__ uint32_t mx4_codes(const __bf16 (&v)[8], uint32_t byte)
{
    const float s = __builtin_bit_cast(float, byte << 23);
    uint32_t r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, (mx4_bf2){v[0], v[1]}, s, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, (mx4_bf2){v[2], v[3]}, s, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, (mx4_bf2){v[4], v[5]}, s, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, (mx4_bf2){v[6], v[7]}, s, 3);
}
__device__ __forceinline__ uint32_t mx4_codes(const float (&v)[8], uint32_t byte)
{
    const float s = __builtin_bit_cast(float, byte << 23);
    uint32_t r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0], v[1], s, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2], v[3], s, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4], v[5], s, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6], v[7], s, 3);
}

// Rows begin at any element, so 16 bytes are read and written at the alignment of one (this target takes global accesses of any
// alignment).
typedef uint32_t mx4_u2 __attribute__((ext_vector_type(2)));
typedef uint32_t mx4_u4 __attribute__((ext_vector_type(4)));
typedef mx4_u2 mx4_u2_any __attribute__((aligned(2)));
typedef mx4_u4 mx4_u4_any __attribute__((aligned(2)));
template <class T> struct Mx4Eight {
    static constexpr int N = sizeof(T) / 2;              // of 16 bytes
    struct alignas(16) Raw { mx4_u4 r[N]; };
    struct alignas(16) Values { T v[8]; };
};
// eight values at p; STREAM: not to be kept in the caches
template <bool STREAM, class T>
__device__ __forceinline__ void mx4_read8(const T *p, T (&v)[8])
{
    using E = Mx4Eight<T>;
    typename E::Raw raw;
#pragma unroll
    for (int i = 0; i < E::N; ++i) {
        const mx4_u4_any *q = (const mx4_u4_any *)(p + i * 8 / E::N);
        if constexpr (STREAM) raw.r[i] = __builtin_nontemporal_load(q);
        else raw.r[i] = *q;
    }
    const typename E::Values e = __builtin_bit_cast(typename E::Values, raw);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = e.v[i];
}
template <class T>
__device__ __forceinline__ void mx4_stream8(const typename Mx4Eight<T>::Values &e, T *p)
{
    using E = Mx4Eight<T>;
    const typename E::Raw raw = __builtin_bit_cast(typename E::Raw, e);
#pragma unroll
    for (int i = 0; i < E::N; ++i) __builtin_nontemporal_store(raw.r[i], (mx4_u4_any *)(p + i * 8 / E::N));
}
// Eight values at p of a row that ends `left` values on (left <= 0: none); past the end zeros.
template <bool STREAM, class T>
__device__ __forceinline__ void mx4_load8(const T *p, int left, T (&v)[8])
{
    if (left >= 8) mx4_read8<STREAM>(p, v);
    else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : (T)0.0f;
    }
}

// silu(g) u = g / (1 + e^-g) u.  EXACT, for fp32 results: each step within one or two units of fp32's last place.  Else, for results of 16 bits, the
// exponential's argument is rounded once, which is about |g| 2^-24 of it, 2^-17 where it is most: far below what the result is rounded by
// (2^-11, 2^-8), and six instructions less in an epilogue in which nothing else multiplies.  All is taken by 2^-8: so 1 + e^-g is a number, and
// its reciprocal a normal one, until silu(g) itself is below the smallest normal number; from there on it is 0.
template <bool EXACT>
__device__ __forceinline__ float mx4_gate(float g, float u)
{
    constexpr float LOG2E = 1.44269504f, LOG2E_REST = 1.92596299e-8f, LN2 = 0.693147181f;
    float e;   // 2^-8 e^-g
    if constexpr (EXACT) {
#pragma clang fp contract(off)
        const float c = __builtin_amdgcn_fmed3f(g, -100.f, 100.f), t = c * -LOG2E - 8.f;   // rounded twice: so t + 8 is exact
        const float rest = fmaf(c, -LOG2E_REST, fmaf(c, -LOG2E, -(t + 8.f)));   // what t lacks: 2^rest is 1 + rest ln 2
        e = __builtin_amdgcn_exp2f(t) * fmaf(rest, LN2, 1.f);
    } else
        e = __builtin_amdgcn_exp2f(fmaf(g, -LOG2E, -8.f));
    return g * 0x1p-8f * __builtin_amdgcn_rcpf(e + 0x1p-8f) * u;
}

__device__ __forceinline__ uint32_t mx4_bits16(float v, int type)
{
    return type == HLQ_F16 ? __builtin_bit_cast(uint16_t, (_Float16)v) : __builtin_bit_cast(uint16_t, (__bf16)v);
}
// four successive results of a row that has `left` more, rounded to nearest even
__device__ __forceinline__ void mx4_store4(void *y, int type, int64_t at, const float *v, int left)
{
    if (type == HLQ_F32) {
        typedef mx4_float4 any __attribute__((aligned(4)));
        float *p = (float *)y + at;
        if (left >= 4) *(any *)p = (mx4_float4){v[0], v[1], v[2], v[3]};
        else
            for (int i = 0; i < left; ++i) p[i] = v[i];
    } else {
        uint32_t b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = mx4_bits16(v[i], type);
        uint16_t *p = (uint16_t *)y + at;
        if (left >= 4) *(mx4_u2_any *)p = (mx4_u2){b[0] | b[1] << 16, b[2] | b[3] << 16};
        else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < left) p[i] = (uint16_t)b[i];
        }
    }
}
// eight of them, not to be kept in the caches
__device__ __forceinline__ void mx4_store8(void *y, int type, int64_t at, const float *v, int left)
{
    if (left < 8) {
        mx4_store4(y, type, at, v, left);
        if (left > 4) mx4_store4(y, type, at + 4, v + 4, left - 4);
    } else if (type == HLQ_F32) {
        Mx4Eight<float>::Values e;
#pragma unroll
        for (int i = 0; i < 8; ++i) e.v[i] = v[i];
        mx4_stream8(e, (float *)y + at);
    } else {
        Mx4Eight<uint16_t>::Values e;
#pragma unroll
        for (int i = 0; i < 8; ++i) e.v[i] = (uint16_t)mx4_bits16(v[i], type);
        mx4_stream8(e, (uint16_t *)y + at);
    }
}
