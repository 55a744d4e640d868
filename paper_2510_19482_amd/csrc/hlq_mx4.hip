// MX4 matrices: quantization of rows, the values back, and the exchange form (codes and scale bytes row by row) in and out.
//
//   block b of 32 k:  e = max(floor(log2(max |x|)) - 2, -127);  value = e2m1 nearest to x 2^-e (ties to the even code, at most 6)
//
// Quantizing reads a value once and writes 4.25 bits: it is bound by memory.  A wavefront takes a panel of four rows: a lane has
// eight successive values (one 16-byte load of 16-bit types, two of fp32), four lanes a block, whose largest magnitudes meet by
// two quad permutations; codes leave as a dword a lane, 256 contiguous bytes.  The values are read, and in dequantizing written, past
// the caches: 8192 x 8192 f16 37 us (170 MB, 4.6 TB/s; through them 38), back 35 (through them 42); one after the other, both in 60.
#include "hlq_mx4.h"

namespace {

constexpr int MX4_WAVES = 4;

template <int T>
__global__ void __launch_bounds__(64 * MX4_WAVES)
hlq_mx4_quantize_kernel(const typename Mx4Type<T>::type *__restrict__ x, int64_t ldx, int64_t rows, int K, int panels,
                        uint8_t *__restrict__ codes, uint8_t *__restrict__ scales, int64_t items)
{
    const int lane = (int)(threadIdx.x & 63u), j = lane & 15;
    for (int64_t it = (int64_t)blockIdx.x * MX4_WAVES + (threadIdx.x >> 6); it < items; it += (int64_t)gridDim.x * MX4_WAVES) {
        const int64_t quad = it / panels, row = quad * 4 + (lane >> 4);
        const int panel = (int)(it - quad * panels), k = panel * MX4_PANEL_K + j * 8;
        if (row >= rows) continue;
        typename Mx4Type<T>::type v[8];
        mx4_load8<true>(x + row * ldx + k, K - k, v);
        const uint32_t byte = mx4_scale_of(mx4_quad_max(mx4_top_bits(v)));
        const int64_t at = panel * rows + row;
        *(uint32_t *)(codes + at * 64 + j * 4) = mx4_codes(v, byte);
        if ((lane & 3) == 0) scales[at * 4 + mx4_scale_byte(j >> 2)] = (uint8_t)byte;
    }
}

// Upper bytes of the f16 that four codes (the low halves of c's bytes) stand for; the lower bytes are 0.
__device__ __forceinline__ uint32_t code_bytes(uint32_t c)
{
    // 0 0.5 1 1.5 2 3 4 6
    return __builtin_amdgcn_perm(0x46444240u, 0x3e3c3800u, c & 0x07070707u) | (c & 0x08080808u) << 4;
}

// As in quantizing: a wavefront takes a panel of four rows, a lane eight successive values.
template <int T>
__global__ void __launch_bounds__(64 * MX4_WAVES)
hlq_mx4_dequantize_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales, int64_t rows, int K, int panels,
                          typename Mx4Type<T>::type *__restrict__ y, int64_t ldy, int64_t items)
{
    using V = typename Mx4Type<T>::type;
    const int lane = (int)(threadIdx.x & 63u), j = lane & 15;
    for (int64_t it = (int64_t)blockIdx.x * MX4_WAVES + (threadIdx.x >> 6); it < items; it += (int64_t)gridDim.x * MX4_WAVES) {
        const int64_t quad = it / panels, row = quad * 4 + (lane >> 4);
        const int panel = (int)(it - quad * panels), k = panel * MX4_PANEL_K + j * 8;
        if (row >= rows || k >= K) continue;
        const int64_t at = panel * rows + row;
        const uint32_t c = *(const uint32_t *)(codes + at * 64 + j * 4);
        const int byte = scales[at * 4 + mx4_scale_byte(j >> 2)];
        const uint32_t even = code_bytes(c), odd = code_bytes(c >> 4);
        typename Mx4Eight<V>::Values out;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint16_t half = (uint16_t)((i & 1 ? odd : even) >> (8 * (i >> 1)) << 8);
            const float v = ldexpf((float)__builtin_bit_cast(_Float16, half), byte - 127);
            out.v[i] = (V)(byte == 255 ? __builtin_nanf("") : v);
        }
        V *p = y + row * ldy + k;
        if (k + 8 <= K) mx4_stream8(out, p);
        else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k + i < K) p[i] = out.v[i];
        }
    }
}

// exchange form: codes [rows][(K + 1) / 2], scales [rows][(K + 31) / 32]; a thread makes eight codes, every fourth one scale byte too.
// Once for weights that are loaded: 8192 x 8192 52 us (71 MB; bound by its byte loads), back 38
__global__ void __launch_bounds__(256)
hlq_mx4_pack_kernel(const uint8_t *__restrict__ in, int64_t ldc, const uint8_t *__restrict__ in_scales, int64_t lds, int64_t rows, int K, int panels,
                    uint8_t *__restrict__ codes, uint8_t *__restrict__ scales, int64_t items)
{
    const int eights = panels * 16, bytes = (K + 1) / 2, blocks = (K + 31) / 32;
    for (int64_t it = (int64_t)blockIdx.x * 256 + threadIdx.x; it < items; it += (int64_t)gridDim.x * 256) {
        const int64_t row = it / eights;
        const int j = (int)(it - row * eights);
        uint32_t c = 0;
        for (int i = 0; i < 4; ++i) {
            const int at = 4 * j + i;
            uint32_t b = at < bytes ? in[row * ldc + at] : 0u;
            if (2 * at + 1 >= K) b &= 15u;
            c |= b << (8 * i);
        }
        *(uint32_t *)(codes + ((int64_t)(j >> 4) * rows + row) * 64 + (j & 15) * 4) = c;
        if ((j & 3) == 0)
            scales[((int64_t)(j >> 4) * rows + row) * 4 + mx4_scale_byte((j >> 2) & 3)] = (j >> 2) < blocks ? in_scales[row * lds + (j >> 2)] : (uint8_t)0;
    }
}

__global__ void __launch_bounds__(256)
hlq_mx4_unpack_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales, int64_t rows, int K, int panels,
                      uint8_t *__restrict__ out, uint8_t *__restrict__ out_scales, int64_t items)
{
    const int eights = panels * 16, bytes = (K + 1) / 2, blocks = (K + 31) / 32;
    for (int64_t it = (int64_t)blockIdx.x * 256 + threadIdx.x; it < items; it += (int64_t)gridDim.x * 256) {
        const int64_t row = it / eights;
        const int j = (int)(it - row * eights);
        if (out) {
            const uint32_t c = *(const uint32_t *)(codes + ((int64_t)(j >> 4) * rows + row) * 64 + (j & 15) * 4);
            for (int i = 0; i < 4 && 4 * j + i < bytes; ++i) out[row * bytes + 4 * j + i] = (uint8_t)(c >> (8 * i));
        }
        if (out_scales && (j & 3) == 0 && (j >> 2) < blocks)
            out_scales[row * blocks + (j >> 2)] = scales[((int64_t)(j >> 4) * rows + row) * 4 + mx4_scale_byte((j >> 2) & 3)];
    }
}

unsigned grid_of(int64_t items, int64_t a_block)
{
    const int64_t g = (items + a_block - 1) / a_block;
    return (unsigned)(g < 65536 ? g : 65536);
}

template <int T>
void launch_quantize(const Mx4Dims &d, const void *x, int64_t ldx, void *blob, hipStream_t st)
{
    using V = typename Mx4Type<T>::type;
    const int64_t items = (d.rows + 3) / 4 * d.panels;
    uint8_t *codes = (uint8_t *)blob, *scales = codes + d.code_bytes;
    const dim3 grid(grid_of(items, MX4_WAVES)), block(64 * MX4_WAVES);
    hlq_mx4_quantize_kernel<T><<<grid, block, 0, st>>>((const V *)x, ldx, d.rows, d.K, d.panels, codes, scales, items);
}

template <int T>
void launch_dequantize(const Mx4Dims &d, const void *blob, void *y, int64_t ldy, hipStream_t st)
{
    using V = typename Mx4Type<T>::type;
    const int64_t items = (d.rows + 3) / 4 * d.panels;
    const uint8_t *codes = (const uint8_t *)blob, *scales = codes + d.code_bytes;
    const dim3 grid(grid_of(items, MX4_WAVES)), block(64 * MX4_WAVES);
    hlq_mx4_dequantize_kernel<T><<<grid, block, 0, st>>>(codes, scales, d.rows, d.K, d.panels, (V *)y, ldy, items);
}

// what the four calls have in common
hlq_status check_matrix(int64_t rows, int32_t K, Mx4Dims *d, const void *blob, size_t blob_bytes)
{
    const hlq_status s = hlq_mx4_check(rows, K, d);
    if (s != HLQ_OK) return s;
    if (rows == 0) return HLQ_OK;
    if (!blob) return HLQ_ERR_NULL;
    if ((uintptr_t)blob & 15u) return HLQ_ERR_BAD_STRIDE;
    return blob_bytes < d->total ? HLQ_ERR_BUFFER_TOO_SMALL : HLQ_OK;
}

}  // namespace

hlq_status hlq_mx4_check(int64_t rows, int32_t K, Mx4Dims *out)
{
    if (rows < 0 || K < 1) return HLQ_ERR_BAD_DESC;
    if (K > HLQ_MAX_K || rows > MX4_MAX_ROWS) return HLQ_ERR_UNSUPPORTED;
    Mx4Dims d;
    d.rows = rows;
    d.K = K;
    d.panels = (K + MX4_PANEL_K - 1) / MX4_PANEL_K;
    d.code_bytes = (size_t)rows * (size_t)d.panels * 64u;
    d.total = d.code_bytes + (size_t)rows * (size_t)d.panels * 4u;
    *out = d;
    return HLQ_OK;
}

hlq_status hlq_mx4_launch_quantize(const Mx4Dims &d, const void *x, hlq_dtype t, int64_t ldx, void *blob, hipStream_t st)
{
    if (t == HLQ_F16) launch_quantize<HLQ_F16>(d, x, ldx, blob, st);
    else if (t == HLQ_BF16) launch_quantize<HLQ_BF16>(d, x, ldx, blob, st);
    else launch_quantize<HLQ_F32>(d, x, ldx, blob, st);
    return hlq_hip_status(hipGetLastError());
}

extern "C" {

hlq_status hlq_mx4_bytes(int64_t rows, int32_t K, size_t *bytes)
{
    Mx4Dims d;
    const hlq_status s = hlq_mx4_check(rows, K, &d);
    if (s != HLQ_OK) return s;
    if (!bytes) return HLQ_ERR_NULL;
    *bytes = d.total;
    return HLQ_OK;
}

hlq_status hlq_mx4_quantize(int64_t rows, int32_t K, const void *x, hlq_dtype type, int64_t ldx, void *blob, size_t blob_bytes, void *stream)
{
    Mx4Dims d;
    const hlq_status s = check_matrix(rows, K, &d, blob, blob_bytes);
    if (s != HLQ_OK) return s;
    if (!hlq_is_float(type)) return HLQ_ERR_UNSUPPORTED;
    if (rows > 1 && ldx < K) return HLQ_ERR_BAD_STRIDE;
    if (rows == 0) return HLQ_OK;
    if (!x) return HLQ_ERR_NULL;
    if ((uintptr_t)x % (unsigned)hlq_dtype_bytes(type)) return HLQ_ERR_BAD_STRIDE;
    hlq_clear_stale_error();
    return hlq_mx4_launch_quantize(d, x, type, ldx, blob, (hipStream_t)stream);
}

hlq_status hlq_mx4_dequantize(int64_t rows, int32_t K, const void *blob, void *y, hlq_dtype type, int64_t ldy, void *stream)
{
    Mx4Dims d;
    const hlq_status s = check_matrix(rows, K, &d, blob, SIZE_MAX);
    if (s != HLQ_OK) return s;
    if (!hlq_is_float(type)) return HLQ_ERR_UNSUPPORTED;
    if (rows > 1 && ldy < K) return HLQ_ERR_BAD_STRIDE;
    if (rows == 0) return HLQ_OK;
    if (!y) return HLQ_ERR_NULL;
    if ((uintptr_t)y % (unsigned)hlq_dtype_bytes(type)) return HLQ_ERR_BAD_STRIDE;
    hlq_clear_stale_error();
    if (type == HLQ_F16) launch_dequantize<HLQ_F16>(d, blob, y, ldy, (hipStream_t)stream);
    else if (type == HLQ_BF16) launch_dequantize<HLQ_BF16>(d, blob, y, ldy, (hipStream_t)stream);
    else launch_dequantize<HLQ_F32>(d, blob, y, ldy, (hipStream_t)stream);
    return hlq_hip_status(hipGetLastError());
}

hlq_status hlq_mx4_pack(int64_t rows, int32_t K, const uint8_t *codes, int64_t ldc, const uint8_t *scales, int64_t lds, void *blob, size_t blob_bytes, void *stream)
{
    Mx4Dims d;
    const hlq_status s = check_matrix(rows, K, &d, blob, blob_bytes);
    if (s != HLQ_OK || rows == 0) return s;
    if (!codes || !scales) return HLQ_ERR_NULL;
    if (rows > 1 && (ldc < (K + 1) / 2 || lds < (K + 31) / 32)) return HLQ_ERR_BAD_STRIDE;
    hlq_clear_stale_error();
    const int64_t items = rows * d.panels * 16;
    hlq_mx4_pack_kernel<<<grid_of(items, 256), 256, 0, (hipStream_t)stream>>>(codes, ldc, scales, lds, rows, K, d.panels, (uint8_t *)blob, (uint8_t *)blob + d.code_bytes, items);
    return hlq_hip_status(hipGetLastError());
}

hlq_status hlq_mx4_unpack(int64_t rows, int32_t K, const void *blob, uint8_t *codes, uint8_t *scales, void *stream)
{
    Mx4Dims d;
    const hlq_status s = check_matrix(rows, K, &d, blob, SIZE_MAX);
    if (s != HLQ_OK || rows == 0) return s;
    if (!codes && !scales) return HLQ_OK;
    hlq_clear_stale_error();
    const int64_t items = rows * d.panels * 16;
    hlq_mx4_unpack_kernel<<<grid_of(items, 256), 256, 0, (hipStream_t)stream>>>((const uint8_t *)blob, (const uint8_t *)blob + d.code_bytes, rows, K, d.panels, codes, scales, items);
    return hlq_hip_status(hipGetLastError());
}

}  // extern "C"
