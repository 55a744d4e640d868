// Products of MX4 matrices for few rows (an expert's few rows, a decoded batch): up to 16 rows a workgroup.
//
//   y[r, n] = sum over blocks b of 2^(a_rb + w_nb - 254) sum_{k in b} A[r, k] W[n, k]        (gated: silu(y[r, n]) y[r, N / 2 + n])
//
// Bound by the weights' bytes.  A wavefront holds 16 rows of W (results' columns) and a share of the panels; the wavefronts of a
// workgroup share the columns and add their sums through LDS, in order.  Weights go straight to registers in the form that the
// matrix core takes.  Activations that come as f16, bf16 or f32 are quantized by the lane that feeds them to the matrix core:
// it holds whole blocks of 32 of a row, so no lane needs another's.
#include "hlq_mx4_gemm.h"

namespace {

struct Operand {   // one lane's share of a panel: block l / 16 of row l % 16
    mx4_int4 code;
    int scale;      // byte 0

    __device__ __forceinline__ void none()
    {
        code = (mx4_int4){0, 0, 0, 0};
        scale = 127;
    }
    __device__ __forceinline__ void load(const Mx4View &m, int64_t at, int g)
    {
        code = *(const mx4_int4 *)(m.codes + at * 64 + g * 16);
        scale = m.scales[at * 4 + mx4_scale_byte(g)];
    }
    template <class T>
    __device__ __forceinline__ void quantize(const T *p, int left, bool aligned)
    {
        T v[4][8];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (aligned) mx4_load8<true>(p + 8 * i, left - 8 * i, v[i]);
            else mx4_load8<false>(p + 8 * i, left - 8 * i, v[i]);
            const uint32_t t = mx4_top_bits(v[i]);
            top = t > top ? t : top;
        }
        scale = (int)mx4_scale_of(top);
#pragma unroll
        for (int i = 0; i < 4; ++i) code[i] = (int)mx4_codes(v[i], (uint32_t)scale);
    }
};

__device__ __forceinline__ mx4_int8 wide(mx4_int4 v) { return (mx4_int8){v.x, v.y, v.z, v.w, 0, 0, 0, 0}; }

template <int XT, bool GATED>
__global__ void __launch_bounds__(1024)
hlq_mx4_few_kernel(const Mx4Product a, int groups, int64_t items)
{
    constexpr int NT = GATED ? 2 : 1;
    extern __shared__ float sums[];   // [wave][NT][4][64]
    const int lane = (int)(threadIdx.x & 63u), wave = (int)(threadIdx.x >> 6), waves = (int)(blockDim.x >> 6);
    const int r = lane & 15, g = lane >> 4;
    for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
        const Mx4RowTile tile = mx4_row_tile<16>(a, (int)(it / groups));
        if (tile.n == 0) break;   // the later ones are no less past the end
        const int n0 = (int)(it % groups) * 16;
        const int xr = r < tile.n ? mx4_x_row(a, tile.row0 + r) : -1;
        int64_t wr[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) wr[t] = (int64_t)tile.e * a.N + t * a.cols + (n0 + r < a.cols ? n0 + r : a.cols - 1);
        mx4_float4 acc[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[t] = (mx4_float4){0.f, 0.f, 0.f, 0.f};
        for (int p = wave; p < a.panels; p += waves) {
            Operand w[NT], x;
#pragma unroll
            for (int t = 0; t < NT; ++t) w[t].load(a.W, p * a.W.rows + wr[t], g);
            if (xr < 0) x.none();
            else if constexpr (XT == HLQ_MX4) x.load(a.A, p * a.A.rows + xr, g);
            else {
                const int k = p * MX4_PANEL_K + g * 32;
                x.quantize((const typename Mx4Type<XT>::type *)a.x + xr * a.ldx + k, a.K - k, a.x_aligned);
            }
#pragma unroll
            for (int t = 0; t < NT; ++t)
                acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(w[t].code), wide(x.code), acc[t], MX4_FP4, MX4_FP4, 0, w[t].scale, 0, x.scale);
        }
        // lane: results of row lane % 16, columns n0 + 4 (lane / 16) ..
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) sums[((wave * NT + t) * 4 + i) * 64 + lane] = acc[t][i];
        __syncthreads();
        if (wave == 0 && r < tile.n && n0 + 4 * g < a.cols) {
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float s[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    s[t] = 0.f;
                    for (int o = 0; o < waves; ++o) s[t] += sums[((o * NT + t) * 4 + i) * 64 + lane];
                }
                v[i] = GATED ? mx4_gate(s[0], s[NT - 1]) : s[0];
            }
            const int left = a.cols - n0 - 4 * g;
            mx4_store(a.y, a.ytype, (int64_t)(tile.row0 + r) * a.ldy + n0 + 4 * g, v, left < 4 ? left : 4, left >= 4 && a.y_aligned);
        }
        __syncthreads();
    }
}

template <int XT, bool GATED>
void launch(const Mx4Product &a, hipStream_t st)
{
    int waves = 1;
    while (waves < 16 && waves < a.panels) waves *= 2;
    const int groups = (a.cols + 15) / 16;
    const int64_t items = mx4_row_tiles(a.R, a.offsets ? a.E : 1, 16) * groups;
    const unsigned grid = (unsigned)(items < (1 << 20) ? items : (1 << 20));
    hlq_mx4_few_kernel<XT, GATED><<<grid, 64 * waves, (size_t)waves * (GATED ? 2 : 1) * 1024, st>>>(a, groups, items);
}

template <int XT>
void launch(const Mx4Product &a, bool gated, hipStream_t st)
{
    if (gated) launch<XT, true>(a, st);
    else launch<XT, false>(a, st);
}

}  // namespace

hlq_status hlq_mx4_launch_few(const Mx4Product &a, int xtype, bool gated, hipStream_t st)
{
    if (xtype == HLQ_F16) launch<HLQ_F16>(a, gated, st);
    else if (xtype == HLQ_BF16) launch<HLQ_BF16>(a, gated, st);
    else if (xtype == HLQ_F32) launch<HLQ_F32>(a, gated, st);
    else launch<HLQ_MX4>(a, gated, st);
    return hlq_hip_status(hipGetLastError());
}
