// Products of MX4 matrices for few rows (a decoded token or batch, an expert's few rows): up to 64 rows a workgroup, no LDS in the loop.
//
//   y[r, n] = sum over blocks b of 2^(a_rb + w_nb - 254) sum_{k in b} A[r, k] W[n, k]        (gated: silu(y[r, n]) y[r, N / 2 + n])
//
// Bound by the weights' bytes.  A wavefront holds 16 or 32 rows of W (results' columns), 16 to 64 rows of x and a share of the
// panels; the wavefronts of a workgroup that share the columns add their sums through LDS, in order.  Operands go straight to
// registers in the form that v_mfma_scale_f32_16x16x128_f8f6f4 takes, panels of several steps requested together.  A few rows
// that come as f16, bf16 or f32 are quantized by the workgroup into LDS while its first weights come; that saves a launch.
// us, weights from memory, one bf16 row: 4096 x 4096 5.4, 6144 x 4096 6.5, 28672 x 4096 15.0 (62 MB, 4.2 TB/s), 4096 x 14336 9.8 (with the weights in
// the memory-side cache 4.4, 5.3, 12.3, 7.2); 16 rows of 32 experts (14 of them used), gated 4096 x 4096: 25.5 (118 MB, 4.6 TB/s; a plain read reaches 7.1).
// With more rows what a compute unit loads into registers (43 bytes a nanosecond) takes over: 32 rows 4096 x 14336 12.6, 128 rows 4096 x 4096 8.4.
// Loads that bypass the caches for the weights: no difference (28672 x 4096, from the memory-side cache, 12.2 -> 12.7).
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
};

// Rows of x in the form that the matrix core takes, in LDS: codes [panel][row][64], scales [panel][row][4], for the n rows of a tile.
template <class T>
__device__ __forceinline__ void quantize_rows(const Mx4Product &a, const Mx4RowTile &tile, uint8_t *codes, uint8_t *scales)
{
    const int eights = a.panels * 16, lane = (int)(threadIdx.x & 63u);
    for (int i = (int)threadIdx.x; i < tile.n * eights; i += (int)blockDim.x) {
        const int m = i / eights, j = i - m * eights, k = j * 8, at = (j >> 4) * tile.n + m;
        const T *p = (const T *)a.x + mx4_x_row(a, tile.row0 + m) * a.ldx + k;
        T v[8];
        mx4_load8<false>(p, a.K - k, v);
        const uint32_t byte = mx4_scale_of(mx4_quad_max(mx4_top_bits(v)));
        *(uint32_t *)(codes + at * 64 + (j & 15) * 4) = mx4_codes(v, byte);
        if ((lane & 3) == 0) scales[at * 4 + mx4_scale_byte((j >> 2) & 3)] = (uint8_t)byte;
    }
}

constexpr int few_ahead(int MT, int CT) { return MT * CT >= 4 ? 2 : 4; }   // panels requested at a time
constexpr int few_waves(int MT, int CT) { return MT * CT >= 4 ? 8 : 16; }   // of a workgroup, at most

// MT blocks of 16 rows, CT blocks of 16 columns a wavefront.  K is cut over the `share` wavefronts that have the same columns; a
// workgroup has blockDim / 64 / share such groups.
template <int XT, bool GATED, int MT, int CT>
__global__ void __launch_bounds__(64 * few_waves(MT, CT))
hlq_mx4_few_kernel(const Mx4Product a, int groups, int share)
{
    constexpr int NT = GATED ? 2 * CT : CT, AHEAD = few_ahead(MT, CT);   // blocks of W: gated ones in pairs
    constexpr bool INSIDE = XT != HLQ_MX4;   // x is quantized here
    static_assert(!INSIDE || MT == 1, "");
    extern __shared__ __attribute__((aligned(16))) float sums[];   // [wavefront][MT][NT][4][64], then x
    const int lane = (int)(threadIdx.x & 63u), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int r = lane & 15, g = lane >> 4, per = (int)(blockDim.x >> 6) / share;
    const Mx4RowTile tile = mx4_row_tile<16 * MT>(a, (int)blockIdx.x / groups);
    if (tile.n == 0) return;
    const int col = ((int)blockIdx.x % groups * per + wave / share) * 16 * CT, part = wave % share;
    const bool mine = col < a.cols;   // the last workgroup may have more wavefronts than columns
    int64_t wr[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int c = col + (GATED ? t >> 1 : t) * 16 + r;
        wr[t] = (int64_t)tile.e * a.N + (GATED && (t & 1) ? a.cols : 0) + (c < a.cols ? c : a.cols - 1);
    }
    Operand w[AHEAD][NT];
    auto load_w = [&](int p0) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int t = 0; t < NT; ++t)
                if (p0 + u * share < a.panels) w[u][t].load(a.W, (p0 + u * share) * a.W.rows + wr[t], g);
                else w[u][t].none();
    };
    load_w(part);
    Mx4View X = a.A;
    if constexpr (INSIDE) {
        // while the first weights come
        uint8_t *codes = (uint8_t *)(sums + (share > 1 ? (int)(blockDim.x >> 6) * NT * 256 : 0)), *scales = codes + tile.n * a.panels * 64;
        quantize_rows<typename Mx4Type<XT>::type>(a, tile, codes, scales);
        X = Mx4View{codes, scales, tile.n};
        __syncthreads();
    }
    int xr[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) xr[m] = m * 16 + r >= tile.n ? -1 : INSIDE ? r : mx4_x_row(a, tile.row0 + m * 16 + r);
    mx4_float4 acc[MT][NT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[m][t] = (mx4_float4){0.f, 0.f, 0.f, 0.f};
    for (int p0 = part; p0 < a.panels; p0 += share * AHEAD) {
        if (p0 > part) load_w(p0);
        Operand x[AHEAD][MT];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int m = 0; m < MT; ++m)
                if (p0 + u * share < a.panels && xr[m] >= 0) x[u][m].load(X, (p0 + u * share) * X.rows + xr[m], g);
                else x[u][m].none();
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    acc[m][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(w[u][t].code), wide(x[u][m].code), acc[m][t], MX4_FP4, MX4_FP4, 0,
                                                                             w[u][t].scale, 0, x[u][m].scale);
    }
    // a lane has results of row lane % 16, columns 4 (lane / 16) .. of each block; the wavefronts of a group add them up block by block
    auto leave = [&](int m, int ct, const mx4_float4 &p, const mx4_float4 &up) {
        const int c = col + ct * 16 + 4 * g, left = a.cols - c;
        if (m * 16 + r >= tile.n || left <= 0) return;
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = GATED ? mx4_gate<true>(p[i], up[i]) : p[i];
        mx4_store4(a.y, a.ytype, (int64_t)(tile.row0 + m * 16 + r) * a.ldy + c, v, left);
    };
    if (share == 1) {
        if (mine)
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int c = 0; c < CT; ++c) leave(m, c, acc[m][GATED ? 2 * c : c], acc[m][GATED ? 2 * c + 1 : c]);
        return;
    }
    float *const group = sums + (wave - part) * (MT * NT * 256);
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) group[((part * MT + m) * NT + t) * 256 + i * 64 + lane] = acc[m][t][i];
    __syncthreads();
    if (!mine) return;
    for (int b = part; b < MT * CT; b += share) {
        const int m = b / CT, c = b % CT;
        mx4_float4 s[2];
#pragma unroll
        for (int t = 0; t < (GATED ? 2 : 1); ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float sum = 0.f;
                for (int o = 0; o < share; ++o) sum += group[((o * MT + m) * NT + (GATED ? 2 * c + t : c)) * 256 + i * 64 + lane];
                s[t][i] = sum;
            }
        leave(m, c, s[0], s[GATED ? 1 : 0]);
    }
}

template <int XT, bool GATED, int MT, int CT>
hlq_status launch(const Mx4Product &a, hipStream_t st)
{
    const Mx4FewShape f = hlq_mx4_few_shape(a.cols, a.K, a.panels, a.offsets ? a.E : 1, a.R, XT, MT, CT);
    if (f.row_tiles * f.groups > (int64_t)(UINT32_MAX / 1024)) return HLQ_ERR_UNSUPPORTED;   // threads of a launch: below 2^32
    size_t lds = f.share > 1 ? (size_t)f.waves * MT * CT * (GATED ? 2 : 1) * 1024 : 0;
    if (XT != HLQ_MX4) lds += (size_t)(a.R < 16 ? a.R : 16) * a.panels * 68;
    hlq_mx4_few_kernel<XT, GATED, MT, CT><<<(unsigned)(f.row_tiles * f.groups), 64 * f.waves, lds, st>>>(a, f.groups, f.share);
    return hlq_hip_status(hipGetLastError());
}

template <int XT, int MT, int CT>
hlq_status launch(const Mx4Product &a, bool gated, hipStream_t st)
{
    return gated ? launch<XT, true, MT, CT>(a, st) : launch<XT, false, MT, CT>(a, st);
}

}  // namespace

Mx4FewShape hlq_mx4_few_shape(int cols, int K, int panels, int E, int64_t R, int xtype, int row_blocks, int col_blocks)
{
    const int col_tiles = (cols + 16 * col_blocks - 1) / (16 * col_blocks), most = few_waves(row_blocks, col_blocks);
    Mx4FewShape f;
    f.row_tiles = mx4_row_tiles(R, E, 16 * row_blocks);
    // wavefronts that share a column tile: about `most` wavefronts a compute unit in all, AHEAD panels or more each
    f.share = 1;
    while (f.share < most && f.row_tiles * col_tiles * f.share < 256 * most && f.share * few_ahead(row_blocks, col_blocks) < panels) f.share *= 2;
    // x quantized inside: by wavefronts enough. us with 8 / 16, weights in the memory-side cache: one row, 4096 x 4096 4.4 / 5.2; four rows, 6144 x 4096 7.1 / 6.2
    f.waves = xtype == HLQ_MX4 ? 4 : (R + E - 1) / E * K > 8192 ? 16 : 8;
    if (f.waves < f.share) f.waves = f.share;
    const int per = f.waves / f.share;
    f.groups = (col_tiles + per - 1) / per;
    return f;
}

hlq_status hlq_mx4_launch_few(const Mx4Product &a, int xtype, bool gated, int row_blocks, int col_blocks, hipStream_t st)
{
    if (xtype == HLQ_F16) return launch<HLQ_F16, 1, 1>(a, gated, st);
    if (xtype == HLQ_BF16) return launch<HLQ_BF16, 1, 1>(a, gated, st);
    if (xtype == HLQ_F32) return launch<HLQ_F32, 1, 1>(a, gated, st);
    if (row_blocks == 1) return launch<HLQ_MX4, 1, 1>(a, gated, st);
    if (row_blocks == 4) return launch<HLQ_MX4, 4, 2>(a, gated, st);
    return col_blocks == 1 ? launch<HLQ_MX4, 2, 1>(a, gated, st) : launch<HLQ_MX4, 2, 2>(a, gated, st);
}
