// Products of MX4 matrices: arguments that the kernels share, and which rows a workgroup takes.
#pragma once

#include "hlq_mx4.h"

struct Mx4Product {
    Mx4View W;              // [E * N, K]: matrix e in rows e * N ..
    int N, cols, K, panels; // cols: of the result, N or N / 2 (gated)
    const int32_t *offsets; // NULL: one matrix, rows 0..R - 1
    int E;
    const int32_t *rows;    // row of x for each of the R rows; NULL: the same
    int R, x_rows;
    const void *x;          // f16, bf16 or f32 rows that the kernel quantizes; else A
    int64_t ldx;
    Mx4View A;
    void *y;
    int ytype;
    int64_t ldy;
};

// Row tile number `tile` of tiles of BM rows that begin anew at each expert.  Every lane of the wavefront takes part and gets
// the same answer; n = 0: there are fewer tiles.  Offsets are device data: whatever they hold, rows stay within 0..R - 1.
struct Mx4RowTile {
    int e, row0, n;
};
// rows [lo, hi) of expert e, within 0..R - 1; none for e >= E
__device__ __forceinline__ void mx4_expert_rows(const Mx4Product &a, int e, int &lo, int &hi)
{
    lo = hi = a.R;
    if (e < a.E) {
        lo = a.offsets[e];
        hi = a.offsets[e + 1];
    }
    lo = lo < 0 ? 0 : lo > a.R ? a.R : lo;
    hi = hi < lo ? lo : hi > a.R ? a.R : hi;
}
// how many there are, in a scalar register
template <int BM>
__device__ __forceinline__ int mx4_count_row_tiles(const Mx4Product &a)
{
    const int lane = (int)(threadIdx.x & 63u);
    int n = 0;
    for (int base = 0; base < a.E; base += 64) {
        int lo, hi;
        mx4_expert_rows(a, base + lane, lo, hi);
        n += (hi - lo) / BM + ((hi - lo) % BM != 0);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) n += __shfl_xor(n, d);
    return __builtin_amdgcn_readfirstlane(n);
}
template <int BM>
__device__ __forceinline__ Mx4RowTile mx4_row_tile(const Mx4Product &a, int tile)
{
    if (!a.offsets) {
        const int64_t r = (int64_t)tile * BM;
        if (r >= a.R) return {0, 0, 0};
        return {0, (int)r, (int)(a.R - r < BM ? a.R - r : BM)};
    }
    const int lane = (int)(threadIdx.x & 63u);
    int before = 0;
    for (int base = 0; base < a.E; base += 64) {
        int lo, hi;
        mx4_expert_rows(a, base + lane, lo, hi);
        int upto = (hi - lo) / BM + ((hi - lo) % BM != 0);
        const int mine = upto;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
        }
        const int all = __builtin_amdgcn_readlane(upto, 63);
        if (tile - before < all) {
            const uint64_t past = __ballot(upto > tile - before);
            const int f = (int)__builtin_ctzll(past);
            const int l = __builtin_amdgcn_readlane(lo, f), h = __builtin_amdgcn_readlane(hi, f);
            const int r = l + (tile - before - (__builtin_amdgcn_readlane(upto, f) - __builtin_amdgcn_readlane(mine, f))) * BM;
            return {base + f, r, h - r < BM ? h - r : BM};
        }
        before += all;
    }
    return {0, 0, 0};
}

// Most row tiles that R rows of E experts make.
static inline int64_t mx4_row_tiles(int64_t R, int E, int BM)
{
    const int64_t full = (R + BM - 1) / BM;
    return E <= 1 ? full : R / BM + (R < E ? R : E);
}

// row of x for row r (r < R); an index outside x is taken as its nearest end, so that nothing outside is read
__device__ __forceinline__ int mx4_x_row(const Mx4Product &a, int r)
{
    if (!a.rows) return r;
    const int i = a.rows[r];
    return i < 0 ? 0 : i >= a.x_rows ? a.x_rows - 1 : i;
}

// a wavefront has row_blocks x col_blocks blocks of 16 x 16: 1 x 1, 2 x 1, 2 x 2 or 4 x 2 (1 x 1 if x is quantized inside)
hlq_status hlq_mx4_launch_few(const Mx4Product &a, int xtype, bool gated, int row_blocks, int col_blocks, hipStream_t st);

// How a launch of the tiled kernel is cut: col_tiles x row_tiles x splits workgroups, a split `share` panels of K.  Partial
// sums lie behind the counters in the workspace.
struct Mx4TilePlan {
    int BM, BN, col_tiles, row_tiles, splits, share;
    size_t partial_at, partial_bytes;
};
hlq_status hlq_mx4_launch_tile(const Mx4Product &a, const Mx4TilePlan &p, bool gated, void *ws, hipStream_t st);
// BM = 256, K not cut; a workgroup takes tile after tile
hlq_status hlq_mx4_launch_big(const Mx4Product &a, const Mx4TilePlan &p, bool gated, hipStream_t st);
