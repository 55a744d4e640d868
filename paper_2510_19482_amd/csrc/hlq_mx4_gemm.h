// Products of MX4 matrices: arguments that the kernels share, and which rows a workgroup takes.
#pragma once

#include "hlq_mx4.h"

// an operand of 4-bit values as the matrix instruction takes it
__device__ __forceinline__ mx4_int8 wide(mx4_int4 v) { return (mx4_int8){v.x, v.y, v.z, v.w, 0, 0, 0, 0}; }

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
// rows [lo, hi) of expert e, within 0..R - 1; none for e >= E.  start(e): offset e
template <class Start>
__device__ __forceinline__ void mx4_expert_rows(const Mx4Product &a, int e, int &lo, int &hi, Start start)
{
    lo = hi = a.R;
    if (e < a.E) {
        lo = start(e);
        hi = start(e + 1);
    }
    lo = lo < 0 ? 0 : lo > a.R ? a.R : lo;
    hi = hi < lo ? lo : hi > a.R ? a.R : hi;
}
// the sum of tiles(n) over the experts, n the rows of one, in a scalar register
template <class Start, class Tiles>
__device__ __forceinline__ int mx4_count_tiles(const Mx4Product &a, Start start, Tiles tiles)
{
    const int lane = (int)(threadIdx.x & 63u);
    int n = 0;
    for (int base = 0; base < a.E; base += 64) {
        int lo, hi;
        mx4_expert_rows(a, base + lane, lo, hi, start);
        n += tiles(hi - lo);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) n += __shfl_xor(n, d);
    return __builtin_amdgcn_readfirstlane(n);
}
// which expert has tile number `tile` of those, the how manieth of its own it is, and the expert's rows; rows 0..-1: there are fewer tiles
struct Mx4ExpertTile {
    int e, index, lo, hi;
};
template <class Start, class Tiles>
__device__ __forceinline__ Mx4ExpertTile mx4_find_tile(const Mx4Product &a, int tile, Start start, Tiles tiles)
{
    const int lane = (int)(threadIdx.x & 63u);
    int before = 0;
    for (int base = 0; base < a.E; base += 64) {
        int lo, hi;
        mx4_expert_rows(a, base + lane, lo, hi, start);
        int upto = tiles(hi - lo);
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
            return {base + f, tile - before - (__builtin_amdgcn_readlane(upto, f) - __builtin_amdgcn_readlane(mine, f)), __builtin_amdgcn_readlane(lo, f),
                    __builtin_amdgcn_readlane(hi, f)};
        }
        before += all;
    }
    return {0, 0, 0, 0};
}
template <int BM>
__device__ __forceinline__ int mx4_count_row_tiles(const Mx4Product &a)
{
    return mx4_count_tiles(a, [&](int e) { return a.offsets[e]; }, [](int n) { return n / BM + (n % BM != 0); });
}
template <int BM>
__device__ __forceinline__ Mx4RowTile mx4_row_tile(const Mx4Product &a, int tile)
{
    if (!a.offsets) {
        const int64_t r = (int64_t)tile * BM;
        if (r >= a.R) return {0, 0, 0};
        return {0, (int)r, (int)(a.R - r < BM ? a.R - r : BM)};
    }
    const Mx4ExpertTile t = mx4_find_tile(a, tile, [&](int e) { return a.offsets[e]; }, [](int n) { return n / BM + (n % BM != 0); });
    const int r = t.lo + t.index * BM;
    return {t.e, r, t.hi - r < BM ? t.hi - r : BM};
}

// Most row tiles that R rows of E experts make.
static inline int64_t mx4_row_tiles(int64_t R, int E, int BM)
{
    const int64_t full = (R + BM - 1) / BM;
    return E <= 1 ? full : R / BM + (R < E ? R : E);
}

// row of x for row r (r < R); an index outside x is taken as its nearest end, so that nothing outside is read
__device__ __forceinline__ int mx4_inside_x(const Mx4Product &a, int i) { return i < 0 ? 0 : i >= a.x_rows ? a.x_rows - 1 : i; }
__device__ __forceinline__ int mx4_x_row(const Mx4Product &a, int r) { return a.rows ? mx4_inside_x(a, a.rows[r]) : r; }

// How a launch for few rows is cut: row_tiles x groups workgroups of `waves` wavefronts, `share` of them for the same columns.
struct Mx4FewShape {
    int share, waves, groups;
    int64_t row_tiles;
};
// a wavefront has row_blocks x col_blocks blocks of 16 x 16: 1 x 1, 2 x 1, 2 x 2 or 4 x 2 (1 x 1 if x is quantized inside: xtype is not HLQ_MX4)
Mx4FewShape hlq_mx4_few_shape(int cols, int K, int panels, int E, int64_t R, int xtype, int row_blocks, int col_blocks);
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
