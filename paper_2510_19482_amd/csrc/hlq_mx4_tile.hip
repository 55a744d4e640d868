// Products of MX4 matrices, many rows: tiles of BM result rows x BN rows of W staged through LDS, on v_mfma_scale_f32_32x32x64_f8f6f4.
//
//   y[r, n] = sum over blocks b of 2^(a_rb + w_nb - 254) sum_{k in b} A[r, k] W[n, k]        (gated: silu(y[r, n]) y[r, N / 2 + n])
//
// The instruction sums a block's 32 products exactly and scales them; the sums over blocks are fp32 in its accumulators.  It is
// the faster of the two forms (random codes, nothing else running: 6.5 PFLOP/s against 5.6 of 16x16x128 with two wavefronts a SIMD).
//
// A stage is a panel of 128 k of the tile's rows, requested straight into LDS (codes 16 bytes a lane, scales 4), a ring of three
// or four stages deep.  Two workgroups share a compute unit: the wavefronts of one multiply while the other waits, starts or
// writes its results.  128 x 256 with a ring of three is the largest that two of fit.  us, 8192 rows, gated, 28672 x 4096:
//   two stages of 256 k, 256 x 256                  605     its requests spread between the matrix instructions       541
//   ... in a ring of four stages of 128 k           495     128 x 256, ring of three, two workgroups a unit           463
//   (128 x 128 529)                                         ... results in streaming stores                     471 (then 481)
// From about one round of the card's units, 256 x 256 with a workgroup that goes from tile to tile is faster (another kernel); this one
// has what is less or does not fill whole rounds.  For experts' rows (512 each on average, 218): waiting for weights that come
// from memory once.
#include "hlq_mx4_stage.h"

namespace {

struct Tiles {
    int col_tiles, row_tiles, splits, share;   // share: panels of a split
    int *arrived;                              // [tile]
    float *partial;                            // [tile][split][wave][register][lane]
};

// Workgroups go to the eight XCDs in turn: each XCD takes a run of tiles, so that its L2 sees few rows and columns.
__device__ __forceinline__ int xcd_order(int id, int n)
{
    const int each = n / 8, more = n % 8, x = id % 8;
    return x * each + (x < more ? x : more) + id / 8;
}

// TM x TN blocks of 32 x 32 a wavefront, GM x GN wavefronts, BUFFERS stages of a panel in LDS; CUT: K may be cut over workgroups.
constexpr int up(int n, int a) { return (n + a - 1) / a * a; }
constexpr int tile_stage(int TM, int TN, int GM, int GN) { return 32 * (TM * GM + TN * GN) * 64 + up(32 * (TM * GM + TN * GN), 64) * 4; }

template <int TM, int TN, int GM, int GN, int BUFFERS, bool CUT, bool GATED>
__global__ void __launch_bounds__(64 * GM * GN, 2)
hlq_mx4_tile_kernel(const Mx4Product a, const Tiles t)
{
    constexpr int BM = 32 * TM * GM, BN = 32 * TN * GN, WAVES = GM * GN;
    constexpr int LOADS = (BM + BN) / 16 / WAVES;                          // requests of 16 rows' codes, a wavefront and stage
    constexpr int SCALE_LOADS = (up(BM + BN, 64) / 64 + WAVES - 1) / WAVES;   // of 64 rows' scales; those past the last repeat it
    constexpr int SCALES = (BM + BN) * 64, STAGE = tile_stage(TM, TN, GM, GN);
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = (int)(threadIdx.x & 63u), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int r = lane & 31, g = lane >> 5, wm = wave / GN, wn = wave % GN;

    // the launch is for the most row tiles that the experts' rows can make; those there are, are dealt out to all XCDs
    const int made = a.offsets ? mx4_count_row_tiles<BM>(a) : t.row_tiles;
    const int row_tiles = made < t.row_tiles ? made : t.row_tiles, tiles = t.col_tiles * row_tiles;   // never more than there is room for
    if ((int)blockIdx.x >= tiles * t.splits) return;
    const int id = xcd_order((int)blockIdx.x, tiles * t.splits);
    const int split = CUT ? id % t.splits : 0, tile_id = CUT ? id / t.splits : id;
    // bands of 8 row tiles, columns after columns
    const int band = tile_id / (8 * t.col_tiles), first = band * 8, high = row_tiles - first < 8 ? row_tiles - first : 8;
    const int in_band = tile_id - first * t.col_tiles;
    const int nt = in_band / high;
    const Mx4RowTile tile = mx4_row_tile<BM>(a, first + in_band - nt * high);

    // row of W for row j of the tile; gated: 32 rows of the first half, then the 32 of the second that go with them
    auto w_row = [&](int j) {
        int c = nt * BN + j, half = 0;
        if (GATED) {
            c = nt * (BN / 2) + (j >> 6) * 32 + (j & 31);
            half = (j >> 5) & 1;
        }
        return (int64_t)tile.e * a.N + (int64_t)half * a.cols + (c < a.cols ? c : a.cols - 1);
    };
    auto x_row = [&](int j) { return (int64_t)mx4_x_row(a, tile.row0 + (j < tile.n ? j : 0)); };

    const int p0 = split * t.share, p1 = p0 + t.share < a.panels ? p0 + t.share : a.panels;
    auto line = [&](int row) { return row < BN ? p0 * a.W.rows + w_row(row) : p0 * a.A.rows + x_row(row - BN); };
    // rows of W and of x are never in one request: BN is a multiple of 64
    const uint8_t *from[LOADS], *scales_from[SCALE_LOADS];
    int64_t step[LOADS], scales_step[SCALE_LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int first_row = (wave * LOADS + i) * 16, row = first_row + (lane >> 2);
        from[i] = (first_row < BN ? a.W.codes : a.A.codes) + line(row) * 64 + ((lane & 3) ^ piece_key(row)) * 16;
        step[i] = (first_row < BN ? a.W.rows : a.A.rows) * 64;
    }
#pragma unroll
    for (int i = 0; i < SCALE_LOADS; ++i) {
        const int n = (wave * SCALE_LOADS + i) * 64 < BM + BN ? wave * SCALE_LOADS + i : up(BM + BN, 64) / 64 - 1;
        const int row = n * 64 + lane < BM + BN ? n * 64 + lane : BM + BN - 1;
        scales_from[i] = (n * 64 < BN ? a.W.scales : a.A.scales) + line(row) * 4;
        scales_step[i] = (n * 64 < BN ? a.W.rows : a.A.rows) * 4;
    }
    // a wavefront's share of a stage, in parts
    constexpr int PER = LOADS + SCALE_LOADS, HALF = PER / 2;
    auto request = [&](int buffer, int i) {
        if (i < SCALE_LOADS) {
            const int n = (wave * SCALE_LOADS + i) * 64 < BM + BN ? wave * SCALE_LOADS + i : up(BM + BN, 64) / 64 - 1;
            dma_4B_per_lane(scales_from[i], (uint32_t)(buffer * STAGE + SCALES + n * 256));
            scales_from[i] += scales_step[i];
        } else {
            const int j = i - SCALE_LOADS;
            dma_16B_per_lane(from[j], (uint32_t)(buffer * STAGE + (wave * LOADS + j) * 1024));
            from[j] += step[j];
        }
    };
    mx4_int4 fw[2][TN], fx[2][TM];
    int ws[2][TN], xs[2][TM];   // [0]: of this stage, [1]: being read
    auto read = [&](int set, int buffer, int s) {
        const int at = buffer * STAGE + r * 64 + ((2 * s + g) ^ piece_key(r)) * 16;
#pragma unroll
        for (int i = 0; i < TN; ++i) fw[set][i] = *(const mx4_int4 *)(lds + at + (wn * TN + i) * 2048);
#pragma unroll
        for (int i = 0; i < TM; ++i) fx[set][i] = *(const mx4_int4 *)(lds + at + BN * 64 + (wm * TM + i) * 2048);
    };
    auto read_scales = [&](int buffer) {
        const int at = buffer * STAGE + SCALES + r * 4 + g * 2;
#pragma unroll
        for (int i = 0; i < TN; ++i) ws[1][i] = *(const uint16_t *)(lds + at + (wn * TN + i) * 128);
#pragma unroll
        for (int i = 0; i < TM; ++i) xs[1][i] = *(const uint16_t *)(lds + at + BN * 4 + (wm * TM + i) * 128);
    };
    auto turn_scales = [&]() {
#pragma unroll
        for (int i = 0; i < TN; ++i) ws[0][i] = ws[1][i];
#pragma unroll
        for (int i = 0; i < TM; ++i) xs[0][i] = xs[1][i];
    };
    mx4_float16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int c = 0; c < 16; ++c) acc[i][j][c] = 0.f;

    // One panel, two steps of 64 k.  The operands of a step are read while the one before is multiplied.  A buffer is free once
    // every wavefront has passed the barrier before its last step's products; it is filled again from there on, a few requests
    // between groups of matrix instructions (in one go they would hold those up), and has come when BUFFERS - 2 later stages
    // may still be on their way.  more: there are stages left to request (else it is waited for all).
    const int count = __builtin_amdgcn_readfirstlane(p1 - p0);
    auto panel = [&](int buffer, auto More) {
        constexpr bool more = decltype(More)::value;
        const int last = buffer == 0 ? BUFFERS - 1 : buffer - 1, next = buffer == BUFFERS - 1 ? 0 : buffer + 1;
        unrolled<2>([&](auto S) {
            constexpr int s = decltype(S)::value;
            if constexpr (s == 0) read(1, buffer, 1);
            else {
                if constexpr (more) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((BUFFERS - 2) * PER) : "memory");
                else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
                read(0, next, 0);   // after the last panel: nobody's
                read_scales(next);
            }
            unrolled<TM>([&](auto I) {
                constexpr int i = decltype(I)::value;
                if constexpr (more) {
                    constexpr int n0 = s == 0 ? HALF : 0, n1 = s == 0 ? PER : HALF;
#pragma unroll
                    for (int n = n0 + (n1 - n0) * i / TM; n < n0 + (n1 - n0) * (i + 1) / TM; ++n) request(s == 0 ? last : buffer, n);
                }
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(fw[s][j]), wide(fx[s][i]), acc[i][j], MX4_FP4, MX4_FP4, s,
                                                                              ws[0][j], s, xs[0][i]);
                if constexpr (more) __builtin_amdgcn_sched_barrier(0);
            });
        });
        turn_scales();
        return next;
    };
    for (int b = 0; b < BUFFERS - 1 && b < count; ++b)
#pragma unroll
        for (int i = 0; i < PER; ++i) request(b, i);
    if (count >= BUFFERS)
#pragma unroll
        for (int i = 0; i < HALF; ++i) request(BUFFERS - 1, i);
    if (count >= BUFFERS) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((BUFFERS - 2) * PER + HALF) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    read(0, 0, 0);
    read_scales(0);
    turn_scales();
    int buffer = 0, p = 0;
    for (; p + BUFFERS < count; ++p) buffer = panel(buffer, std::true_type{});
    if (count >= BUFFERS)
#pragma unroll
        for (int i = HALF; i < PER; ++i) request(buffer == 0 ? BUFFERS - 1 : buffer - 1, i);
    for (; p < count; ++p) buffer = panel(buffer, std::false_type{});
    __syncthreads();

    if (CUT && t.splits > 1) {
        // Partial sums go past the XCD's own L2 (device-scope stores, complete before the arrival is counted); whoever is last of
        // the tile adds them in the order of the splits, those of four splits on their way at a time.
        constexpr int64_t TILE = (int64_t)BM * BN / 2;   // in pairs
        uint64_t *const all = (uint64_t *)t.partial + (int64_t)tile_id * t.splits * TILE + (wave * TM * TN * 8) * 64 + lane;
        uint64_t *const mine = all + split * TILE;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const float low = acc[i][j][2 * c], high = acc[i][j][2 * c + 1];
                    const uint64_t pair = __builtin_bit_cast(uint32_t, low) | (uint64_t)__builtin_bit_cast(uint32_t, high) << 32;
                    __hip_atomic_store(mine + ((i * TN + j) * 8 + c) * 64, pair, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        int *last = (int *)lds;
        if (threadIdx.x == 0) *last = __hip_atomic_fetch_add(t.arrived + tile_id, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == t.splits - 1;
        __syncthreads();
        if (!*last) return;
        if (threadIdx.x == 0) __hip_atomic_store(t.arrived + tile_id, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int c = 0; c < 16; ++c) acc[i][j][c] = 0.f;
            for (int o = 0; o < t.splits; o += 4) {
                uint64_t pair[4][TN][8];
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int j = 0; j < TN; ++j)
#pragma unroll
                        for (int c = 0; c < 8; ++c)
                            pair[q][j][c] = __hip_atomic_load(all + (o + q < t.splits ? o + q : o) * TILE + ((i * TN + j) * 8 + c) * 64, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (o + q < t.splits)
#pragma unroll
                        for (int j = 0; j < TN; ++j)
#pragma unroll
                            for (int c = 0; c < 8; ++c) {
                                acc[i][j][2 * c] += __builtin_bit_cast(float, (uint32_t)pair[q][j][c]);
                                acc[i][j][2 * c + 1] += __builtin_bit_cast(float, (uint32_t)(pair[q][j][c] >> 32));
                            }
            }
        }
        __syncthreads();
    }

    // Results leave by way of LDS, so that rows are written in whole lines: a lane has row m and of each 32 columns 8 q + 4 g .. + 3.
    constexpr int OUT = GATED ? BN / 2 : BN;   // columns of the tile
    auto leave = [&](auto Tag) {
        using V = decltype(Tag);
        constexpr int PITCH = OUT * (int)sizeof(V) + 16, ROWS = 32 * GM, EIGHTS = OUT / 8;
        static_assert(ROWS * PITCH <= BUFFERS * STAGE, "");
        constexpr int SETS = 2 * ROWS * PITCH <= BUFFERS * STAGE ? 2 : 1;
        const int col0 = nt * OUT;
        unrolled<TM>([&](auto I) {
            constexpr int i = decltype(I)::value;
            char *out = lds + (i % SETS) * ROWS * PITCH;
            if (SETS == 1 && i > 0) __syncthreads();
#pragma unroll
            for (int j = 0; j < TN; j += GATED ? 2 : 1) {
                const int c0 = GATED ? ((wn * TN + j) >> 1) * 32 : (wn * TN + j) * 32;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    struct alignas(4 * sizeof(V)) Four { V v[4]; } four;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        four.v[e] = (V)(GATED ? mx4_gate<sizeof(V) == 4>(acc[i][j][4 * q + e], acc[i][j + (GATED ? 1 : 0)][4 * q + e]) : acc[i][j][4 * q + e]);
                    *(Four *)(out + (wm * 32 + r) * PITCH + (c0 + 8 * q + 4 * g) * (int)sizeof(V)) = four;
                }
            }
            __syncthreads();
            for (int n = (int)threadIdx.x; n < ROWS * EIGHTS; n += 64 * WAVES) {
                const int row = n / EIGHTS, c = (n % EIGHTS) * 8, m = ((row >> 5) * TM + i) * 32 + (row & 31);
                if (m >= tile.n || col0 + c >= a.cols) continue;
                const auto v = *(const typename Mx4Eight<V>::Values *)(out + row * PITCH + c * (int)sizeof(V));
                V *to = (V *)a.y + (int64_t)(tile.row0 + m) * a.ldy + col0 + c;
                if (col0 + c + 8 <= a.cols) mx4_stream8(v, to);
                else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (col0 + c + e < a.cols) to[e] = v.v[e];
                }
            }
        });
    };
    if (a.ytype == HLQ_F32) leave(float{});
    else if (a.ytype == HLQ_F16) leave((_Float16)0.f);
    else leave((__bf16)0.f);
}

template <int TM, int TN, int GM, int GN, int BUFFERS, bool CUT>
hlq_status launch(const Mx4Product &a, const Mx4TilePlan &p, bool gated, void *ws, hipStream_t st)
{
    constexpr size_t lds = (size_t)tile_stage(TM, TN, GM, GN) * BUFFERS;
    const Tiles t{p.col_tiles, p.row_tiles, p.splits, p.share, (int *)ws, (float *)((char *)ws + p.partial_at)};
    const int64_t blocks = (int64_t)p.col_tiles * p.row_tiles * p.splits;
    if (blocks > (int64_t)(UINT32_MAX / 256)) return HLQ_ERR_UNSUPPORTED;   // threads of a launch: below 2^32
    auto kernel = gated ? hlq_mx4_tile_kernel<TM, TN, GM, GN, BUFFERS, CUT, true> : hlq_mx4_tile_kernel<TM, TN, GM, GN, BUFFERS, CUT, false>;
    kernel<<<(unsigned)blocks, 64 * GM * GN, lds, st>>>(a, t);
    return hlq_hip_status(hipGetLastError());
}

}  // namespace

hlq_status hlq_mx4_launch_tile(const Mx4Product &a, const Mx4TilePlan &p, bool gated, void *ws, hipStream_t st)
{
    if (p.BM == 128 && p.BN == 256) return launch<2, 4, 2, 2, 3, false>(a, p, gated, ws, st);
    if (p.BM == 128) return launch<2, 2, 2, 2, 4, true>(a, p, gated, ws, st);
    if (p.BM == 64) return launch<2, 2, 1, 2, 4, true>(a, p, gated, ws, st);
    return launch<1, 2, 1, 2, 4, true>(a, p, gated, ws, st);
}
