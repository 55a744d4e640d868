// Products of MX4 matrices, large launches: tiles of 256 rows x 256 rows of W, one workgroup a compute unit, which goes from tile to
// tile.  The mathematics and the staging are those of the smaller tiles.
//
// What bounds large products: the clock, which power holds at 1.74 to 1.81 GHz (the matrix cores alone, busy all the time: 1.6 on random codes, 2.3 on
// zeros; with zeros for operands 454 us become 331), and the cycles in which nothing multiplies, 42 % of them: 5 us a tile are its
// results, over K the panels run at 5.2 PFLOP/s.  It helps to feed the cores less: of LDS a wavefront with 2 x 4 blocks reads 6 pieces
// for 8 products (2 x 2 blocks: 8), of memory and L2 a tile loads 256 + 256 rows where two of 128 x 256 load 768.  A unit holds one
// such workgroup (four stages, 136 KB), so nothing hides a tile's first loads and its results but the kernel itself: the next tile's
// first stages are requested before the results leave.
// us, 8192 rows, 28672 x 4096 gated / 8192 x 28672 plain, against 485 / 874 of 128 x 256 in the same minute:
//   one workgroup a tile                                    453 / 786 (then 465 / 846)
//   a workgroup goes from tile to tile                      438 / 771
//   results in lines of 128 bytes, not 64                   450 / 809 (8192 x 28672 x 256 plain, all results: 172 -> 110)
//   a step's operands read 6 products behind the barrier    426 / 777 (devices differ by 5 %: 454 / 771 and 445 / 771 on two others)
// 4 wavefronts with 4 x 4 blocks: 4 % less a panel, but 20 us a tile for results that spill.  A wavefront's priority raised for its
// products: 2 % slower.
// Experts' rows, 16384 of 32, gated 4096 x 4096, skewed / 512 each give or take 22, against 193 / 208 of 128 x 256:
//   every tile multiplied in full                           188 / 230
//   offsets from LDS, the next tile's rows looked up early, wavefronts without rows do not multiply    177 / 230
//   low tiles after the high ones                           180 / 207 (8192 rows of 8 89 -> 85, of 64 133; with weights that take turns 194)
//   (a queue that workgroups take tiles from: 182 / 203, but 8192 rows of 8 102: a number's way is 5 us a tile)
// What bounds them: weights that come from memory once, and rows gathered by index (512 each exactly: 150; rows in order 131).
#include "hlq_mx4_stage.h"

namespace {

constexpr int TM = 2, TN = 4, GM = 4, GN = 2;       // blocks of 32 x 32 a wavefront, wavefronts
constexpr int BM = 32 * TM * GM, BN = 32 * TN * GN, WAVES = GM * GN;
constexpr int BAND = 4;   // row tiles that a run of tiles goes through column after column
constexpr int BUFFERS = 4, SCALES = (BM + BN) * 64, STAGE = (BM + BN) * 68;
constexpr int LOADS = (BM + BN) / 16 / WAVES, PER = LOADS + 1, HALF = PER / 2;   // requests of a wavefront and stage: codes, scales
constexpr int PITCH = 144, STAGING = 16 * PITCH;    // of a wavefront: 16 rows of 128 bytes
constexpr int STARTS = BUFFERS * STAGE + WAVES * STAGING, LDS = STARTS + 4 * (HLQ_MAX_EXPERTS + 1);   // where the experts' offsets are
static_assert((BM + BN) == 64 * WAVES && LDS <= 160 * 1024 && TM == 2 && TN == 4 && PER == 5 && HALF == 2, "the schedule of a panel");

struct Place {
    int nt;
    Mx4RowTile rows;
};

template <bool GATED>
__global__ void __launch_bounds__(64 * WAVES, 2)
hlq_mx4_big_kernel(const Mx4Product a, int col_tiles, int most_row_tiles)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = (int)(threadIdx.x & 63u), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int r = lane & 31, g = lane >> 5, wm = wave / GN, wn = wave % GN;
    const bool of_x = wave >= BN / 64;   // a wavefront requests 64 rows of W or of x

    // Row tiles of experts: the high ones first, then those of an expert's last 128 rows or fewer, in which half of the wavefronts have
    // nothing to multiply; so that the workgroups end nearly together.
    const int *const starts = (const int *)(lds + STARTS);
    const auto start = [&](int e) { return starts[e]; };
    const auto high = [](int n) { return n / BM + (n % BM > BM / 2); };
    const auto low = [](int n) { return (int)(n % BM > 0 && n % BM <= BM / 2); };
    int row_tiles = most_row_tiles, low_row_tiles = 0;
    if (a.offsets) {
        for (int e = (int)threadIdx.x; e <= a.E; e += 64 * WAVES) *(int *)(lds + STARTS + 4 * e) = a.offsets[e];
        __syncthreads();
        // never more than the host has counted on, whatever the offsets are
        row_tiles = mx4_count_tiles(a, start, high);
        low_row_tiles = mx4_count_tiles(a, start, low);
        row_tiles = row_tiles < 0 || row_tiles > most_row_tiles ? most_row_tiles : row_tiles;
    }
    // Workgroups go to the eight XCDs in turn: each XCD has a run of tiles, in bands of four row tiles, columns after columns, so that
    // its L2 sees few rows and columns; its workgroups take them in turn.
    const int xcd = (int)blockIdx.x % 8, step = ((int)gridDim.x - xcd + 7) / 8;   // workgroups of this XCD
    auto run = [&](int tiles, int x) { return x * (tiles / 8) + (x < tiles % 8 ? x : tiles % 8); };   // where XCD x begins
    const int first_high = run(col_tiles * row_tiles, xcd), high_ones = run(col_tiles * row_tiles, xcd + 1) - first_high;
    const int first_low = run(col_tiles * low_row_tiles, xcd), end = high_ones + run(col_tiles * low_row_tiles, xcd + 1) - first_low;
    auto place = [&](int id) {
        const bool is_low = id >= high_ones;
        const int tile = is_low ? first_low + id - high_ones : first_high + id, rows = is_low ? low_row_tiles : row_tiles;
        const int band = tile / (BAND * col_tiles), first = band * BAND, height = rows - first < BAND ? rows - first : BAND;
        const int in_band = tile - first * col_tiles, nt = in_band / height, mt = first + in_band - nt * height;
        if (!a.offsets) return Place{nt, mx4_row_tile<BM>(a, mt)};
        const Mx4ExpertTile t = is_low ? mx4_find_tile(a, mt, start, low) : mx4_find_tile(a, mt, start, high);
        const int n = t.hi - t.lo, r = is_low ? n / BM * BM : t.index * BM;
        return Place{nt, Mx4RowTile{t.e, t.lo + r, n - r < BM ? n - r : BM}};
    };
    // the row of W or of x that this lane's number of the wavefront's 64 rows is; of x as it stands, not yet known to be inside
    auto look = [&](const Place &p) {
        if (of_x) {
            const int j = wave * 64 - BN + lane;
            const int i = p.rows.row0 + (j < p.rows.n ? j : 0);
            return a.rows ? a.rows[i] : i;
        }
        const int j = wave * 64 + lane;
        int c = p.nt * BN + j, half = 0;
        if (GATED) {   // 32 rows of the first half, then the 32 of the second that go with them
            c = p.nt * (BN / 2) + (j >> 6) * 32 + (j & 31);
            half = (j >> 5) & 1;
        }
        return p.rows.e * a.N + half * a.cols + (c < a.cols ? c : a.cols - 1);
    };
    const int64_t rows64 = (of_x ? a.A.rows : a.W.rows) * 64, rows4 = (of_x ? a.A.rows : a.W.rows) * 4;
    const uint8_t *from[LOADS], *scale_from;
    auto aim = [&](int found) {
        const int row = of_x ? mx4_inside_x(a, found) : found;
        const uint8_t *codes = of_x ? a.A.codes : a.W.codes, *scales = of_x ? a.A.scales : a.W.scales;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int in_tile = wave * 64 + i * 16 + (lane >> 2);
            from[i] = codes + (int64_t)__shfl(row, i * 16 + (lane >> 2)) * 64 + ((lane & 3) ^ piece_key(in_tile)) * 16;
        }
        scale_from = scales + (int64_t)row * 4;
    };
    auto request = [&](int buffer, int i) {
        if (i == 0) {
            dma_4B_per_lane(scale_from, (uint32_t)(buffer * STAGE + SCALES + wave * 256));
            scale_from += rows4;
        } else {
            dma_16B_per_lane(from[i - 1], (uint32_t)(buffer * STAGE + (wave * LOADS + i - 1) * 1024));
            from[i - 1] += rows64;
        }
    };
    const int count = a.panels;
    auto request_first = [&]() {
        for (int b = 0; b < BUFFERS - 1 && b < count; ++b)
#pragma unroll
            for (int i = 0; i < PER; ++i) request(b, i);
        if (count >= BUFFERS)
#pragma unroll
            for (int i = 0; i < HALF; ++i) request(BUFFERS - 1, i);
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
    auto multiply = [&](auto S, int i, int j) {
        constexpr int s = decltype(S)::value;
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(fw[s][j]), wide(fx[s][i]), acc[i][j], MX4_FP4, MX4_FP4, s, ws[0][j], s, xs[0][i]);
    };
    constexpr std::integral_constant<int, 0> first{};
    constexpr std::integral_constant<int, 1> second{};
    // One panel, two steps of 64 k.  The next step's operands are read late: behind the barrier every wavefront has them to read, and
    // products that wait for none of them come first.
    auto panel = [&](int buffer, auto More) {
        constexpr bool more = decltype(More)::value;
        const int last = buffer == 0 ? BUFFERS - 1 : buffer - 1, next = buffer == BUFFERS - 1 ? 0 : buffer + 1;
        for (int j = 0; j < 4; ++j) multiply(first, 0, j);
        __builtin_amdgcn_sched_barrier(0);
        read(1, buffer, 1);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (more) request(last, 2);
        __builtin_amdgcn_sched_barrier(0);
        multiply(first, 1, 0);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (more) {
            request(last, 3);
            request(last, 4);
        }
        __builtin_amdgcn_sched_barrier(0);
        for (int j = 1; j < 4; ++j) multiply(first, 1, j);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (more) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((BUFFERS - 2) * PER) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        for (int j = 0; j < 4; ++j) multiply(second, 0, j);
        for (int j = 0; j < 2; ++j) multiply(second, 1, j);
        __builtin_amdgcn_sched_barrier(0);
        read(0, next, 0);   // after the last panel: nobody's
        read_scales(next);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (more) request(buffer, 0);
        __builtin_amdgcn_sched_barrier(0);
        multiply(second, 1, 2);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (more) request(buffer, 1);
        __builtin_amdgcn_sched_barrier(0);
        multiply(second, 1, 3);
        __builtin_amdgcn_sched_barrier(0);
        turn_scales();
        return next;
    };

    auto idle = [&](int buffer, auto More) {   // a panel without products
        if constexpr (decltype(More)::value) {
#pragma unroll
            for (int i = HALF; i < PER; ++i) request(buffer == 0 ? BUFFERS - 1 : buffer - 1, i);
            asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((BUFFERS - 2) * PER) : "memory");
#pragma unroll
            for (int i = 0; i < HALF; ++i) request(buffer, i);
        } else
            asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
        return buffer == BUFFERS - 1 ? 0 : buffer + 1;
    };
    auto request_rest = [&](int buffer) {
        if (count >= BUFFERS)
#pragma unroll
            for (int i = HALF; i < PER; ++i) request(buffer == 0 ? BUFFERS - 1 : buffer - 1, i);
    };

    // Results of one tile: a wavefront turns its blocks round in LDS of its own, 16 rows of 128 bytes at a time, so that rows leave
    // in whole lines.  No barrier: LDS accesses of a wavefront keep their order.
    constexpr int OUT = GATED ? BN / 2 : BN;   // columns of the tile
    auto leave = [&](const Place &p, auto Tag) {
        using V = decltype(Tag);
        constexpr int N = 16 / (int)sizeof(V), BLOCKS = 4 / (int)sizeof(V);   // columns of 16 bytes, blocks of 32 columns that make 128
        constexpr int JS = GATED ? 2 * BLOCKS : BLOCKS;
        struct alignas(4 * sizeof(V)) Four { V v[4]; };
        struct alignas(16) Some { V v[N]; };
        char *const mine = lds + BUFFERS * STAGE + wave * STAGING;
        // Pieces that are whole lines leave L2 to the operands (28672 x 4096 plain 478 -> 455); parts of lines have to meet there
        // (3000 rows, 5000 x 4096: 44.5 -> 38.4).
        const bool lines = ((uintptr_t)a.y | ((uintptr_t)a.ldy * sizeof(V))) % 128u == 0;
        unrolled<TM>([&](auto I) {
            constexpr int i = decltype(I)::value;
            unrolled<TN / JS>([&](auto J) {
                constexpr int j0 = decltype(J)::value * JS;
                Four four[BLOCKS][4];
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                    for (int n = 0; n < 16; ++n)
                        four[b][n / 4].v[n % 4] = (V)(GATED ? mx4_gate<sizeof(V) == 4>(acc[i][GATED ? j0 + 2 * b : 0][n], acc[i][GATED ? j0 + 2 * b + 1 : 0][n]) : acc[i][j0 + (GATED ? 0 : b)][n]);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if ((r >> 4) == h)
#pragma unroll
                        for (int q = 0; q < 4 * BLOCKS; ++q) *(Four *)(mine + (r & 15) * PITCH + (8 * q + 4 * g) * (int)sizeof(V)) = four[q / 4][q % 4];
                    __builtin_amdgcn_wave_barrier();
#pragma unroll
                    for (int o = 0; o < 2; ++o) {
                        const int row = o * 8 + (lane >> 3), m = (wm * TM + i) * 32 + h * 16 + row;
                        const int c = p.nt * OUT + (GATED ? (wn * TN + j0) / 2 : wn * TN + j0) * 32 + (lane & 7) * N;
                        const Some v = *(const Some *)(mine + row * PITCH + (lane & 7) * 16);
                        V *to = (V *)a.y + (int64_t)(p.rows.row0 + m) * a.ldy + c;
                        if (m < p.rows.n && c + N <= a.cols) {
                            if (lines) __builtin_nontemporal_store(__builtin_bit_cast(mx4_u4, v), (mx4_u4_any *)to);
                            else {
                                asm volatile("" ::: "memory");   // else the compiler makes one store of the two, an ordinary one
                                *(mx4_u4_any *)to = __builtin_bit_cast(mx4_u4, v);
                                asm volatile("" ::: "memory");
                            }
                        }
                        else if (m < p.rows.n) {
#pragma unroll
                            for (int e = 0; e < N; ++e)
                                if (c + e < a.cols) to[e] = v.v[e];
                        }
                    }
                    __builtin_amdgcn_wave_barrier();
                }
            });
        });
    };

    int id = (int)blockIdx.x / 8;
    Place now{};
    if (id < end) {
        now = place(id);
        aim(look(now));
        request_first();
    }
    while (id < end) {
        // loads come in the order of their requests; stores of the tile before, where there are any, only add to the count
        if (count >= BUFFERS) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((BUFFERS - 2) * PER + HALF) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        // where the next tile is: its rows are looked up while this one is multiplied (nothing here waits for memory: loads come in
        // order, so that would be waiting for all that is requested)
        const int next_id = id + step;
        const bool more = next_id < end;
        Place next = now;
        int found = 0;
        if (more) {
            next = place(next_id);
            found = look(next);
        }
        int buffer = 0, p = 0;
        // every wavefront has passed the last panel's barrier, behind which nothing of this tile is read: the next one is requested, and
        // comes while this one's results leave
        auto turn = [&]() {
            if (more) {
                aim(found);
                request_first();
            }
        };
        if (wm * 32 * TM < now.rows.n) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int c = 0; c < 16; ++c) acc[i][j][c] = 0.f;
            read(0, 0, 0);
            read_scales(0);
            turn_scales();
            for (; p + BUFFERS < count; ++p) buffer = panel(buffer, std::true_type{});
            request_rest(buffer);
            for (; p < count; ++p) buffer = panel(buffer, std::false_type{});
            turn();
            if (a.ytype == HLQ_F32) leave(now, float{});
            else if (a.ytype == HLQ_F16) leave(now, (_Float16)0.f);
            else leave(now, (__bf16)0.f);
        } else {   // none of this wavefront's rows is there: it only requests
            for (; p + BUFFERS < count; ++p) buffer = idle(buffer, std::true_type{});
            request_rest(buffer);
            for (; p < count; ++p) buffer = idle(buffer, std::false_type{});
            turn();
        }
        id = next_id;
        now = next;
    }
}

}  // namespace

hlq_status hlq_mx4_launch_big(const Mx4Product &a, const Mx4TilePlan &p, bool gated, hipStream_t st)
{
    const int64_t tiles = (int64_t)p.col_tiles * p.row_tiles;
    if (tiles > INT32_MAX / 2) return HLQ_ERR_UNSUPPORTED;
    auto kernel = gated ? hlq_mx4_big_kernel<true> : hlq_mx4_big_kernel<false>;
    kernel<<<256, 64 * WAVES, LDS, st>>>(a, p.col_tiles, p.row_tiles);
    return hlq_hip_status(hipGetLastError());
}
