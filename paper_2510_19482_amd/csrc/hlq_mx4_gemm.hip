// Products of MX4 matrices, dense and grouped by expert: argument checks, quantization of the activations, choice of the kernel.
#include "hlq_mx4_gemm.h"

namespace {

// The kernel for few rows quantizes activations by itself where that is little work for each of its workgroups: rows of an
// expert (on average) times K up to QUANTIZE_INSIDE, and what 16 rows take of LDS.
constexpr int64_t QUANTIZE_INSIDE = 16384, QUANTIZED_BYTES = 65536;

size_t up256(size_t n) { return (n + 255u) & ~(size_t)255u; }

// Which kernel takes a product, by an estimate of its time (us) from measurements of its parts; mx4_few: rows and columns a
// wavefront, mx4_tile and mx4_big: of a workgroup.
//
// A start (2.9, tiled 3.1), then the longer of two.  First, what the busiest compute unit does.  Few rows: it loads the panels of its
// workgroups' rows and columns.  Tiled: a workgroup takes `alone` a panel where it has the unit for itself, `shared` where there are
// more, and `own` for its start and results (`search` more for experts, whose rows it looks up).  Second, memory: weights at 4.6 TB/s
// (experts' 5.1), tiled 5.3, an expert's again in part for a second row tile; results, taken as 16 bits, at 4.2.  Cutting K adds the hand-over of
// the partial sums: 1, and 3 for each 32 rows a wavefront has and four splits.
//
// Fitted to products that were each timed on every kernel (experts' rows 2 to 800 each, even and skewed; 17 to 16384 rows of one
// matrix).  On 420 others (profiles/mx4_plan_choice.txt) what is chosen is from the fastest on average: 2.7 % up to 1500 rows, 1.4 % above, 4.4 %
// for experts; at most 54 %, two rows each of 68 experts with K = 273.
// 256 x 256 against 128 x 256, measured, rows x N x K: 4096 x 4096 x 14336 107 / 116 (one round of the card), 8192 x 4096 x 4096 65 / 73
// (two), 8192 x 28672 x 4096 gated 440 / 485 (14), but half a round, 2048 x 4096 x 4096, 24 / 22.  Experts' rows, gated 4096 x 4096: 16384
// of 32 experts 180 / 193, 8192 of 8 85 / 92, 8192 of 64 133 / 169 (weights: 4.3 TB/s); against 32 x 128, 4096 of 64 117 / 181; 7686 of 126,
// 796 x 303 not gated, 22 / 12.
constexpr int MOST_SPLITS = 8, LEAST_SHARE = 4, MOST_CUT = 512;   // of K, panels of one, workgroups of a product whose K is cut
constexpr int share_of(int panels, int parts) { return (panels + parts - 1) / parts; }
constexpr bool may_cut(int panels) { return share_of(panels, 2) >= LEAST_SHARE; }   // where the workspace has to have room for partial sums
constexpr int64_t MOST_GROUPS = 1 << 22, MOST_TILES = 1 << 23;    // workgroups, so that a launch stays below 2^32 threads

struct Choice {
    int row_blocks, col_blocks;   // few rows, if row_blocks > 0
    Mx4TilePlan tile;
};

Choice choose(int64_t N, bool gated, int panels, int32_t E, int64_t R)
{
    const int64_t used = E < R ? E : R;                      // experts that have rows, at most
    const double each = (double)R / (double)used;
    auto row_tiles = [&](int BM) { return E == 1 ? (double)((R + BM - 1) / BM) : (double)used * (each <= 1.0 ? 1.0 : each / BM + 0.5 > 1.0 ? each / BM + 0.5 : 1.0); };
    const double weights = (double)used * (double)N * panels * 68.0 * 1e-6;   // MB; 1 TB/s is 1 MB a microsecond
    Choice best{};
    if (R <= 16) {   // whatever else there is reads as much
        best.row_blocks = best.col_blocks = 1;
        return best;
    }
    double least = 1e30;
    const double results = (double)R * (double)(gated ? N / 2 : N) * 2e-6 / 4.2;
    struct Few {
        int rows, cols;
        double load;   // bytes a nanosecond and compute unit
    };
    static const Few few[] = {{1, 1, 43}, {2, 1, 43}, {2, 2, 43}, {4, 2, 34}};
    for (const auto &k : few) {
        const int64_t cols = gated ? N / 2 : N, col_tiles = (cols + 16 * k.cols - 1) / (16 * k.cols);
        if (each > (E == 1 ? 600 : 64) || mx4_row_tiles(R, E, 16 * k.rows) * col_tiles > MOST_GROUPS) continue;   // above, no faster anywhere
        const double groups = row_tiles(16 * k.rows) * (double)col_tiles, rounds = groups < 1024 ? (double)(((int64_t)groups + 255) / 256) : groups / 256;
        const double loads = rounds * panels * 1.1 * (k.rows + k.cols * (gated ? 2 : 1)) / k.load, stream = weights / (E == 1 ? 4.6 : 5.1) + results;
        const double t = 2.9 + (loads > stream ? loads : stream);
        if (t < least) {
            least = t;
            best.row_blocks = k.rows;
            best.col_blocks = k.cols;
        }
    }
    struct Tile {
        int BM, BN, passes;   // passes: of four splits' partial sums; 0: K is not cut
        double alone, shared, own, search;
    };
    static const Tile tiles[] = {{32, 128, 1, 0.19, 0.12, 0.28, 0.55}, {64, 128, 2, 0.39, 0.204, 0.35, 1.0}, {128, 128, 2, 0.216, 0.211, 1.02, 1.7},
                                 {128, 256, 0, 0.57, 0.42, 1.41, 1.0}, {256, 256, 0, 0.70, 0.70, 4.0, 2.0}};
    const int64_t width = gated ? (N / 2 + 31) / 32 * 64 : N;   // gated halves are interleaved 32 columns at a time
    for (const auto &k : tiles) {
        const int64_t col_tiles = (width + k.BN - 1) / k.BN;
        if (mx4_row_tiles(R, E, k.BM) * col_tiles > MOST_TILES && k.BN < 256) continue;
        const double count = row_tiles(k.BM) * (double)col_tiles, own = k.own + (E > 1 ? k.search : 0.0);
        const double stream = weights / 5.3 * (E == 1 ? 1.0 : 0.52 + 0.48 * row_tiles(k.BM) / (double)used) + results;
        for (int want = 1; want <= (k.passes ? MOST_SPLITS : 1); want += want < 4 ? 1 : 2) {
            const int share = share_of(panels, want), splits = (panels + share - 1) / share;
            if (splits < want || (want > 1 && (!may_cut(panels) || mx4_row_tiles(R, E, k.BM) * col_tiles * want > MOST_CUT || share < LEAST_SHARE))) break;
            // workgroups, or tiles of 256 x 256, of a compute unit: whole rounds of the latter that are alike (an expert's last one, up to
            // half of them not even half filled, counts 0.58); of the former two where some units have two, later as units are free
            double full, most;
            if (k.BM == 256) {
                full = E == 1 ? (double)(((int64_t)count + 255) / 256) : (double)used * (each / 256 + 0.58) * (double)col_tiles / 256;
                most = full;
            } else {
                full = count * splits / 256;
                most = full < 2.0 ? 2.0 : full + 0.33;
            }
            double work = share * k.alone + own;
            if (full > 1.0 && most * (share * k.shared + own) > work) work = most * (share * k.shared + own);
            double t = 3.1 + (work > stream ? work : stream);
            if (splits > 1) t += 1.0 + 3.0 * k.passes * ((splits + 3) / 4);
            // as near where memory bounds both: larger tiles (gated 4096 x 4096, 24 rows each of 32 experts 51 / 54, of 64 not gated
            // 105 / 115), but for experts' fewest rows (16 each, not gated 4096 x 2048 30 / 27) and rows that do not fill them (64,
            // 28672 x 4096 13.7 / 12.7)
            if (t < least || (t == least && (E == 1 ? R >= k.BM : each > 16))) {
                least = t;
                best.row_blocks = 0;
                best.tile = Mx4TilePlan{k.BM, k.BN, (int)col_tiles, (int)mx4_row_tiles(R, E, k.BM), splits, share, 0, 0};
            }
        }
    }
    Mx4TilePlan &p = best.tile;
    if (best.row_blocks == 0 && p.splits > 1) p.partial_bytes = (size_t)p.row_tiles * (size_t)p.col_tiles * (size_t)p.splits * (size_t)p.BM * (size_t)p.BN * 4u;
    return best;
}

struct Plan {
    Choice how;
    bool inside;     // the kernel quantizes the activations
    size_t need;     // of workspace: counters, quantized activations, partial sums
};
Plan plan_of(int64_t N, int32_t K, bool gated, int32_t E, int64_t R, const Mx4Dims &dx, int xtype)
{
    Plan p;
    p.how = choose(N, gated, dx.panels, E, R);
    const bool quantize = xtype != HLQ_MX4;
    p.inside = quantize && p.how.row_blocks == 1 && (R + E - 1) / E * K <= QUANTIZE_INSIDE && (R < 16 ? R : 16) * (int64_t)dx.panels * 68 <= QUANTIZED_BYTES;
    p.how.tile.partial_at = HLQ_WS_COUNTER_BYTES + (quantize ? up256(dx.total) : 0u);
    p.need = p.how.tile.partial_at + up256(p.how.row_blocks ? 0 : p.how.tile.partial_bytes);
    return p;
}

struct Call {
    int64_t N;
    int32_t K;
    const void *W;
    int64_t x_rows;
    const void *X;
    hlq_dtype xtype;
    int64_t ldx;
    void *Y;
    hlq_dtype ytype;
    int64_t ldy;
    hlq_mx4_epilogue epilogue;
    void *ws;
    size_t ws_bytes;
    hipStream_t stream;
};

hlq_status product(const Call &c, int32_t E, const int32_t *offsets, const int32_t *rows, int64_t R)
{
    if (c.N < 1 || c.K < 1 || E < 1 || R < 0 || c.x_rows < 0) return HLQ_ERR_BAD_DESC;
    const bool gated = c.epilogue == HLQ_MX4_GATED;
    if (c.epilogue != HLQ_MX4_PLAIN && !gated) return HLQ_ERR_UNSUPPORTED;
    if (gated && c.N % 2) return HLQ_ERR_BAD_DESC;
    if (E > HLQ_MAX_EXPERTS || c.N > HLQ_MAX_N) return HLQ_ERR_UNSUPPORTED;
    if (!hlq_is_float(c.ytype) || (!hlq_is_float(c.xtype) && c.xtype != HLQ_MX4)) return HLQ_ERR_UNSUPPORTED;
    Mx4Dims dw, dx;
    hlq_status s = hlq_mx4_check((int64_t)E * c.N, c.K, &dw);
    if (s == HLQ_OK) s = hlq_mx4_check(c.x_rows, c.K, &dx);
    if (s != HLQ_OK) return s;
    if (R >= ((int64_t)1 << 31) - 256 || c.x_rows >= ((int64_t)1 << 31) - 256) return HLQ_ERR_UNSUPPORTED;
    const int64_t cols = gated ? c.N / 2 : c.N;
    if ((R > 1 && c.ldy < cols) || (c.xtype != HLQ_MX4 && c.x_rows > 1 && c.ldx < c.K)) return HLQ_ERR_BAD_STRIDE;
    if (R == 0) return HLQ_OK;
    if (c.x_rows == 0 || (!rows && c.x_rows < R)) return HLQ_ERR_BAD_DESC;   // rows to be computed, and none to read
    if (!c.W || !c.X || !c.Y) return HLQ_ERR_NULL;
    if (((uintptr_t)c.W & 15u) || (c.xtype == HLQ_MX4 && ((uintptr_t)c.X & 15u)) || (uintptr_t)c.Y % (unsigned)hlq_dtype_bytes(c.ytype) ||
        (c.xtype != HLQ_MX4 && (uintptr_t)c.X % (unsigned)hlq_dtype_bytes(c.xtype)) || ((uintptr_t)offsets & 3u) || ((uintptr_t)rows & 3u))
        return HLQ_ERR_BAD_STRIDE;

    Mx4Product a{};
    a.W = hlq_mx4_view(dw, c.W);
    a.N = (int)c.N;
    a.cols = (int)cols;
    a.K = c.K;
    a.panels = dw.panels;
    a.offsets = offsets;
    a.E = E;
    a.rows = rows;
    a.R = (int)R;
    a.x_rows = (int)c.x_rows;
    a.y = c.Y;
    a.ytype = c.ytype;
    a.ldy = c.ldy;
    const Plan p = plan_of(c.N, c.K, gated, E, R, dx, c.xtype);
    const Choice &how = p.how;
    if (!c.ws) return HLQ_ERR_NULL;
    if (c.ws_bytes < p.need) return HLQ_ERR_BUFFER_TOO_SMALL;
    if ((uintptr_t)c.ws & 15u) return HLQ_ERR_BAD_STRIDE;
    hlq_clear_stale_error();
    if (c.xtype == HLQ_MX4) a.A = hlq_mx4_view(dx, c.X);
    else if (p.inside) {
        a.x = c.X;
        a.ldx = c.ldx;
        return hlq_mx4_launch_few(a, c.xtype, gated, 1, 1, c.stream);
    } else {
        void *blob = (char *)c.ws + HLQ_WS_COUNTER_BYTES;
        s = hlq_mx4_launch_quantize(dx, c.X, c.xtype, c.ldx, blob, c.stream);
        if (s != HLQ_OK) return s;
        a.A = hlq_mx4_view(dx, blob);
    }
    if (how.row_blocks) return hlq_mx4_launch_few(a, HLQ_MX4, gated, how.row_blocks, how.col_blocks, c.stream);
    if (how.tile.BM == 256) return hlq_mx4_launch_big(a, how.tile, gated, c.stream);
    return hlq_mx4_launch_tile(a, how.tile, gated, c.ws, c.stream);
}

}  // namespace

extern "C" {

hlq_status hlq_mx4_workspace_bytes(int64_t N, int32_t K, int32_t experts, int64_t x_rows, int64_t rows, size_t *bytes)
{
    Mx4Dims d;
    if (N < 1 || experts < 1 || rows < 0) return HLQ_ERR_BAD_DESC;
    hlq_status s = hlq_mx4_check(x_rows, K, &d);
    if (s != HLQ_OK) return s;
    if (!bytes) return HLQ_ERR_NULL;
    // partial sums: a bound that grows with the rows, so that fewer rows never need more
    size_t part = 0;
    if (may_cut(d.panels) && rows > 0) {
        const size_t used = (size_t)(rows < experts ? rows : experts);
        part = ((size_t)rows + used * 128u) * (size_t)(up256((size_t)N) + 256u) * (size_t)MOST_SPLITS * 4u;
        const size_t most = (size_t)MOST_CUT * 128u * 128u * 4u;
        if (part > most) part = most;
    }
    *bytes = HLQ_WS_COUNTER_BYTES + up256(d.total) + up256(part);
    return HLQ_OK;
}

hlq_status hlq_mx4_plan_query(int64_t N, int32_t K, int32_t experts, int64_t x_rows, int64_t rows, hlq_dtype xtype, hlq_mx4_epilogue epilogue, hlq_mx4_plan_info *out)
{
    const bool gated = epilogue == HLQ_MX4_GATED;
    if (N < 1 || experts < 1 || rows < 1 || (gated && N % 2)) return HLQ_ERR_BAD_DESC;
    if ((epilogue != HLQ_MX4_PLAIN && !gated) || experts > HLQ_MAX_EXPERTS || N > HLQ_MAX_N || rows >= ((int64_t)1 << 31) - 256 ||
        (!hlq_is_float(xtype) && xtype != HLQ_MX4))
        return HLQ_ERR_UNSUPPORTED;
    Mx4Dims d;
    const hlq_status s = hlq_mx4_check(x_rows, K, &d);
    if (s != HLQ_OK) return s;
    if (!out) return HLQ_ERR_NULL;
    const Plan p = plan_of(N, K, gated, experts, rows, d, xtype);
    *out = hlq_mx4_plan_info{};
    out->workspace_bytes = (int64_t)p.need;
    out->quantizes = p.inside;
    if (p.how.row_blocks) {
        const Mx4FewShape f = hlq_mx4_few_shape((int)(gated ? N / 2 : N), K, d.panels, experts, rows, p.inside ? xtype : HLQ_MX4, p.how.row_blocks, p.how.col_blocks);
        out->kernel = 1;
        out->tile_rows = 16 * p.how.row_blocks;
        out->tile_cols = 16 * p.how.col_blocks;
        out->k_parts = f.share;
        return HLQ_OK;
    }
    const Mx4TilePlan &t = p.how.tile;
    out->kernel = t.BM == 256 ? 3 : 2;
    out->tile_rows = t.BM;
    out->tile_cols = t.BN;
    out->k_parts = t.splits;
    return HLQ_OK;
}

hlq_status hlq_mx4_gemm(int64_t N, int32_t K, const void *W, int64_t M, const void *X, hlq_dtype xtype, int64_t ldx, void *Y,
                        hlq_dtype ytype, int64_t ldy, hlq_mx4_epilogue epilogue, void *ws, size_t ws_bytes, void *stream)
{
    return product(Call{N, K, W, M, X, xtype, ldx, Y, ytype, ldy, epilogue, ws, ws_bytes, (hipStream_t)stream}, 1, nullptr, nullptr, M);
}

hlq_status hlq_expert_gemm(int32_t experts, int64_t N, int32_t K, const void *W, const int32_t *offsets, const int32_t *rows, int64_t R,
                           int64_t x_rows, const void *X, hlq_dtype xtype, int64_t ldx, void *Y, hlq_dtype ytype, int64_t ldy,
                           hlq_mx4_epilogue epilogue, void *ws, size_t ws_bytes, void *stream)
{
    if (!offsets) return HLQ_ERR_NULL;
    return product(Call{N, K, W, x_rows, X, xtype, ldx, Y, ytype, ldy, epilogue, ws, ws_bytes, (hipStream_t)stream}, experts, offsets, rows, R);
}

}  // extern "C"
