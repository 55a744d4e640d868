// Products of MX4 matrices, dense and grouped by expert: argument checks, quantization of the activations, choice of the kernel.
#include "hlq_mx4_gemm.h"

namespace {

// rows up to which the kernel for few rows quantizes activations by itself
constexpr int64_t QUANTIZE_INSIDE = 16;
// rows of an expert (on average) up to which the kernel for few rows takes the product; only it can quantize inside
constexpr int FEW_ROWS = 16;

size_t up256(size_t n) { return (n + 255u) & ~(size_t)255u; }

// Launch of the tiled kernel for R rows of E experts, `width` rows of W each.
Mx4TilePlan tile_plan(int64_t width, int panels, int32_t E, int64_t R)
{
    Mx4TilePlan p{};
    const int64_t each = (R + E - 1) / E;   // rows of an expert, on average
    const int64_t wide = mx4_row_tiles(R, E, 128) * ((width + 255) / 256);
    p.BM = each > 64 ? 128 : each > 32 ? 64 : 32;
    p.BN = p.BM == 128 && wide >= 512 ? 256 : 128;
    p.col_tiles = (int)((width + p.BN - 1) / p.BN);
    p.row_tiles = (int)mx4_row_tiles(R, E, p.BM);
    const int64_t tiles = (int64_t)p.col_tiles * p.row_tiles, room = 512;
    p.splits = 1;
    p.share = panels;
    if (tiles > 0 && tiles * 2 <= room) {
        int splits = (int)(room / tiles);
        if (splits > panels / 4) splits = panels / 4;
        if (splits > 16) splits = 16;
        if (splits > 1) {
            p.share = (panels + splits - 1) / splits;
            p.splits = (panels + p.share - 1) / p.share;
        }
    }
    if (p.splits > 1) p.partial_bytes = (size_t)tiles * (size_t)p.splits * (size_t)p.BM * (size_t)p.BN * 4u;
    return p;
}

// rows of W that tiles of BN rows go over: gated halves are cut into 32 columns each
int64_t tiled_width(int64_t N, bool gated) { return gated ? (N / 2 + 31) / 32 * 64 : N; }

// counters, quantized activations, partial sums
size_t workspace_need(int64_t N, int32_t K, int32_t E, int64_t x_rows, int64_t R)
{
    Mx4Dims d;
    if (hlq_mx4_check(x_rows, K, &d) != HLQ_OK) return 0;
    size_t part = 0;
    for (int gated = 0; gated < 2; ++gated) {
        const size_t n = R ? tile_plan(tiled_width(N, gated), d.panels, E, R).partial_bytes : 0;
        if (n > part) part = n;
    }
    return HLQ_WS_COUNTER_BYTES + up256(d.total) + up256(part);
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
    a.y_aligned = ((uintptr_t)c.Y & 15u) == 0 && (R == 1 || c.ldy * hlq_dtype_bytes(c.ytype) % 16 == 0);
    int xtype = c.xtype;
    const bool few = R <= (int64_t)FEW_ROWS * E;
    hlq_clear_stale_error();
    if (xtype == HLQ_MX4) a.A = hlq_mx4_view(dx, c.X);
    else if (few && R <= QUANTIZE_INSIDE) {
        a.x = c.X;
        a.ldx = c.ldx;
        a.x_aligned = ((uintptr_t)c.X & 15u) == 0 && (c.x_rows == 1 || c.ldx * hlq_dtype_bytes(c.xtype) % 16 == 0);
    } else {
        if (!c.ws) return HLQ_ERR_NULL;
        if (c.ws_bytes < workspace_need(c.N, c.K, E, c.x_rows, R)) return HLQ_ERR_BUFFER_TOO_SMALL;
        if ((uintptr_t)c.ws & 15u) return HLQ_ERR_BAD_STRIDE;
        void *blob = (char *)c.ws + HLQ_WS_COUNTER_BYTES;
        s = hlq_mx4_launch_quantize(dx, c.X, c.xtype, c.ldx, blob, c.stream);
        if (s != HLQ_OK) return s;
        a.A = hlq_mx4_view(dx, blob);
        xtype = HLQ_MX4;
    }
    if (few) return hlq_mx4_launch_few(a, xtype, gated, c.stream);
    Mx4TilePlan p = tile_plan(tiled_width(c.N, gated), dw.panels, E, R);
    p.partial_at = HLQ_WS_COUNTER_BYTES + up256(dx.total);
    return hlq_mx4_launch_tile(a, p, gated, c.ws, c.stream);
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
    *bytes = workspace_need(N, K, experts, x_rows, rows);
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
