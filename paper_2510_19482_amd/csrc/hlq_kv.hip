// Rotary positions, and rows into and out of the paged cache of keys and values.
//
//   turned pair   (a, b) -> m (a cos - b sin, b cos + a sin),  angle = position * frequency
//   8 or 4 bits   per 32 values e = max(floor(log2(max |x|)) - 8 or 2, -127), a value the code nearest to x 2^-e
//
// An angle is kept in turns, as a fraction of 64 bits: position times frequency is one integer product whose overflow drops whole turns,
// so far positions lose nothing.  Sine and cosine are Taylor polynomials in 64 bits over an eighth of a turn to either side, the turn of a pair is
// taken in 64 bits too: the memory hides it, and a result that lies next to a border of a 4-bit code falls on the right side.
//
// Lanes: eight successive values of a head each, so that a head is dim / 8 lanes of one wavefront and four lanes are a block of 32.  A wavefront has a
// token and goes through heads of it, queries, keys, then values; the angles of its lanes stay in registers.
//
// What bounds them: memory.  8192 tokens of 40 f16 heads turned 29 us (168 MB, 5.8 TB/s); the same with 8 heads of values into 4 bits 42 us (200 MB, 4.8 TB/s); 65536 tokens
// read from 4 bits 54 us (340 MB, 6.2 TB/s), from 16 bits 90.  A step of 32 tokens takes 4.5 to 4.8 us, of which a launch and three dependent loads are most; 77 tokens read 2.8.
#include "hlq_kv.h"

namespace {

constexpr int WAVES = 4;

struct Rows {
    int64_t T;
    int parts, per_part;         // a token's heads are cut over wavefronts
    int D, lanes, fit;           // lanes of a head, heads that a wavefront has at once
    int q_heads, kv_heads;
    int dims, half, interleaved, whole;   // whole: a lane's eight values are all of one half, or behind both
    double magnitude;
    const uint64_t *turns;
    const int32_t *positions;
    const int64_t *slots;
    KvRows q, q_out, k, k_out, v;
    KvView kv;
};

// sine and cosine of a fraction of a turn, times m
__device__ __forceinline__ void sine_of(uint64_t turn, double m, double &s, double &c)
{
    const uint32_t quarter = (uint32_t)((turn + ((uint64_t)1 << 61)) >> 62);
    const int64_t rest = (int64_t)(turn - ((uint64_t)quarter << 62));       // an eighth of a turn to either side
    const double x = (double)rest * 3.4061215800865545e-19, z = x * x;      // 2 pi / 2^64
    // z^n / (2 n + 1)! and z^n / (2 n)!, signs in turn; what is left out is below 5e-17 and 2e-18 at pi / 4
    double a = -1. / 1307674368000.;
    a = fma(a, z, 1. / 6227020800.);
    a = fma(a, z, -1. / 39916800.);
    a = fma(a, z, 1. / 362880.);
    a = fma(a, z, -1. / 5040.);
    a = fma(a, z, 1. / 120.);
    a = fma(a, z, -1. / 6.);
    a = fma(a * z, x, x) * m;
    double b = 1. / 20922789888000.;
    b = fma(b, z, -1. / 87178291200.);
    b = fma(b, z, 1. / 479001600.);
    b = fma(b, z, -1. / 3628800.);
    b = fma(b, z, 1. / 40320.);
    b = fma(b, z, -1. / 720.);
    b = fma(b, z, 1. / 24.);
    b = fma(b, z, -.5);
    b = fma(b, z, 1.) * m;
    s = quarter & 1 ? b : a;
    c = quarter & 1 ? a : b;
    if (quarter & 2) s = -s;
    if (quarter == 1 || quarter == 2) c = -c;
}

// scale byte of a block of e4m3 values, whose largest exponent is 8; as mx4_scale_of
__device__ __forceinline__ uint32_t mx8_scale_of(uint32_t top)
{
    const uint32_t e = top >> 23;
    return e == 255u ? 255u : e > 8u ? e - 8u : 0u;
}
// e4m3 codes of eight values under a scale byte: to nearest, ties to the even code, above 448 it is 448
template <class V>
__device__ __forceinline__ mx4_u2 mx8_codes(const V (&v)[8], uint32_t byte)
{
    const float up = __builtin_bit_cast(float, byte == 255u ? 0u : (254u - byte) << 23);   // 2^(127 - byte); finite blocks have bytes up to 246
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __builtin_amdgcn_fmed3f((float)v[i] * up, -448.f, 448.f);
    mx4_u2 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i], x[4 * i + 1], 0, false);
        r[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2], x[4 * i + 3], w, true);
    }
    return r;
}

// Eight values of a row, in the cache.  Four lanes next to each other have a block.
template <int C, class V>
__device__ __forceinline__ void put(const KvView &kv, int64_t slot, int what, int h, int chunk, const V (&v)[8])
{
    const int64_t page = slot >> kv.log_page;
    const int at = (int)(slot & ((1 << kv.log_page) - 1));
    uint8_t *row = kv.rows(page, what, h) + (int64_t)at * kv.row_bytes;
    if constexpr (C == HLQ_MX4 || C == HLQ_MX8) {
        const uint32_t top = mx4_quad_max(mx4_top_bits(v)), byte = C == HLQ_MX8 ? mx8_scale_of(top) : mx4_scale_of(top);
        if constexpr (C == HLQ_MX4) {
            V w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = v[i];
            *(uint32_t *)(row + chunk * 4) = mx4_codes(w, byte);
        }
        else *(mx4_u2 *)(row + chunk * 8) = mx8_codes(v, byte);
        if ((chunk & 3) == 0) kv.bytes(page, what, h)[((chunk >> 2) << kv.log_page) + at] = (uint8_t)byte;
    } else {
        using S = typename KvType<C>::type;
        typename Mx4Eight<S>::Values e;
#pragma unroll
        for (int i = 0; i < 8; ++i) e.v[i] = (S)(float)v[i];
        *(mx4_u4 *)(row + chunk * 16) = __builtin_bit_cast(typename Mx4Eight<S>::Raw, e).r[0];
    }
}

// past the caches: 65536 tokens read from 4 bits 77 -> 54 us, 8192 turned 42 -> 30
template <class V>
__device__ __forceinline__ void store_eight(const V (&v)[8], V *p)
{
    using E = Mx4Eight<V>;
    typename E::Values e;
#pragma unroll
    for (int i = 0; i < 8; ++i) e.v[i] = v[i];
    const typename E::Raw raw = __builtin_bit_cast(typename E::Raw, e);
#pragma unroll
    for (int i = 0; i < E::N; ++i) __builtin_nontemporal_store(raw.r[i], (mx4_u4_any *)(p + i * 8 / E::N));
}

constexpr int NO_CACHE = -1;

// C: the cache's type, or none
template <int T, int C>
__global__ void __launch_bounds__(64 * WAVES)
hlq_kv_rows_kernel(const Rows a)
{
    using V = typename Mx4Type<T>::type;
    const int lane = (int)(threadIdx.x & 63u), sub = lane / a.lanes, chunk = lane - sub * a.lanes, d0 = chunk * 8;
    const int64_t item = (int64_t)blockIdx.x * WAVES + (threadIdx.x >> 6), t = item / a.parts;
    if (t >= a.T) return;
    const int part = (int)(item - t * a.parts), first = part * a.per_part;
    const int all = a.q_heads + (C == NO_CACHE ? 0 : 2 * a.kv_heads), end = first + a.per_part < all ? first + a.per_part : all;

    // A lane has the angle of a pair or two, by way of LDS each lane has sine (its sign that of the partner's part) and cosine of its own values.
    double sine[8], cosine[8];
    const bool turn = a.dims > 0 && first < a.q_heads + (C == NO_CACHE ? 0 : a.kv_heads);
    if (turn) {
        struct alignas(16) Angle { double s, c; };
        __shared__ Angle angles[WAVES][KV_MOST_DIM / 2];
        Angle *const mine = angles[threadIdx.x >> 6];
        const auto place = [](int pair) { return (pair & 7) * (KV_MOST_DIM / 16) + (pair >> 3); };   // so that lanes read what stands side by side
        const uint64_t at = (uint64_t)(int64_t)a.positions[t];
        for (int pair = lane; pair < a.half; pair += 64) {
            Angle x;
            sine_of(at * a.turns[pair], a.magnitude, x.s, x.c);
            mine[place(pair)] = x;
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");   // the lanes of a wavefront read what others of it wrote
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int d = d0 + i;
            sine[i] = 0, cosine[i] = 1;
            if (d < a.dims) {
                const Angle x = mine[place(a.interleaved ? d >> 1 : d < a.half ? d : d - a.half)];
                sine[i] = (a.interleaved ? (d & 1) == 0 : d < a.half) ? -x.s : x.s;
                cosine[i] = x.c;
            }
        }
    }
    if (sub >= a.fit) return;
    int64_t slot = -1;
    if constexpr (C != NO_CACHE) {
        slot = a.slots[t];
        if (slot < 0 || slot >= a.kv.pages << a.kv.log_page) slot = -1;
    }
    const int partner = 4 * (d0 < a.half ? lane + a.half / 8 : lane - a.half / 8);   // the lane that has the other halves of this one's pairs
    auto row_of = [&](int h) {
        const bool is_q = h < a.q_heads, is_v = h >= a.q_heads + a.kv_heads;
        const KvRows &from = is_q ? a.q : is_v ? a.v : a.k;
        return (const V *)from.p + t * from.ts + (is_q ? h : is_v ? h - a.q_heads - a.kv_heads : h - a.q_heads) * from.hs;
    };
    // Six heads' values (two of f32) are on their way at a time: 8192 tokens of 40 heads 37 us with four, 46 with one.
    constexpr int BATCH = sizeof(V) == 2 ? 6 : 2;
    for (int h0 = first + sub; h0 < end; h0 += BATCH * a.fit) {
        V every[BATCH][8];
#pragma unroll
        for (int n = 0; n < BATCH; ++n)
            if (h0 + n * a.fit < end) mx4_read8<false>(row_of(h0 + n * a.fit) + d0, every[n]);
#pragma unroll
        for (int n = 0; n < BATCH; ++n) {
            const int h = h0 + n * a.fit;
            if (h >= end) break;
            V (&v)[8] = every[n];
            const bool is_q = h < a.q_heads, is_v = h >= a.q_heads + a.kv_heads;
            const int own_h = is_q ? h : is_v ? h - a.q_heads - a.kv_heads : h - a.q_heads;
            if (turn && !is_v) {
                V other[8];
                if (a.interleaved) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) other[i] = v[i ^ 1];
                } else if (a.whole) {
                    using E = Mx4Eight<V>;
                    typename E::Values e;
#pragma unroll
                    for (int i = 0; i < 8; ++i) e.v[i] = v[i];
                    typename E::Raw raw = __builtin_bit_cast(typename E::Raw, e);
#pragma unroll
                    for (int i = 0; i < E::N; ++i)
#pragma unroll
                        for (int w = 0; w < 4; ++w) raw.r[i][w] = (uint32_t)__builtin_amdgcn_ds_bpermute(partner, (int)raw.r[i][w]);
                    e = __builtin_bit_cast(typename E::Values, raw);
#pragma unroll
                    for (int i = 0; i < 8; ++i) other[i] = e.v[i];
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int d = d0 + i;
                        other[i] = d >= a.dims ? v[i] : row_of(h)[d < a.half ? d + a.half : d - a.half];
                    }
                }
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (d0 + i < a.dims) {
                        float y = (float)fma((double)(float)other[i], sine[i], (double)(float)v[i] * cosine[i]);
                        asm("" : "+v"(y));   // by way of f32: from 64 to 16 bits in one step the compiler has ten instructions
                        v[i] = (V)y;
                    }
            }
            if (is_q || (!is_v && a.k_out.p)) {
                const KvRows &to = is_q ? a.q_out : a.k_out;
                store_eight(v, (V *)to.p + t * to.ts + own_h * to.hs + d0);
            }
            if constexpr (C != NO_CACHE)
                if (!is_q && slot >= 0) put<C>(a.kv, slot, is_v ? 1 : 0, own_h, chunk, v);
        }
    }
}

struct Read {
    int64_t T;
    int parts, per_part, lanes, fit, H, first;   // heads of the keys, then of the values; first: where they begin
    const int64_t *slots;
    KvRows k, v;
    KvView kv;
};

template <int T, int C>
__global__ void __launch_bounds__(64 * WAVES)
hlq_kv_read_kernel(const Read a)
{
    using V = typename Mx4Type<T>::type;
    const int lane = (int)(threadIdx.x & 63u), sub = lane / a.lanes, chunk = lane - sub * a.lanes;
    const int64_t item = (int64_t)blockIdx.x * WAVES + (threadIdx.x >> 6), t = item / a.parts;
    if (t >= a.T || sub >= a.fit) return;
    const int64_t slot = a.slots[t];
    if (slot < 0 || slot >= a.kv.pages << a.kv.log_page) return;
    const int64_t page = slot >> a.kv.log_page;
    const int at = (int)(slot & ((1 << a.kv.log_page) - 1));
    const int first = a.first + (int)(item - t * a.parts) * a.per_part, all = a.first + (a.k.p ? a.H : 0) + (a.v.p ? a.H : 0);
    const int end = first + a.per_part < all ? first + a.per_part : all;
    for (int h = first + sub; h < end; h += a.fit) {
        const int what = h >= a.H, own_h = what ? h - a.H : h;
        const uint8_t *row = a.kv.rows(page, what, own_h) + (int64_t)at * a.kv.row_bytes;
        const KvRows &to = what ? a.v : a.k;
        V v[8];
        if constexpr (C == HLQ_MX4 || C == HLQ_MX8) {
            const int byte = a.kv.bytes(page, what, own_h)[((chunk >> 2) << a.kv.log_page) + at];
            // values without their scale, exact; then the scale in two steps where one power of two is no normal number
            float f[8];
            if constexpr (C == HLQ_MX4) {
                const uint32_t c = *(const uint32_t *)(row + chunk * 4);
                const auto p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 1);
                const auto p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 3);
                f[0] = p0[0], f[1] = p0[1], f[2] = p1[0], f[3] = p1[1], f[4] = p2[0], f[5] = p2[1], f[6] = p3[0], f[7] = p3[1];
            } else {
                const mx4_u2 c = *(const mx4_u2 *)(row + chunk * 8);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i], true);
                    f[4 * i] = lo[0], f[4 * i + 1] = lo[1], f[4 * i + 2] = hi[0], f[4 * i + 3] = hi[1];
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (V)(byte == 255 ? __builtin_nanf("") : ldexpf(f[i], byte - 127));
        } else {
            typename Mx4Eight<typename KvType<C>::type>::Raw raw;
            raw.r[0] = *(const mx4_u4 *)(row + chunk * 16);
            const auto e = __builtin_bit_cast(typename Mx4Eight<typename KvType<C>::type>::Values, raw);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (V)(float)e.v[i];
        }
        store_eight(v, (V *)to.p + t * to.ts + own_h * to.hs + chunk * 8);
    }
}

// A token's heads on one wavefront, so that its angles are made once, unless that leaves the card half empty: then on several.  (1024 tokens of 48 heads into 16 bits and back:
// 2048 wavefronts 11.6 us, 4096 10.0, 16384 15.0; 8192 tokens of 40 heads turned: one a token 31, two 35, four 45.)
void cut_heads(int64_t T, int all, int fit, int &parts, int &per_part)
{
    const int rounds = (all + fit - 1) / fit;
    int64_t want = T > 0 ? (4096 + T - 1) / T : 1;
    if (want > rounds) want = rounds;
    per_part = (int)((rounds + want - 1) / want) * fit;
    parts = (all + per_part - 1) / per_part;
}

// A launch has fewer than 2^32 lanes: the tokens of one, and its grid.
int64_t tokens_of_launch(int parts) { return (((int64_t)1 << 32) / (64 * WAVES) - 1) * WAVES / parts; }
dim3 grid_of(int64_t T, int parts) { return dim3((unsigned)((T * parts + WAVES - 1) / WAVES)); }

KvRows behind(const KvRows &x, int64_t tokens, int bytes) { return KvRows{x.p ? (char *)x.p + tokens * x.ts * bytes : nullptr, x.ts, x.hs}; }

template <int T>
void launch_rows(const Rows &a, int cache, dim3 grid, hipStream_t st)
{
    const dim3 block(64 * WAVES);
    switch (cache) {
    case HLQ_F16: hlq_kv_rows_kernel<T, HLQ_F16><<<grid, block, 0, st>>>(a); break;
    case HLQ_BF16: hlq_kv_rows_kernel<T, HLQ_BF16><<<grid, block, 0, st>>>(a); break;
    case HLQ_MX8: hlq_kv_rows_kernel<T, HLQ_MX8><<<grid, block, 0, st>>>(a); break;
    case HLQ_MX4: hlq_kv_rows_kernel<T, HLQ_MX4><<<grid, block, 0, st>>>(a); break;
    default: hlq_kv_rows_kernel<T, NO_CACHE><<<grid, block, 0, st>>>(a); break;
    }
}
template <int T>
void launch_read(const Read &a, int cache, dim3 grid, hipStream_t st)
{
    const dim3 block(64 * WAVES);
    switch (cache) {
    case HLQ_F16: hlq_kv_read_kernel<T, HLQ_F16><<<grid, block, 0, st>>>(a); break;
    case HLQ_BF16: hlq_kv_read_kernel<T, HLQ_BF16><<<grid, block, 0, st>>>(a); break;
    case HLQ_MX8: hlq_kv_read_kernel<T, HLQ_MX8><<<grid, block, 0, st>>>(a); break;
    default: hlq_kv_read_kernel<T, HLQ_MX4><<<grid, block, 0, st>>>(a); break;
    }
}

hlq_status check_sizes(int64_t T, int32_t heads, int32_t dim)
{
    if (T < 0 || heads < 1 || dim < 8 || dim % 8) return HLQ_ERR_BAD_DESC;
    return T >= (int64_t)1 << 31 || heads > KV_MOST_HEADS || dim > KV_MOST_DIM ? HLQ_ERR_UNSUPPORTED : HLQ_OK;
}
hlq_status check_rotary(const hlq_rotary_desc *r, int dim, int64_t T, const int32_t *positions)
{
    if (!r) return HLQ_ERR_NULL;
    if (r->dims < 2 || r->dims % 2 || r->dims > dim) return HLQ_ERR_BAD_DESC;
    if (T > 0 && (!r->turns || !positions)) return HLQ_ERR_NULL;
    return (uintptr_t)r->turns & 7u || (uintptr_t)positions & 3u ? HLQ_ERR_BAD_STRIDE : HLQ_OK;
}
void take_rotary(Rows &a, const hlq_rotary_desc *r, const int32_t *positions)
{
    a.dims = r->dims;
    a.half = r->dims / 2;
    a.interleaved = r->interleaved != 0;
    a.whole = a.interleaved ? r->dims % 8 == 0 : a.half % 8 == 0;
    a.magnitude = r->magnitude;
    a.turns = r->turns;
    a.positions = positions;
}
hlq_status check_cache(const hlq_kv_desc *c, const void *cache, size_t cache_bytes, KvDims *d)
{
    const hlq_status s = hlq_kv_check(c, d);
    if (s != HLQ_OK) return s;
    if (!cache) return HLQ_ERR_NULL;
    if ((uintptr_t)cache & 15u) return HLQ_ERR_BAD_STRIDE;
    return cache_bytes < d->total ? HLQ_ERR_BUFFER_TOO_SMALL : HLQ_OK;
}
hlq_status go(Rows &a, int all, int type, int cache, void *stream)
{
    a.lanes = a.D / 8;
    a.fit = 64 / a.lanes;
    cut_heads(a.T, all, a.fit, a.parts, a.per_part);
    const int64_t each = tokens_of_launch(a.parts);
    const int bytes = hlq_dtype_bytes((hlq_dtype)type);
    const hipStream_t st = (hipStream_t)stream;
    hlq_clear_stale_error();
    for (int64_t t = 0; t < a.T; t += each) {
        Rows b = a;
        b.T = a.T - t < each ? a.T - t : each;
        b.q = behind(a.q, t, bytes), b.q_out = behind(a.q_out, t, bytes), b.k = behind(a.k, t, bytes), b.k_out = behind(a.k_out, t, bytes), b.v = behind(a.v, t, bytes);
        if (a.positions) b.positions = a.positions + t;
        if (a.slots) b.slots = a.slots + t;
        const dim3 grid = grid_of(b.T, b.parts);
        if (type == HLQ_F16) launch_rows<HLQ_F16>(b, cache, grid, st);
        else if (type == HLQ_BF16) launch_rows<HLQ_BF16>(b, cache, grid, st);
        else launch_rows<HLQ_F32>(b, cache, grid, st);
    }
    return hlq_hip_status(hipGetLastError());
}

}  // namespace

hlq_status hlq_kv_check(const hlq_kv_desc *c, KvDims *out)
{
    if (!c) return HLQ_ERR_NULL;
    const bool mx = c->type == HLQ_MX8 || c->type == HLQ_MX4;
    if (c->type != HLQ_F16 && c->type != HLQ_BF16 && !mx) return HLQ_ERR_UNSUPPORTED;
    const int p = c->page_tokens;
    if (c->pages < 1 || p < 16 || p > 1024 || (p & (p - 1)) || c->heads < 1 || c->dim < 8 || c->dim % (mx ? KV_BLOCK : 8)) return HLQ_ERR_BAD_DESC;
    if (c->pages >= (int64_t)1 << 31 || c->heads > KV_MOST_HEADS || c->dim > KV_MOST_DIM) return HLQ_ERR_UNSUPPORTED;
    KvDims d{};
    d.pages = c->pages;
    d.H = c->heads;
    d.D = c->dim;
    d.type = c->type;
    d.log_page = __builtin_ctz((unsigned)p);
    d.row_bytes = c->type == HLQ_MX4 ? c->dim / 2 : c->type == HLQ_MX8 ? c->dim : 2 * c->dim;
    d.blocks = mx ? c->dim / KV_BLOCK : 0;
    const size_t rows = (size_t)c->pages * 2u * (size_t)c->heads * (size_t)p;   // below 2^52
    d.code_bytes = rows * (size_t)d.row_bytes;
    d.total = d.code_bytes + rows * (size_t)d.blocks;
    *out = d;
    return HLQ_OK;
}

extern "C" {

hlq_status hlq_kv_bytes(const hlq_kv_desc *c, size_t *bytes)
{
    KvDims d;
    const hlq_status s = hlq_kv_check(c, &d);
    if (s != HLQ_OK) return s;
    if (!bytes) return HLQ_ERR_NULL;
    *bytes = d.total;
    return HLQ_OK;
}

hlq_status hlq_rotary_turns(int32_t pairs, const double *frequencies, uint64_t *turns)
{
    if (pairs < 1 || pairs > KV_MOST_DIM / 2) return HLQ_ERR_BAD_DESC;
    if (!frequencies || !turns) return HLQ_ERR_NULL;
    for (int i = 0; i < pairs; ++i)
        if (!(fabs(frequencies[i]) < 4294967296.)) return HLQ_ERR_BAD_DESC;
    for (int i = 0; i < pairs; ++i) {
        long double f = (long double)frequencies[i] / 6.28318530717958647692528676655900577L;
        f -= floorl(f);
        const long double n = roundl(f * 18446744073709551616.L);
        turns[i] = n >= 18446744073709551616.L ? 0u : (uint64_t)n;
    }
    return HLQ_OK;
}

hlq_status hlq_rotary(const hlq_rotary_desc *r, int64_t T, int32_t heads, int32_t dim, hlq_dtype type, const int32_t *positions, const void *x, int64_t x_ts,
                      int64_t x_hs, void *y, int64_t y_ts, int64_t y_hs, void *stream)
{
    hlq_status s = check_sizes(T, heads, dim);
    if (s != HLQ_OK) return s;
    if (!hlq_is_float(type)) return HLQ_ERR_UNSUPPORTED;
    if ((s = check_rotary(r, dim, T, positions)) != HLQ_OK) return s;
    if (T == 0) return HLQ_OK;
    if ((s = hlq_check_rows(x, T, heads, dim, x_ts, x_hs, type, false)) != HLQ_OK) return s;
    if ((s = hlq_check_rows(y, T, heads, dim, y_ts, y_hs, type, true)) != HLQ_OK) return s;
    if (hlq_rows_in_the_way(hlq_span(x, T, heads, x_ts, x_hs, type), hlq_span(y, T, heads, y_ts, y_hs, type), dim)) return HLQ_ERR_BAD_STRIDE;
    Rows a{};
    a.T = T;
    a.D = dim;
    a.q_heads = heads;
    a.q = KvRows{const_cast<void *>(x), x_ts, x_hs};
    a.q_out = KvRows{y, y_ts, y_hs};
    take_rotary(a, r, positions);
    return go(a, heads, type, NO_CACHE, stream);
}

hlq_status hlq_kv_write(const hlq_kv_desc *c, void *cache, size_t cache_bytes, int64_t T, hlq_dtype type, const void *k, int64_t k_ts, int64_t k_hs,
                        const void *v, int64_t v_ts, int64_t v_hs, const int64_t *slots, const hlq_rotary_desc *r, const int32_t *positions, void *k_out,
                        int64_t ko_ts, int64_t ko_hs, int32_t q_heads, const void *q, int64_t q_ts, int64_t q_hs, void *q_out, int64_t qo_ts, int64_t qo_hs,
                        void *stream)
{
    KvDims d;
    hlq_status s = check_cache(c, cache, cache_bytes, &d);
    if (s != HLQ_OK) return s;
    if ((s = check_sizes(T, d.H, d.D)) != HLQ_OK) return s;
    if (!hlq_is_float(type) || q_heads > KV_MOST_HEADS) return HLQ_ERR_UNSUPPORTED;
    if (q_heads < 0 || (!r && (q_heads > 0 || k_out))) return HLQ_ERR_BAD_DESC;
    if (r && (s = check_rotary(r, d.D, T, positions)) != HLQ_OK) return s;
    if (T == 0) return HLQ_OK;
    if (!slots) return HLQ_ERR_NULL;
    if ((uintptr_t)slots & 7u) return HLQ_ERR_BAD_STRIDE;
    if ((s = hlq_check_rows(k, T, d.H, d.D, k_ts, k_hs, type, false)) != HLQ_OK) return s;
    if ((s = hlq_check_rows(v, T, d.H, d.D, v_ts, v_hs, type, false)) != HLQ_OK) return s;
    if (k_out && (s = hlq_check_rows(k_out, T, d.H, d.D, ko_ts, ko_hs, type, true)) != HLQ_OK) return s;
    if (q_heads > 0) {
        if ((s = hlq_check_rows(q, T, q_heads, d.D, q_ts, q_hs, type, false)) != HLQ_OK) return s;
        if ((s = hlq_check_rows(q_out, T, q_heads, d.D, qo_ts, qo_hs, type, true)) != HLQ_OK) return s;
    }
    const KvSpan ki = hlq_span(k, T, d.H, k_ts, k_hs, type), vi = hlq_span(v, T, d.H, v_ts, v_hs, type), ko = hlq_span(k_out, T, d.H, ko_ts, ko_hs, type);
    const KvSpan qi = hlq_span(q_heads > 0 ? q : nullptr, T, q_heads, q_ts, q_hs, type), qo = hlq_span(q_heads > 0 ? q_out : nullptr, T, q_heads, qo_ts, qo_hs, type);
    if (hlq_rows_in_the_way(ki, ko, d.D) || hlq_rows_in_the_way(qi, qo, d.D) || hlq_rows_overlap(vi, ko, d.D) || hlq_rows_overlap(qi, ko, d.D) || hlq_rows_overlap(ki, qo, d.D) ||
        hlq_rows_overlap(vi, qo, d.D) || hlq_rows_overlap(ko, qo, d.D))
        return HLQ_ERR_BAD_STRIDE;
    Rows a{};
    a.T = T;
    a.D = d.D;
    a.q_heads = q_heads;
    a.kv_heads = d.H;
    a.slots = slots;
    a.q = KvRows{const_cast<void *>(q), q_ts, q_hs};
    a.q_out = KvRows{q_out, qo_ts, qo_hs};
    a.k = KvRows{const_cast<void *>(k), k_ts, k_hs};
    a.k_out = KvRows{k_out, ko_ts, ko_hs};
    a.v = KvRows{const_cast<void *>(v), v_ts, v_hs};
    a.kv = hlq_kv_view(d, cache);
    if (r) take_rotary(a, r, positions);
    return go(a, q_heads + 2 * d.H, type, d.type, stream);
}

hlq_status hlq_kv_read(const hlq_kv_desc *c, const void *cache, size_t cache_bytes, int64_t T, const int64_t *slots, hlq_dtype type, void *k, int64_t k_ts,
                       int64_t k_hs, void *v, int64_t v_ts, int64_t v_hs, void *stream)
{
    KvDims d;
    hlq_status s = check_cache(c, cache, cache_bytes, &d);
    if (s != HLQ_OK) return s;
    if ((s = check_sizes(T, d.H, d.D)) != HLQ_OK) return s;
    if (!hlq_is_float(type)) return HLQ_ERR_UNSUPPORTED;
    if (T == 0 || (!k && !v)) return HLQ_OK;
    if (!slots) return HLQ_ERR_NULL;
    if ((uintptr_t)slots & 7u) return HLQ_ERR_BAD_STRIDE;
    if (k && (s = hlq_check_rows(k, T, d.H, d.D, k_ts, k_hs, type, true)) != HLQ_OK) return s;
    if (v && (s = hlq_check_rows(v, T, d.H, d.D, v_ts, v_hs, type, true)) != HLQ_OK) return s;
    if (hlq_rows_overlap(hlq_span(k, T, d.H, k_ts, k_hs, type), hlq_span(v, T, d.H, v_ts, v_hs, type), d.D)) return HLQ_ERR_BAD_STRIDE;
    Read a{};
    a.T = T;
    a.H = d.H;
    a.first = k ? 0 : d.H;
    a.slots = slots;
    a.k = KvRows{k, k_ts, k_hs};
    a.v = KvRows{v, v_ts, v_hs};
    a.kv = hlq_kv_view(d, cache);
    a.lanes = d.D / 8;
    a.fit = 64 / a.lanes;
    cut_heads(T, (k && v ? 2 : 1) * d.H, a.fit, a.parts, a.per_part);
    const int64_t each = tokens_of_launch(a.parts);
    const int bytes = hlq_dtype_bytes(type);
    const hipStream_t st = (hipStream_t)stream;
    hlq_clear_stale_error();
    for (int64_t t = 0; t < T; t += each) {
        Read b = a;
        b.T = T - t < each ? T - t : each;
        b.slots = slots + t;
        b.k = behind(a.k, t, bytes), b.v = behind(a.v, t, bytes);
        const dim3 grid = grid_of(b.T, b.parts);
        if (type == HLQ_F16) launch_read<HLQ_F16>(b, d.type, grid, st);
        else if (type == HLQ_BF16) launch_read<HLQ_BF16>(b, d.type, grid, st);
        else launch_read<HLQ_F32>(b, d.type, grid, st);
    }
    return hlq_hip_status(hipGetLastError());
}

}  // extern "C"
