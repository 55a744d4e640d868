// Attention of one new token over the paged cache:  out = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q . k_j - m),  m the largest score.
//
// One pass over keys and values with the running maximum and sum; the maximum that exponentials are taken from is
// kept while no score passes it by 2^8, and is a whole power of two: so sums are rarely multiplied, and exactly.  A wavefront has the query heads of one
// kv head (16 of them at most) and goes through tiles of 32 tokens, all in registers:
//   scores    two products 16 tokens x 16 heads, keys the first operand.  A lane has tokens 4 g .. 4 g + 3 of each for one head (g = lane / 16).
//   weights   are then where the second product wants them: its sum over tokens may take them in any order, so place 8 g + e of the sum is
//             token 4 g + e for e < 4 and 16 + 4 g + e - 4 behind.  No weight changes lanes.
//   values    a lane loads dim / 16 successive values of its eight tokens, rows whole, and turns the block in registers (a byte permutation
//             makes two tokens' values of one column): dim / 16 products whose row r is column (dim / 16) r + j.
// The four wavefronts of a workgroup take tiles in turn and meet in LDS.  A sequence is cut over up to `cuts` workgroups by its length; the last one to
// end adds their sums in order (hand-over by device-scope stores and a counter), so results do not depend on which is last.
// Weights are two terms of 16 bits (the second product runs twice: it waits for memory anyway), so that p is not rounded to 8 bits.  8- and 4-bit
// values become bf16, which holds them and their scale exactly (from 2^-126 up); f16 queries are two bf16 terms then.
// A wavefront that ends with a NaN, or with scores so large that their rounding is felt, goes through its tiles once more, multiplies without the values that are infinite or NaN, and adds what they do to those that see them by counting.
// Keys' rows are asked for in lines of 128 bytes, and rows are not kept in the caches: by 64 bytes of each of 16 rows, and kept, 64 x 4096 tokens took 204 us for 184.
// What bounds it: memory.  64 sequences of 4096 tokens, 8 heads of 128 with 64 queries: 16 bits 182 to 185 us = 5.8 to 5.9 TB/s (a plain read reaches 6.9), 8 bits 111 to 118 = 4.7 to 5.0, 4 bits
// 65 to 68 = 4.3; the fewer bits a tile has, the less of it is on its way (a wavefront has one tile, 17, 8.5 or 4.4 KB; two tiles a wavefront, or fewer registers and four
// workgroups a unit, brought nothing), and vector instructions take 44 % of the cycles at 4 bits (19 % at 16).  Pages of 16 tokens 5.1 TB/s.  A single sequence of 1000 tokens takes 8.6 us, one token 5.3: of dependent steps,
// the length, the table, keys, and the cuts' hand-over.
// Pages' pieces are read through buffer descriptors that end with the sequence's last token: what lies behind, and columns past dim, is 0 without a
// comparison.
#include "hlq_kv.h"

namespace {

constexpr int WAVES = 4, TILE = 32;
constexpr float NONE = -__builtin_inff();

typedef __bf16 bf8v __attribute__((ext_vector_type(8)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));

struct Decode {
    KvView kv;
    int D, group, blocks, cuts;   // blocks of 16 query heads of a kv head
    KvRows q;
    const int32_t *table;
    int64_t ld_table;
    int width;
    const int32_t *lengths;
    int window;
    float scale, sign;            // the scale's magnitude times log2(e) (1 if it is 0), and its sign
    KvRows out;
    int otype;
    int *arrived;
    float *partial;
    int rows;                     // of a partial result: min(16, group)
};

// LIFT: what the largest weight is brought to is 2^(LIFT - 1) to 2^LIFT (2^8 times that while the base is kept); REST: what a weight's second term is multiplied by.
// f16 ends at 2^16 and has steps of 2^-24 at its lower end, so that small weights beside a large one would be lost (8192 tokens of which 128 have a score that is 17 higher: a tenth
// of the others' share): they stand as high as they can, and their second terms are 2^11 times as large, with a product that is brought back before it is added.
// bf16 has fp32's exponents and needs neither.
template <int C> struct Fragment { using type = bf8v; using scalar = __bf16; static constexpr float LIFT = 0.f, REST = 1.f; };
template <> struct Fragment<HLQ_F16> { using type = half8v; using scalar = _Float16; static constexpr float LIFT = 7.f, REST = 2048.f; };

__device__ __forceinline__ float4v multiply(bf8v a, bf8v b, float4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ float4v multiply(half8v a, half8v b, float4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// lanes 8..15 of sixteen get of b what lanes 0..7 have, and these of a what lanes 8..15 had: a of the first eight lanes and b of the last stay
__device__ __forceinline__ void change_places(uint32_t &a, uint32_t &b)
{
    const uint32_t was = a;
    a = (uint32_t)__builtin_amdgcn_update_dpp((int)a, (int)b, 0x128, 0xf, 0xc, false);
    b = (uint32_t)__builtin_amdgcn_update_dpp((int)b, (int)was, 0x128, 0xf, 0x3, false);
}

// over the four lanes of a head
__device__ __forceinline__ float over_lanes_max(float v)
{
    auto s = __builtin_amdgcn_permlane32_swap(as_bits(v), as_bits(v), false, false);
    v = fmaxf(as_float(s[0]), as_float(s[1]));
    s = __builtin_amdgcn_permlane16_swap(as_bits(v), as_bits(v), false, false);
    return fmaxf(as_float(s[0]), as_float(s[1]));
}
__device__ __forceinline__ float over_lanes_sum(float v)
{
    auto s = __builtin_amdgcn_permlane32_swap(as_bits(v), as_bits(v), false, false);
    v = as_float(s[0]) + as_float(s[1]);
    s = __builtin_amdgcn_permlane16_swap(as_bits(v), as_bits(v), false, false);
    return as_float(s[0]) + as_float(s[1]);
}
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
// what a maximum is subtracted as: where nothing was seen, or only -infinity, 0, so that no difference is NaN
__device__ __forceinline__ float base_of(float m) { return m == NONE ? 0.f : m; }

// adds +infinity, -infinity, or for a NaN both to the sums of the heads that have its token in `present`
template <class F>
__device__ __forceinline__ void count_odd(F v, uint32_t present, float4v &sum)
{
    const float4v none = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int sign = 0; sign < 2; ++sign) {
        F sees, is;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            sees[e] = present >> e & 1u ? 1.f : 0.f;
            is[e] = (sign ? (float)v[e] > NONE : (float)v[e] < __builtin_inff()) ? 0.f : 1.f;
        }
        const float4v count = multiply(is, sees, none);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (count[i] > 0.f) sum[i] += sign ? NONE : __builtin_inff();
    }
}
// two values, 0 where they are infinite or NaN
template <class F>
__device__ __forceinline__ uint32_t without_odd(uint32_t two)
{
    constexpr uint32_t most = __is_same(F, half8v) ? 0x7c00u : 0x7f80u;
    const uint32_t low = (two & most) == most ? 0u : two & 0xffffu, high = (two >> 16 & most) == most ? 0u : two & 0xffff0000u;
    return low | high;
}

constexpr int OUTSIDE = 0x7fffffff;   // an offset that every descriptor ends before

__device__ __forceinline__ __amdgpu_buffer_rsrc_t descriptor(const void *p, int bytes) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, bytes, 0x00020000); }

// N dwords (or 2 bytes: N = 0) through a descriptor, not to be kept in the caches.  (No scalar offset: only what is added in the lane counts in the comparison with the end.)
template <int N>
__device__ __forceinline__ void fetch(uint32_t *to, __amdgpu_buffer_rsrc_t r, int offset)
{
    if constexpr (N == 0) to[0] = __builtin_amdgcn_raw_buffer_load_b16(r, offset, 0, 2);
    else if constexpr (N == 1) to[0] = __builtin_amdgcn_raw_buffer_load_b32(r, offset, 0, 2);
    else if constexpr (N == 2) {
        const mx4_u2 v = __builtin_bit_cast(mx4_u2, __builtin_amdgcn_raw_buffer_load_b64(r, offset, 0, 2));
        to[0] = v.x, to[1] = v.y;
    } else {
        static_assert(N == 4, "");
        const mx4_u4 v = __builtin_bit_cast(mx4_u4, __builtin_amdgcn_raw_buffer_load_b128(r, offset, 0, 2));
        to[0] = v.x, to[1] = v.y, to[2] = v.z, to[3] = v.w;
    }
}

// two values of 8 or 4 bits as bf16, times their scale; i: which two of the four or eight in c
template <int C, int I>
__device__ __forceinline__ uint32_t widen(uint32_t c, float scale)
{
    if constexpr (C == HLQ_MX4) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, I));
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, scale, I));
}

// C: the cache's type, T: the queries', DP: dim up to 64, 128 or 256.  Dims above 128 have one wavefront a SIMD, but two where 8- or 4-bit rows and queries of one term leave the
// registers for it (32 x 4096 tokens of dim 256, 8 bits 115 -> 104 us, 4 bits 91 -> 72; queries of two terms 118 -> 146 and 93 -> 100).
template <int C, int T, int DP>
__global__ void __launch_bounds__(64 * WAVES, DP <= 128 ? 3 : (C == HLQ_MX8 || C == HLQ_MX4) && T == HLQ_BF16 ? 2 : 1)
hlq_attn_decode_kernel(const Decode a)
{
    using F = typename Fragment<C>::type;
    using S = typename Fragment<C>::scalar;
    constexpr float LIFT = Fragment<C>::LIFT, REST = Fragment<C>::REST;
    constexpr bool MX = C == HLQ_MX8 || C == HLQ_MX4;
    constexpr int PER = C == HLQ_MX4 ? 8 : C == HLQ_MX8 ? 4 : 2;   // values of a dword
    constexpr int KS = DP / 32, E = DP / 16;                       // products over dim; columns of a lane
    constexpr int TERMS = MX && T == HLQ_F16 ? 2 : 1;              // of the queries
    constexpr int PITCH = DP + 4;                                  // of a row in LDS
    // a lane's pieces of a key (16 bytes or a quarter of a row), and their values; products of a piece; pieces of a value's row (VALUE_DWORDS 0: two bytes)
    constexpr int KEY_DWORDS = KS * 8 / PER, KEY_PIECE = KEY_DWORDS < 4 ? KEY_DWORDS : 4, KEY_PIECES = KEY_DWORDS / KEY_PIECE, PIECE_VALUES = KEY_PIECE * PER;
    constexpr int PRODUCTS = PIECE_VALUES / 8;
    constexpr bool PAIRED = KEY_PIECES > 1, TWO_ROWS = C == HLQ_MX4 && DP == 128;
    constexpr int VALUE_DWORDS = TWO_ROWS ? 2 : E / PER, VALUE_PIECE = VALUE_DWORDS < 4 ? VALUE_DWORDS : 4, VALUE_PIECES = VALUE_DWORDS ? VALUE_DWORDS / VALUE_PIECE : 1;
    constexpr int VALUE_LOADS = TWO_ROWS ? 2 : 4;                  // of 16 tokens
    __shared__ __attribute__((aligned(16))) float sums[WAVES * 16 * PITCH];
    __shared__ float tops[WAVES][16], totals[WAVES][16];

    const int lane = (int)(threadIdx.x & 63u), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int col = lane & 15, g = lane >> 4;
    const auto column_of = [](int lane) { return TWO_ROWS ? 16 * (lane & 7) + 8 * (lane >> 3) : E * lane; };   // the first of a lane's E columns
    int id = (int)blockIdx.x;
    const int h = id % a.kv.H;
    id /= a.kv.H;
    const int block = id % a.blocks;
    id /= a.blocks;
    const int cut = id % a.cuts, b = id / a.cuts;

    const int log_page = a.kv.log_page;
    int64_t room = (int64_t)a.width << log_page;
    int n = a.lengths[b];
    n = n < 0 ? 0 : n > room ? (int)room : n;
    const int start = a.window > 0 && n > a.window ? n - a.window : 0, first = start & ~(TILE - 1);
    const int steps = (n - first + TILE - 1) / TILE;
    // workgroups that have a share, at least one, which writes the zeros of an empty sequence
    int share = (steps + a.cuts - 1) / a.cuts;
    share = (share + WAVES - 1) / WAVES * WAVES;
    const int active = steps > 0 ? (steps + share - 1) / share : 1;
    if (cut >= active) return;
    const int step_end = (cut + 1) * share < steps ? (cut + 1) * share : steps;

    const int head0 = block * 16, heads = a.group - head0 < 16 ? a.group - head0 : 16;   // of this workgroup
    const int first_head = h * a.group + head0;
    // queries, the second operand: lane (head, g) has what the keys' lanes have of place g of a product
    F query[TERMS][KS];
    {
        using V = typename Mx4Type<T>::type;
        const V *q = (const V *)a.q.p + b * a.q.ts + (int64_t)(first_head + (col < heads ? col : 0)) * a.q.hs;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int d = (4 * (s / PRODUCTS) + g) * PIECE_VALUES + s % PRODUCTS * 8;
            V v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (V)0.f;
            if (col < heads && d < a.D && a.sign != 0.f) mx4_read8<false>(q + d, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = a.sign < 0.f ? -v[i] : v[i];   // so that the largest score has the largest product
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const S hi = (S)(float)v[i];
                query[0][s][i] = hi;
                if constexpr (TERMS == 2) query[1][s][i] = (S)((float)v[i] == (float)hi ? 0.f : (float)v[i] - (float)hi);   // (infinities have no rest)
            }
        }
    }

    // Offsets of this lane.  Keys' rows come in eights, 128 bytes of each at a time where they are that long, so that lines are asked for whole: lanes
    // 0..7 of sixteen have the first four pieces of rows 0..7, lanes 8..15 the next four, a second load rows 8..15; then they change places.
    // Values: a lane's eight tokens row by row; rows of 64 bytes two at a time (TWO_ROWS), then lanes change places too.
    const int row_bytes = a.kv.row_bytes;
    int key_at[KEY_PIECES], value_at[VALUE_LOADS][VALUE_PIECES];
#pragma unroll
    for (int i = 0; i < KEY_PIECES; ++i) {
        const int row = PAIRED ? (i & 1) * 8 + (col & 7) : col, d = (PAIRED ? 8 * (i >> 1) + 4 * (col >> 3) + g : 4 * i + g) * PIECE_VALUES;
        key_at[i] = d < a.D ? row * row_bytes + d * 4 / PER : OUTSIDE;
    }
#pragma unroll
    for (int i = 0; i < VALUE_PIECES; ++i) {
        const int d = TWO_ROWS ? 16 * (col & 7) : E * col + i * VALUE_PIECE * PER;
#pragma unroll
        for (int e = 0; e < VALUE_LOADS; ++e) value_at[e][i] = d < a.D ? (4 * g + (TWO_ROWS ? 2 * e + (col >> 3) : e)) * row_bytes + d * 4 / PER : OUTSIDE;
    }
    int key_scale_at[KEY_PIECES], value_scale_at = 0;
    if constexpr (MX) {
#pragma unroll
        for (int i = 0; i < KEY_PIECES; ++i) {
            const int blk = (4 * i + g) * PIECE_VALUES / 32;
            key_scale_at[i] = blk < a.kv.blocks ? (blk << log_page) + col : OUTSIDE;
        }
        const int blk = column_of(col) / 32;
        value_scale_at = blk < a.kv.blocks ? (blk << log_page) + 4 * g : OUTSIDE;
    }

    // what is loaded of a tile: its two halves of 16 tokens lie in a page each
    struct Keys { uint32_t v[2][KEY_DWORDS], scale[2][KEY_PIECES]; };
    struct Values { uint32_t v[2 * VALUE_LOADS][VALUE_DWORDS ? VALUE_DWORDS : 1], scale[2]; };
    struct Half { int page, at, bytes; };   // where its tokens begin in which page, the bytes of those up to the sequence's end
    const int32_t *const table = a.table + b * a.ld_table;
    auto half_of = [&](int tok, int half) {
        tok += 16 * half;
        const int left = n - tok;
        int page = table[(left > 0 ? tok : n - 1) >> log_page];
        page = page < 0 ? 0 : page >= (int)a.kv.pages ? (int)a.kv.pages - 1 : page;   // (fewer than 2^31)
        return Half{uniform(page), uniform(tok & ((1 << log_page) - 1)), uniform((left < 0 ? 0 : left < 16 ? left : 16) * row_bytes)};
    };
    // of this kv head: the keys' rows of page 0, bytes from page to page, from keys to values; the same of scale bytes
    const uint32_t piece = (uint32_t)row_bytes << log_page, scale_piece = (uint32_t)a.kv.blocks << log_page;
    const uint8_t *const rows0 = a.kv.codes + (uint64_t)piece * h, *const scales0 = a.kv.scales + (uint64_t)scale_piece * h;
    const uint32_t to_values = piece * a.kv.H, page_bytes = 2 * to_values, scale_to_values = scale_piece * a.kv.H, scale_page_bytes = 2 * scale_to_values;
    auto load_keys = [&](Keys &k, const Half (&where)[2]) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const Half &w = where[half];
            const auto r = descriptor(rows0 + (uint64_t)page_bytes * (uint32_t)w.page + (uint32_t)(w.at * row_bytes), w.bytes);
#pragma unroll
            for (int i = 0; i < KEY_PIECES; ++i) fetch<KEY_PIECE>(k.v[half] + i * KEY_PIECE, r, key_at[i]);
            if constexpr (MX) {
                const auto rs = descriptor(scales0 + (uint64_t)scale_page_bytes * (uint32_t)w.page + (uint32_t)w.at, uniform((int)scale_piece - w.at));
#pragma unroll
                for (int i = 0; i < KEY_PIECES; ++i) k.scale[half][i] = __builtin_amdgcn_raw_buffer_load_b8(rs, key_scale_at[i], 0, 0);
            }
        }
    };
    auto load_values = [&](Values &v, const Half (&where)[2]) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const Half &w = where[half];
            const auto r = descriptor(rows0 + (uint64_t)page_bytes * (uint32_t)w.page + (to_values + (uint32_t)(w.at * row_bytes)), w.bytes);
#pragma unroll
            for (int e = 0; e < VALUE_LOADS; ++e)
#pragma unroll
                for (int i = 0; i < VALUE_PIECES; ++i) fetch<VALUE_PIECE>(v.v[VALUE_LOADS * half + e] + i * VALUE_PIECE, r, value_at[e][i]);
            if constexpr (MX) {
                const auto rs = descriptor(scales0 + (uint64_t)scale_page_bytes * (uint32_t)w.page + (scale_to_values + (uint32_t)w.at), uniform((int)scale_piece - w.at));
                v.scale[half] = __builtin_amdgcn_raw_buffer_load_b32(rs, value_scale_at, 0, 0);
            }
        }
    };

    float4v acc[E];
    float base = 0.f, most = NONE, total = 0.f;   // most: scores up to it need no new base
    // lane (head, g) has the columns of lane 4 g + i in its row i
    auto own_sums = [&](int i, int j) { return (float4v *)(sums + (wave * 16 + col) * PITCH + column_of(4 * g + i) + j); };
    // The first pass looks at nothing.  What an infinite or NaN value makes of other heads' or tokens' weights, 0 times itself, shows as NaN; then comes a careful one, which multiplies
    // the values that are numbers and adds +infinity, -infinity, or both for a NaN, where a head sees one: with a score above -infinity, however small the weight.
    const auto pass = [&](auto careful) {
        constexpr bool CAREFUL = decltype(careful)::value;
#pragma unroll
        for (int j = 0; j < E; ++j) acc[j] = (float4v){0.f, 0.f, 0.f, 0.f};
        base = 0.f, most = NONE, total = 0.f;
        int step = cut * share + wave;
        if (step < step_end) {
            Keys keys;
            Values values;
            Half where[2];
            auto look_up = [&](int step) {
#pragma unroll
                for (int half = 0; half < 2; ++half) where[half] = half_of(first + step * TILE, half);
            };
            look_up(step);
            load_keys(keys, where);
            load_values(values, where);
            for (;;) {
                const int next = step + WAVES;
                const bool more = next < step_end;
                if (!CAREFUL && more) look_up(next);   // (a careful pass has no registers for the next tile)
                const int tok0 = first + step * TILE;
                const bool part = tok0 < start || tok0 + TILE > n;   // some tokens are not to be seen

                // scores
                float x[8];
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    float4v s = {0.f, 0.f, 0.f, 0.f};
                    if constexpr (PAIRED)
#pragma unroll
                        for (int i = 0; i < KEY_DWORDS; i += 8)
#pragma unroll
                            for (int w = i; w < i + 4; ++w) change_places(keys.v[half][w], keys.v[half][w + 4]);
#pragma unroll
                    for (int i = 0; i < KS; ++i) {
                        mx4_u4 w;
                        if constexpr (C == HLQ_MX4) {
                            const float scale = as_float(keys.scale[half][i / PRODUCTS] << 23);
                            const uint32_t c = keys.v[half][i];
                            w = (mx4_u4){widen<C, 0>(c, scale), widen<C, 1>(c, scale), widen<C, 2>(c, scale), widen<C, 3>(c, scale)};
                        } else if constexpr (C == HLQ_MX8) {
                            const float scale = as_float(keys.scale[half][i / PRODUCTS] << 23);
                            const uint32_t c = keys.v[half][2 * i], d = keys.v[half][2 * i + 1];
                            w = (mx4_u4){widen<C, 0>(c, scale), widen<C, 1>(c, scale), widen<C, 0>(d, scale), widen<C, 1>(d, scale)};
                        } else
                            w = (mx4_u4){keys.v[half][4 * i], keys.v[half][4 * i + 1], keys.v[half][4 * i + 2], keys.v[half][4 * i + 3]};
                        const F k = __builtin_bit_cast(F, w);
#pragma unroll
                        for (int t = 0; t < TERMS; ++t) s = multiply(k, query[t][i], s);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[4 * half + e] = s[e];
                }
                if (!CAREFUL && more) load_keys(keys, where);
                if (part) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int tok = tok0 + (e < 4 ? 4 * g + e : 12 + 4 * g + e);
                        if (tok < start || tok >= n) x[e] = NONE;
                    }
                }
                float m = x[0];
#pragma unroll
                for (int e = 1; e < 8; ++e) m = fmaxf(m, x[e]);
                m = over_lanes_max(m) * a.scale;
                if (__builtin_expect(__any(m > most), 0)) {
                    const bool now = m > most;
                    const float to = now ? ceilf(m) - LIFT : base;
                    const float keep = !now || most == NONE ? 1.f : exp2_above_0(base - to);
                    base = to;
                    most = now ? to + (LIFT + 8.f) : most;
                    total *= keep;
#pragma unroll
                    for (int j = 0; j < E; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[j][i] *= keep;
                }
                uint32_t present = 0;   // tokens that this lane's head sees
                if constexpr (CAREFUL)
#pragma unroll
                    for (int e = 0; e < 8; ++e) present |= (uint32_t)(x[e] > NONE) << e;
                F p, rest;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float w = __builtin_amdgcn_exp2f(CAREFUL ? above_base(x[e], a.scale, base) : fmaf(x[e], a.scale, -base));
                    total += w;
                    p[e] = (S)w;
                    rest[e] = (S)((w - (float)p[e]) * REST);
                }

                // values, two tokens' of one column in a register
                uint32_t rows[8][E / 2];
                if constexpr (TWO_ROWS)
#pragma unroll
                    for (int e = 0; e < 4; ++e) change_places(values.v[e][0], values.v[e][1]);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if constexpr (MX) {
                        // the conversion takes the eight bits of the exponent only
                        const uint32_t four = values.scale[e >> 2];
                        const float scale = as_float((e & 3) == 3 ? four >> 1 : four << (23 - 8 * (e & 3)));
#pragma unroll
                        for (int i = 0; i < E / 2; ++i) {
                            const uint32_t c = TWO_ROWS ? values.v[e >> 1][e & 1] : values.v[e][i * 2 / PER];
                            if constexpr (C == HLQ_MX4) rows[e][i] = i % 4 == 0 ? widen<C, 0>(c, scale) : i % 4 == 1 ? widen<C, 1>(c, scale) : i % 4 == 2 ? widen<C, 2>(c, scale) : widen<C, 3>(c, scale);
                            else rows[e][i] = i % 2 == 0 ? widen<C, 0>(c, scale) : widen<C, 1>(c, scale);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < E / 2; ++i) rows[e][i] = values.v[e][i];
                    }
                }
                if (part) {
                    // of tokens that are not to be seen nothing enters, whatever stands there
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int tok = tok0 + (e < 4 ? 4 * g + e : 12 + 4 * g + e);
                        if (tok < start || tok >= n) {
                            p[e] = (S)0.f;
                            rest[e] = (S)0.f;
#pragma unroll
                            for (int i = 0; i < E / 2; ++i) rows[e][i] = 0u;
                        }
                    }
                }
                const auto turned = [&](int j) {
                    const uint32_t pick = j & 1 ? 0x07060302u : 0x05040100u;
                    const mx4_u4 w = {__builtin_amdgcn_perm(rows[1][j >> 1], rows[0][j >> 1], pick), __builtin_amdgcn_perm(rows[3][j >> 1], rows[2][j >> 1], pick),
                                      __builtin_amdgcn_perm(rows[5][j >> 1], rows[4][j >> 1], pick), __builtin_amdgcn_perm(rows[7][j >> 1], rows[6][j >> 1], pick)};
                    return __builtin_bit_cast(F, w);
                };
                if constexpr (CAREFUL) {
#pragma unroll
                    for (int j = 0; j < E; ++j) count_odd(turned(j), present, acc[j]);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
#pragma unroll
                        for (int i = 0; i < E / 2; ++i) rows[e][i] = without_odd<F>(rows[e][i]);
                }
                if constexpr (REST == 1.f) {
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        const F v = turned(j);
                        acc[j] = multiply(v, p, acc[j]);
                        acc[j] = multiply(v, rest, acc[j]);
                    }
                } else {
                    // Several columns at a time, so that nothing waits for a second term's product (32 x 4096 tokens of dim 256: one by one 214 us, so 198).  Dim 128: the branch,
                    // which is hardly ever passed by, keeps the compiler from having more on its way than there are registers (64 x 4096 tokens 205 us, so 183).
                    constexpr int AT_ONCE = DP > 128 ? 4 : 2;
                    const mx4_u4 second = __builtin_bit_cast(mx4_u4, rest);
                    const bool two = DP != 128 || __any(((second.x | second.y | second.z | second.w) & 0x7fff7fffu) != 0u);
#pragma unroll
                    for (int j0 = 0; j0 < E; j0 += AT_ONCE) {
                        float4v low[AT_ONCE];
#pragma unroll
                        for (int i = 0; i < AT_ONCE; ++i) {
                            const F v = turned(j0 + i);
                            acc[j0 + i] = multiply(v, p, acc[j0 + i]);
                            low[i] = multiply(v, rest, (float4v){0.f, 0.f, 0.f, 0.f});
                        }
                        if (two)
#pragma unroll
                            for (int i = 0; i < 4 * AT_ONCE; ++i) acc[j0 + i / 4][i % 4] = fmaf(low[i / 4][i % 4], 1.f / REST, acc[j0 + i / 4][i % 4]);
                    }
                }
                if (CAREFUL && more) {
                    look_up(next);
                    load_keys(keys, where);
                }
                if (more) load_values(values, where);
                if (!more) break;
                step = next;
            }
        }
    };
    pass(std::false_type());
    bool odd = !(total < __builtin_inff()) || fabsf(base) >= LARGE;
#pragma unroll
    for (int j = 0; j < E; ++j) odd = odd || __builtin_isunordered(acc[j][0], acc[j][1]) || __builtin_isunordered(acc[j][2], acc[j][3]);
    if (__builtin_expect(__any(odd && col < heads), 0)) pass(std::true_type());   // (lanes past the heads have queries of 0, which an infinite key makes NaN)
    total = over_lanes_sum(total);

    // the wavefronts' sums meet in LDS
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < E; j += 4) *own_sums(i, j) = (float4v){acc[j][i], acc[j + 1][i], acc[j + 2][i], acc[j + 3][i]};
    if (g == 0) {
        tops[wave][col] = most == NONE ? NONE : base;
        totals[wave][col] = total;
    }
    __syncthreads();
    const int64_t who = ((int64_t)b * a.blocks + block) * a.kv.H + h;
    const int64_t size = (int64_t)a.rows * (DP + 2);              // of a partial result: sums, then maximum and total of each head
    float *const partial = active > 1 ? a.partial + who * a.cuts * size : nullptr;
    const bool alone = active == 1;
    auto put = [&](int head, int d, float4v v) {
        const int64_t at = b * a.out.ts + (int64_t)(first_head + head) * a.out.hs + d;
        mx4_store4(a.out.p, a.otype, at, (const float *)&v, 4);
    };
    for (int it = (int)threadIdx.x; it < heads * (DP / 4); it += 64 * WAVES) {
        const int head = it / (DP / 4), d = it % (DP / 4) * 4;
        float m = NONE;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) m = fmaxf(m, tops[w][head]);
        const float base = base_of(m);
        float4v sum = {0.f, 0.f, 0.f, 0.f};
        float all = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float weight = exp2_above_0(tops[w][head] - base);
            const float4v v = *(const float4v *)(sums + (w * 16 + head) * PITCH + d);
            all = fmaf(weight, totals[w][head], all);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] = fmaf(weight, v[i], sum[i]);
        }
        if (alone) {
            const float by = 1.f / all;
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] = all == 0.f ? 0.f : sum[i] * by;   // nothing seen is 0, whatever the values are
            if (d < a.D) put(head, d, sum);
        } else {
            uint64_t *to = (uint64_t *)(partial + cut * size) + it;   // the first two of each four, then the others, so that a store's lanes stand side by side
#pragma unroll
            for (int i = 0; i < 2; ++i)
                __hip_atomic_store(to + i * (a.rows * (DP / 4)), as_bits(sum[2 * i]) | (uint64_t)as_bits(sum[2 * i + 1]) << 32, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (d == 0)
                __hip_atomic_store((uint64_t *)(partial + cut * size + a.rows * DP) + head, as_bits(m) | (uint64_t)as_bits(all) << 32,
                                   __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    if (alone) return;

    // Device-scope stores are complete before the arrival is counted; whoever is last adds the cuts in their order.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    int *const last = (int *)&tops[0][0];
    if (threadIdx.x == 0) *last = __hip_atomic_fetch_add(a.arrived + who, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == active - 1;
    __syncthreads();
    if (!*last) return;
    if (threadIdx.x == 0) __hip_atomic_store(a.arrived + who, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // the sums of eight cuts at a time; the first of them are on their way while the weights are made
    uint64_t pair[8][2];
    auto fetch_sums = [&](int it, int c0) {
        const uint64_t *from = (const uint64_t *)partial + it;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = c0 + i < active ? c0 + i : c0;
#pragma unroll
            for (int e = 0; e < 2; ++e) pair[i][e] = __hip_atomic_load(from + c * (size / 2) + e * (a.rows * (DP / 4)), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    };
    const int items = heads * (DP / 4);
    if ((int)threadIdx.x < items) fetch_sums((int)threadIdx.x, 0);
    float *const weights = sums, *const shares = sums + 16 * 128;   // [head][cut], then 1 / total of each head
    for (int head = wave; head < heads; head += WAVES) {
        float m[2], all[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int c = lane + 64 * i;
            m[i] = NONE, all[i] = 0.f;
            if (c < active) {
                const uint64_t pair = __hip_atomic_load((const uint64_t *)(partial + c * size + a.rows * DP) + head, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                m[i] = as_float((uint32_t)pair);
                all[i] = as_float((uint32_t)(pair >> 32));
            }
        }
        float most = fmaxf(m[0], m[1]), sum = 0.f;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) most = fmaxf(most, __shfl_xor(most, o));
        const float base = base_of(most);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float w = exp2_above_0(m[i] - base);
            sum = fmaf(w, all[i], sum);
            weights[head * 128 + lane + 64 * i] = w;
        }
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
        if (lane == 0) shares[head] = sum == 0.f ? 0.f : 1.f / sum;   // (0: nothing seen)
    }
    __syncthreads();
    for (int it = (int)threadIdx.x; it < items; it += 64 * WAVES) {
        const int head = it / (DP / 4), d = it % (DP / 4) * 4;
        float4v sum = {0.f, 0.f, 0.f, 0.f};
        for (int c0 = 0; c0 < active; c0 += 8) {
            if (c0 > 0 || it != (int)threadIdx.x) fetch_sums(it, c0);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c0 + i < active) {
                    const float w = weights[head * 128 + c0 + i];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        sum[2 * e] = fmaf(w, as_float((uint32_t)pair[i][e]), sum[2 * e]);
                        sum[2 * e + 1] = fmaf(w, as_float((uint32_t)(pair[i][e] >> 32)), sum[2 * e + 1]);
                    }
                }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = shares[head] == 0.f ? 0.f : sum[i] * shares[head];
        if (d < a.D) put(head, d, sum);
    }
}

// How a launch is cut.  One round of the card, three workgroups a compute unit, if there are tokens for that, 128 a workgroup at least; and workgroups of 512 KB of
// keys and values at most (1024 tokens at least), so that long sequences do not end alone, where that is not more than 16384 of them.  (Two sequences of
// 131072 tokens in 4 bits: 2048 workgroups 79 us, 768 58; 64 of 0 .. 8191 in 16 bits: workgroups of 512, 1024, 2048 tokens 223, 215, 217.)  As the last workgroup of a
// sequence adds its cuts, they are no more than the root of a sixteenth of the tokens unless a quarter of the card would be empty (one sequence, 8 heads: 1000 tokens 8,
// 4, 2 cuts 8.7, 9.5, 11.7 us; 4000 tokens 32, 16, 8 cuts 12.9, 11.6, 12.8; 16000 tokens 63, 32 cuts 22.0, 18.2).  128 cuts at most, none where the counters do not suffice.
constexpr int64_t WANTED = 768, FILLED = 192, MOST_WORKGROUPS = 16384, MOST_BYTES = 512 << 10, LEAST_TOKENS = 128, MOST_CUTS = 128;
struct Cuts {
    int cuts;
    size_t room;   // partial results in the workspace, enough for fewer sequences and narrower tables too
};
Cuts cuts_of(int64_t workgroups, int64_t tokens, int row_bytes)
{
    if (workgroups < 1 || tokens <= LEAST_TOKENS) return {1, 0};
    const bool whole = workgroups > HLQ_WS_ARRIVAL_COUNTERS;
    if (whole) workgroups = HLQ_WS_ARRIVAL_COUNTERS;
    const auto up = [](int64_t n, int64_t by) { return (n + by - 1) / by; };
    const auto least = [](int64_t a, int64_t b) { return a < b ? a : b; };
    const auto most = [](int64_t a, int64_t b) { return a < b ? b : a; };
    int64_t root = 8;
    while (root < MOST_CUTS && root * root * 16 < tokens) ++root;
    const int64_t share = most(1024, MOST_BYTES / (2 * row_bytes)), possible = least(up(tokens, LEAST_TOKENS), MOST_CUTS);
    const int64_t round = least(most(WANTED / workgroups, 1), most(root, FILLED / workgroups));
    const int64_t cuts = least(most(round, least(up(tokens, share), MOST_WORKGROUPS / workgroups)), possible);
    const int64_t room = least(most(WANTED + workgroups, least(workgroups * up(tokens, share), MOST_WORKGROUPS + workgroups)), workgroups * possible);
    return {whole ? 1 : (int)cuts, (size_t)room};
}
int padded(int D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }

struct Shape {
    KvDims d;
    int group, blocks, cuts;
    int64_t workgroups;
    size_t bytes;
};
hlq_status shape_of(const hlq_kv_desc *c, int32_t q_heads, int64_t B, int32_t width, Shape *out)
{
    Shape s{};
    const hlq_status st = hlq_kv_check(c, &s.d);
    if (st != HLQ_OK) return st;
    if (q_heads < 1 || q_heads % s.d.H || B < 0 || width < 0) return HLQ_ERR_BAD_DESC;
    if (q_heads > KV_MOST_HEADS) return HLQ_ERR_UNSUPPORTED;
    s.group = q_heads / s.d.H;
    s.blocks = (s.group + 15) / 16;
    const int64_t tokens = (int64_t)width << s.d.log_page;
    if (B > ((int64_t)1 << 24) / (s.d.H * s.blocks) || tokens > 0x7fffffe0) return HLQ_ERR_UNSUPPORTED;   // a launch has fewer than 2^32 lanes
    s.workgroups = B * s.d.H * s.blocks;
    const Cuts k = cuts_of(s.workgroups, tokens, s.d.row_bytes);
    s.cuts = k.cuts;
    s.bytes = HLQ_WS_COUNTER_BYTES + k.room * (size_t)((s.group < 16 ? s.group : 16) * (padded(s.d.D) + 2)) * sizeof(float);
    s.bytes = (s.bytes + 255u) & ~(size_t)255u;
    *out = s;
    return HLQ_OK;
}

template <int C, int T>
void launch(const Decode &a, int64_t grid, hipStream_t st)
{
    const dim3 g((unsigned)grid), block(64 * WAVES);
    switch (padded(a.D)) {
    case 64: hlq_attn_decode_kernel<C, T, 64><<<g, block, 0, st>>>(a); break;
    case 128: hlq_attn_decode_kernel<C, T, 128><<<g, block, 0, st>>>(a); break;
    default: hlq_attn_decode_kernel<C, T, 256><<<g, block, 0, st>>>(a); break;
    }
}

}  // namespace

extern "C" {

hlq_status hlq_attn_decode_workspace_bytes(const hlq_kv_desc *c, int32_t q_heads, int64_t B, int32_t table_width, size_t *bytes)
{
    Shape s;
    const hlq_status st = shape_of(c, q_heads, B, table_width, &s);
    if (st != HLQ_OK) return st;
    if (!bytes) return HLQ_ERR_NULL;
    *bytes = s.bytes;
    return HLQ_OK;
}

hlq_status hlq_attn_decode(const hlq_kv_desc *c, const void *cache, size_t cache_bytes, int32_t q_heads, int64_t B, hlq_dtype type, const void *q,
                           int64_t q_ts, int64_t q_hs, const int32_t *table, int64_t ld_table, int32_t table_width, const int32_t *lengths, int32_t window,
                           float scale, void *out, hlq_dtype otype, int64_t o_ts, int64_t o_hs, void *ws, size_t ws_bytes, void *stream)
{
    Shape s;
    hlq_status st = shape_of(c, q_heads, B, table_width, &s);
    if (st != HLQ_OK) return st;
    const bool mx = s.d.type == HLQ_MX8 || s.d.type == HLQ_MX4;
    if ((type != HLQ_F16 && type != HLQ_BF16) || (!mx && (int)type != s.d.type) || !hlq_is_float(otype)) return HLQ_ERR_UNSUPPORTED;
    if (window < 0) return HLQ_ERR_BAD_DESC;
    if (B == 0) return HLQ_OK;
    if (!cache || !lengths || (!table && table_width > 0)) return HLQ_ERR_NULL;
    if ((uintptr_t)cache & 15u || (uintptr_t)table & 3u || (uintptr_t)lengths & 3u || ld_table < 0 || ld_table > (int64_t)1 << 40 || (B > 1 && ld_table < table_width))
        return HLQ_ERR_BAD_STRIDE;
    if (cache_bytes < s.d.total) return HLQ_ERR_BUFFER_TOO_SMALL;
    if ((st = hlq_check_rows(q, B, q_heads, s.d.D, q_ts, q_hs, type, false)) != HLQ_OK) return st;
    if ((st = hlq_check_rows(out, B, q_heads, s.d.D, o_ts, o_hs, otype, true)) != HLQ_OK) return st;
    if (s.cuts > 1) {
        if (!ws) return HLQ_ERR_NULL;
        if ((uintptr_t)ws & 15u) return HLQ_ERR_BAD_STRIDE;
        if (ws_bytes < s.bytes) return HLQ_ERR_BUFFER_TOO_SMALL;
    }
    if (hlq_rows_in_the_way(hlq_span(q, B, q_heads, q_ts, q_hs, type), hlq_span(out, B, q_heads, o_ts, o_hs, otype), s.d.D)) return HLQ_ERR_BAD_STRIDE;
    Decode a{};
    a.kv = hlq_kv_view(s.d, cache);
    a.D = s.d.D;
    a.group = s.group;
    a.blocks = s.blocks;
    a.cuts = s.cuts;
    a.q = KvRows{const_cast<void *>(q), q_ts, q_hs};
    a.table = table;
    a.ld_table = ld_table;
    a.width = table_width;
    a.lengths = lengths;
    a.window = window;
    a.scale = scale == 0.f ? 1.f : fabsf(scale) * 1.44269504f;
    a.sign = scale < 0.f ? -1.f : scale == 0.f ? 0.f : 1.f;
    a.out = KvRows{out, o_ts, o_hs};
    a.otype = otype;
    a.arrived = (int *)ws;
    a.partial = ws ? (float *)((char *)ws + HLQ_WS_COUNTER_BYTES) : nullptr;
    a.rows = s.group < 16 ? s.group : 16;
    const int64_t grid = s.workgroups * s.cuts;
    if (grid > ((int64_t)1 << 24) - 1) return HLQ_ERR_UNSUPPORTED;
    const hipStream_t stm = (hipStream_t)stream;
    hlq_clear_stale_error();
    if (s.d.type == HLQ_F16) launch<HLQ_F16, HLQ_F16>(a, grid, stm);
    else if (s.d.type == HLQ_BF16) launch<HLQ_BF16, HLQ_BF16>(a, grid, stm);
    else if (s.d.type == HLQ_MX8) type == HLQ_F16 ? launch<HLQ_MX8, HLQ_F16>(a, grid, stm) : launch<HLQ_MX8, HLQ_BF16>(a, grid, stm);
    else type == HLQ_F16 ? launch<HLQ_MX4, HLQ_F16>(a, grid, stm) : launch<HLQ_MX4, HLQ_BF16>(a, grid, stm);
    return hlq_hip_status(hipGetLastError());
}

}  // extern "C"
