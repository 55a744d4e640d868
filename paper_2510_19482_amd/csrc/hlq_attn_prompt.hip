// Attention of packed prompts:  out_i = sum_j p_ij v_j / sum_j p_ij over the keys j that query i sees,  p_ij = exp(scale q_i . k_j - m_i).
//
// One pass over the keys with the running maximum and sum of each query.  A wavefront has 32 queries of a head, a workgroup four wavefronts: four heads of a
// kv head with the same queries where the group allows, else two, or one with more queries.  Keys and values come through LDS
// in tiles of 32, written there by the loads themselves, three tiles of each.
//   scores    K Q^T with keys the first operand, 32 keys x 32 queries: a lane has 16 keys of one query, so that maximum and sum are the lane's own and
//             one exchange with the lane 32 on
//   weights   are then where the second product, V^T P^T, wants them: its sum over keys may take them in any order
//   values    are turned as they are read from LDS (four keys of a column to a lane)
// A step multiplies the next tile's keys and the last tile's values while it takes the exponentials of this one, so that matrix cores and vector units work side by
// side within a wavefront.  Most steps mask nothing and look at nothing; they have a loop of their own.
// The maximum that exponentials are taken from is kept while no score passes it by 2^8, and is a whole power of two: so sums are rarely multiplied, and exactly.
// Weights are rounded once, to the inputs' type, for the second product; their sum is of the rounded ones, so that a result is a true mean of values.
// What is not seen: its score is -infinity, its weight 0.  A value that is infinite or NaN would still enter as 0 times itself: a workgroup that ends with a NaN (or with scores
// so large that their rounding is felt) goes through its tiles once more, multiplies without such values, and adds what they do to those that see them by counting.
// Rows that do not begin at multiples of 16 bytes go to LDS by way of registers (8192 tokens 534 -> 840 us, of dim 64 310 -> 424; 4096 of dim 256, where that spills, 331 -> 615).
// The look for a NaN, and the barrier that joins it, take 0.4 us of a workgroup; 8192 tokens of which all see a NaN 1390 us.
//
// What bounds it: 8192 bf16 tokens, causal, 32 heads of 128 over 8 take 530 us, 1040 TFLOP/s (a library product reaches 1250 on this card).  Of the cycles the matrix
// cores are busy 50 to 58 %, vector instructions issue in 45 to 55 % (105 a step and wavefront, 16 of them exponentials of 16 cycles each), at 1.7 GHz, the clock that power holds; LDS without its
// bank conflicts (28 % of its time) made 1 % of difference, raised priority none.  Dims of 64 and 256: 890 and 815 TFLOP/s.  Short sequences (16 x 512: 73 us, 470 TFLOP/s) are bound by
// what a workgroup does before its first product and after its last: where it is 0.7 us, queries and first keys 1.9, results 1.2, and the steps at the edge.
#include "hlq_kv.h"

namespace {

constexpr int WAVES = 4, KEYS = 32, STAGES = 3;
constexpr int LEAST_STEPS = 8;                  // of a cut
constexpr int64_t UNITS = 256, MOST_PARTIALS = 4 * UNITS, MOST_CUTS = 128;   // compute units; workgroups that a cut launch makes at most; cuts
constexpr float NONE = -__builtin_inff();

typedef __bf16 bf8v __attribute__((ext_vector_type(8)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef short short4v __attribute__((ext_vector_type(4)));

struct Prompt {
    int B, H, group, D;
    int abreast;   // heads of a workgroup: 4, 2 or 1
    int cuts;      // workgroups that a tile's keys may be cut over
    int *arrived;
    uint64_t *partial;
    int Tq, Tk;
    KvRows q, k, v, out;
    const int32_t *q_offsets, *k_offsets;
    int causal, window;
    float scale, sign;   // the scale's magnitude times log2(e) (1 if it is 0), and its sign
};

// LIFT: what the largest weight is brought to is 2^(LIFT - 1) to 2^LIFT (2^8 times that while the base is kept).  f16 ends at 2^16 and has steps of 2^-24 at its lower end: there weights
// stand as high as they can, so that small ones beside a large one count (16384 keys of which 8 have a score that is 17 higher: without it their share, 8.5e-5, is off by 22 to 44 %).
template <int T> struct Fragment { using type = bf8v; using scalar = __bf16; static constexpr uint32_t EXPONENT = 0x7f807f80u, ONE = 0x00800080u; static constexpr float LIFT = 0.f; };
template <> struct Fragment<HLQ_F16> { using type = half8v; using scalar = _Float16; static constexpr uint32_t EXPONENT = 0x7c007c00u, ONE = 0x04000400u; static constexpr float LIFT = 7.f; };

__device__ __forceinline__ float16v multiply(bf8v a, bf8v b, float16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ float16v multiply(half8v a, half8v b, float16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ float other_half(float v, float &own)
{
    const auto s = __builtin_amdgcn_permlane32_swap(as_bits(v), as_bits(v), false, false);
    own = as_float(s[0]);
    return as_float(s[1]);
}

// c + a + b
__device__ __forceinline__ float add_pair(__bf16 a, __bf16 b, float c)
{
    const mx4_bf2 one = {(__bf16)1.f, (__bf16)1.f};
    return __builtin_amdgcn_fdot2_f32_bf16((mx4_bf2){a, b}, one, c, false);
}
__device__ __forceinline__ float add_pair(_Float16 a, _Float16 b, float c)
{
    const mx4_half2 one = {(_Float16)1.f, (_Float16)1.f};
    return __builtin_amdgcn_fdot2((mx4_half2){a, b}, one, c, false);
}

// 16 bytes a lane from an offset of a descriptor (zeros past its end) to LDS at `to`, lane after lane
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t r, int offset, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(offset), "s"(r), "s"(__builtin_amdgcn_readfirstlane(to)) : "memory", "m0");
}

// sequence and tile of a workgroup; every lane of the wavefront takes part and gets the same answer
struct Place {
    int q0, n_q, k0, n_k;   // rows of the sequence
    int first;              // query of the tile's first row; n_q = 0: there are fewer tiles
};
__device__ __forceinline__ Place place_of(const Prompt &a, int tile, int rows)
{
    const int lane = (int)(threadIdx.x & 63u);
    // offsets are device data: whatever they hold, rows stay inside
    auto offset = [](const int32_t *o, int i, int most) { const int v = o[i]; return v < 0 ? 0 : v > most ? most : v; };
    if (a.B == 1) {
        const int lo = offset(a.q_offsets, 0, a.Tq), n = offset(a.q_offsets, 1, a.Tq) - lo, k0 = offset(a.k_offsets, 0, a.Tk), n_k = offset(a.k_offsets, 1, a.Tk) - k0;
        const int first = ((n < 0 ? 0 : n) - 1) / rows * rows - tile * rows;
        return {lo, n > 0 && first >= 0 ? n : 0, k0, n_k < 0 ? 0 : n_k, first};
    }
    int before = 0;
    for (int at = 0; at < a.B; at += 64) {
        const int b = at + lane;
        int lo = 0, n = 0, k0 = 0, n_k = 0;
        if (b < a.B) {
            lo = offset(a.q_offsets, b, a.Tq);
            n = offset(a.q_offsets, b + 1, a.Tq) - lo;
            k0 = offset(a.k_offsets, b, a.Tk);
            n_k = offset(a.k_offsets, b + 1, a.Tk) - k0;
            n = n < 0 ? 0 : n;
            n_k = n_k < 0 ? 0 : n_k;
        }
        const int mine = n / rows + (n % rows > 0);
        int upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
        }
        const int all = __builtin_amdgcn_readlane(upto, 63);
        if (tile - before < all) {
            const int f = (int)__builtin_ctzll(__ballot(upto > tile - before));
            // of a sequence the last tile first: it sees most keys
            return {__builtin_amdgcn_readlane(lo, f), __builtin_amdgcn_readlane(n, f), __builtin_amdgcn_readlane(k0, f), __builtin_amdgcn_readlane(n_k, f),
                    (__builtin_amdgcn_readlane(upto, f) - 1 - (tile - before)) * rows};
        }
        before += all;
    }
    return {0, 0, 0, 0, 0};
}

// DMA: rows of keys and values begin at multiples of 16 bytes
template <int T, int DP, bool DMA>
__global__ void __launch_bounds__(64 * WAVES, DP > 128 ? 1 : DP > 64 ? 2 : 3)
hlq_attn_prompt_kernel(const Prompt a)
{
    using F = typename Fragment<T>::type;
    using S = typename Fragment<T>::scalar;
    constexpr int KS = DP / 16, DS = DP / 32;
    constexpr int ROW = DP * 2, PIECES = DP / 8, TILE = KEYS * ROW;     // bytes; 16-byte pieces of a row
    constexpr int LOADS = TILE / 1024 / WAVES;                          // of a wavefront, 1024 bytes each, of keys and as many of values
    __shared__ __attribute__((aligned(1024))) char lds[2 * STAGES * TILE];
    const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;

    const int lane = (int)(threadIdx.x & 63u), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int col = lane & 31, half = lane >> 5;
    int id = (int)blockIdx.x;
    const int h = id % a.H;   // kv heads in turn: one each XCD where there are eight
    id /= a.H;
    const int cut = id % a.cuts;
    id /= a.cuts;
    const int sets = a.group / a.abreast, set = id % sets;
    const int rows = 32 * (WAVES / a.abreast);                 // queries of a workgroup
    const Place p = place_of(a, id / sets, rows);
    if (p.n_q == 0) return;
    const int head = h * a.group + set * a.abreast + wave % a.abreast;
    const int row0 = wave / a.abreast * 32;                    // of this wavefront in the tile

    const int shift = p.n_k - p.n_q;                                    // place of query 0
    const int tile_rows = p.n_q - p.first < rows ? p.n_q - p.first : rows;
    // steps of 32 keys that some query of rows [from, from + n) sees
    auto steps_of = [&](int from, int n, int &begin, int &end) {
        int last = p.n_k;
        if (a.causal) last = shift + p.first + from + n < last ? shift + p.first + from + n : last;
        int first = 0;
        if (a.window > 0) {
            const int64_t lowest = (int64_t)shift + p.first + from - a.window + 1;
            first = lowest > 0 ? (int)lowest : 0;
        }
        begin = first / KEYS;
        end = n > 0 && last > first ? (last + KEYS - 1) / KEYS : begin;
    };
    int all_begin, all_end, begin, end;
    steps_of(0, tile_rows, all_begin, all_end);
    // this workgroup's share of them; one at least has one, which writes zeros where nothing is seen
    int active = 1;
    if (a.cuts > 1) {
        const int steps = all_end - all_begin;
        int share = (steps + a.cuts - 1) / a.cuts;
        share = share < LEAST_STEPS ? LEAST_STEPS : share;
        active = steps > share ? (steps + share - 1) / share : 1;
        if (cut >= active) return;
        all_begin += cut * share;
        all_end = all_begin + share < all_end ? all_begin + share : all_end;
    }
    const int own_rows = tile_rows - row0 < 0 ? 0 : tile_rows - row0 < 32 ? tile_rows - row0 : 32;
    steps_of(row0, own_rows, begin, end);
    begin = begin < all_begin ? all_begin : begin;
    end = end > all_end ? all_end : end;

    const int first_place = shift + p.first + row0;                     // of the wavefront's first query

    // Tiles in LDS: row after row, a row's 16-byte pieces in another order, so that reads meet every bank evenly: piece c of key k at c ^ (k & 7), of a
    // value's row at c ^ 2 (k & 3).  A lane loads what belongs in its place.
    constexpr int OUTSIDE = 0x7fffffff;
    const int key_step = (int)(a.k.ts * 2), value_step = (int)(a.v.ts * 2);   // bytes from row to row (DMA)
    int at_key[LOADS], key_piece[LOADS], value_piece[LOADS], key_at[LOADS], value_at[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        at_key[i] = (wave * LOADS + i) * (64 / PIECES) + lane / PIECES;
        key_piece[i] = (lane % PIECES ^ (at_key[i] & 7)) * 8;
        value_piece[i] = (lane % PIECES ^ (at_key[i] & 3) << 1) * 8;
        key_at[i] = key_piece[i] < a.D ? at_key[i] * key_step + key_piece[i] * 2 : OUTSIDE;
        value_at[i] = value_piece[i] < a.D ? at_key[i] * value_step + value_piece[i] * 2 : OUTSIDE;
    }
    // what the next requests read: tiles of keys or values one after the other, nothing behind the last key that somebody sees
    struct Feed {
        const char *from;
        int64_t step;
        int left;
    };
    const int limit = all_end * KEYS < p.n_k ? all_end * KEYS : p.n_k;
    auto feed = [&](const KvRows &x) {
        const int first = all_begin * KEYS;
        return Feed{(const char *)((const S *)x.p + (int64_t)(p.k0 + first) * x.ts + h * x.hs), x.ts * 2 * KEYS, limit - first};
    };
    mx4_u4 kept[DMA ? 1 : 2 * LOADS];
    auto request = [&](bool of_keys, Feed &f, uint32_t slot) {
        const int n = f.left < 0 ? 0 : f.left < KEYS ? f.left : KEYS;
        if constexpr (DMA) {
            const int step = of_keys ? key_step : value_step, bytes = n * step - (step - a.D * 2);   // rows are no nearer than their length
            const auto r = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(f.from), 0, bytes > 0 ? bytes : 0, 0x00020000);
            const uint32_t to = lds_at + slot + wave * LOADS * 1024;
#pragma unroll
            for (int i = 0; i < LOADS; ++i) load_to_lds(r, of_keys ? key_at[i] : value_at[i], to + i * 1024);
        } else {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int piece = of_keys ? key_piece[i] : value_piece[i];
                kept[of_keys ? i : LOADS + i] = at_key[i] < n && piece < a.D ? *(const mx4_u4_any *)(f.from + (at_key[i] * (of_keys ? a.k.ts : a.v.ts) + piece) * 2) : (mx4_u4){0u, 0u, 0u, 0u};
            }
        }
        f.from += f.step;
        f.left -= KEYS;
    };
    auto enter = [&](bool of_keys, uint32_t slot) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) *(mx4_u4 *)(lds + slot + (wave * LOADS + i) * 1024 + lane * 16) = kept[of_keys ? i : LOADS + i];
    };

    // reads: a key's pieces 2 s + half, and four keys of a column of values
    int key_read[4], value_read[2];
#pragma unroll
    for (int s = 0; s < 4; ++s) key_read[s] = col * ROW + ((2 * s + half) ^ (col & 7)) * 16;
    {
        const int i = lane & 15, c = ((lane >> 4) & 1) * 2 + ((i & 3) >> 1), turn = (i >> 2) << 1;
#pragma unroll
        for (int j = 0; j < 2; ++j) value_read[j] = (4 * half + (i >> 2)) * ROW + ((4 * j + c) ^ turn) * 16 + (i & 1) * 8;
    }
    auto key = [&](uint32_t slot, int s) { return *(const F *)(lds + slot + key_read[s & 3] + (s >> 2) * 128); };
    auto value = [&](uint32_t slot, int j, int u) {
        typedef __attribute__((address_space(3))) short4v *Four;
        const char *at = lds + slot + value_read[j & 1] + (j >> 1) * 128 + 16 * u * ROW;
        struct { short4v v[2]; } two;
        two.v[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Four)at);
        two.v[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Four)(at + 8 * ROW));
        return __builtin_bit_cast(F, two);
    };

    float16v acc[DS];
    float base, most, total;   // most: scores up to it need no new base
    const auto clear = [&]() {
        base = 0.f, most = NONE, total = 0.f;
#pragma unroll
        for (int j = 0; j < DS; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[j][i] = 0.f;
    };
    clear();
    // steps of which every query of the wavefront sees every key
    const int last_place = first_place + own_rows - 1;
    int full_end = p.n_k;
    if (a.causal && first_place + 1 < full_end) full_end = first_place + 1;
    full_end = full_end < 0 ? 0 : full_end / KEYS;
    const int full_begin = a.window > 0 && last_place >= a.window ? (last_place - a.window) / KEYS + 1 : 0;
    auto edge = [&](int step) { return step < full_begin || step >= full_end; };
    // the keys that this lane's query sees; of a step the lane's keys are 4 half + offset_of(i)
    const int place = first_place + col, last_seen = a.causal && place < p.n_k ? place : p.n_k - 1, first_seen = a.window > 0 ? place - a.window + 1 : 0;
    const auto offset_of = [](int i) { return 8 * (i >> 2) + (i & 3); };
    struct Seen {
        int first, last;   // offsets
        __device__ __forceinline__ bool operator()(int offset) const { return offset <= last && offset >= first; }
    };
    auto seen_of = [&](int step) { return Seen{first_seen - step * KEYS - 4 * half, last_seen - step * KEYS - 4 * half}; };

    auto multiply_values = [&](const F (&weight)[2], uint32_t slot) {
#pragma unroll
        for (int j = 0; j < DS; ++j)
#pragma unroll
            for (int u = 0; u < 2; ++u) acc[j] = multiply(value(slot, j, u), weight[u], acc[j]);
    };
    // values that are numbers as above; +infinity, and -infinity, and NaN as both, once for each query that sees one (`present`: the lane's keys that do)
    auto multiply_odd_values = [&](const F (&weight)[2], uint32_t present, uint32_t slot) {
#pragma unroll
        for (int j = 0; j < DS; ++j) {
            F c[2];
            uint32_t found = 0;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                c[u] = value(slot, j, u);
                const mx4_u4 w = __builtin_bit_cast(mx4_u4, c[u]);
#pragma unroll
                for (int i = 0; i < 4; ++i) found |= (w[i] & Fragment<T>::EXPONENT) + Fragment<T>::ONE;
            }
            if (__any((found & 0x80008000u) != 0u)) {
#pragma unroll
                for (int sign = 0; sign < 2; ++sign) {
                    float16v count;
#pragma unroll
                    for (int i = 0; i < 16; ++i) count[i] = 0.f;
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        F is, sees;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float f = (float)c[u][e];
                            is[e] = (S)((sign ? f > NONE : f < __builtin_inff()) ? 0.f : 1.f);
                            sees[e] = (S)(present >> (8 * u + e) & 1u ? 1.f : 0.f);
                        }
                        count = multiply(is, sees, count);
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (count[i] > 0.f) acc[j][i] += sign ? NONE : __builtin_inff();
                }
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (!(fabsf((float)c[u][e]) < __builtin_inff())) c[u][e] = (S)0.f;
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) acc[j] = multiply(c[u], weight[u], acc[j]);
        }
    };
    // sees to it that scores are at most 2^8 times what the exponentials are taken from; `weight`, not yet multiplied, goes by that too
    auto keep_up = [&](const float16v &score, F (&weight)[2]) {
        float m = score[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) m = fmaxf(m, score[i]);
        float own;
        const float other = other_half(m, own);
        m = fmaxf(own, other) * a.scale;
        if (__builtin_expect(__any(m > most), 0)) {
            const bool now = m > most;
            const float to = now ? ceilf(m) - Fragment<T>::LIFT : base;
            const float keep = !now || most == NONE ? 1.f : exp2_above_0(base - to);
            base = to;
            most = now ? to + (Fragment<T>::LIFT + 8.f) : most;
            total *= keep;
#pragma unroll
            for (int j = 0; j < DS; ++j)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[j][i] *= keep;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 8; ++e) weight[u][e] = (S)((float)weight[u][e] * keep);
        }
    };
    auto two_exponentials = [&](const float16v &score, F (&weight)[2], int i, auto careful) {
        const auto of = [&](float x) { return (S)__builtin_amdgcn_exp2f(decltype(careful)::value ? above_base(x, a.scale, base) : fmaf(x, a.scale, -base)); };
        const S w0 = of(score[i]), w1 = of(score[i + 1]);
        weight[i >> 3][i & 7] = w0;
        weight[i >> 3][(i & 7) + 1] = w1;
        total = add_pair(w0, w1, total);
    };
    auto exponentials = [&](const float16v &score, F (&weight)[2], auto careful) {
#pragma unroll
        for (int i = 0; i < 16; i += 2) two_exponentials(score, weight, i, careful);
    };

    // The first pass looks at no value.  What an infinite or NaN value makes of the weights of those that do not see it, 0 times itself, shows as NaN; then the workgroup takes a
    // careful one, which looks at each tile, and adds infinities by counting for who sees them: with a score above -infinity, however small the weight.
    const auto pass = [&](auto careful) {
        constexpr bool CAREFUL = decltype(careful)::value;
        // Step t multiplies the keys of t + 1 and the values of t - 1, takes the exponentials of t, and requests the keys of t + 3 and the values of t + 1.
        // Three slots of each: t's is `here`, t + 1's `ahead`, t - 1's `behind`.
        constexpr uint32_t OF_VALUES = STAGES * TILE;
        Feed key_feed = feed(a.k), value_feed = feed(a.v);
        uint32_t here = 2 * TILE, ahead = 0, behind = TILE;
        float16v score;
        F weight[2];
        uint32_t present = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) score[i] = 0.f, weight[i >> 3][i & 7] = (S)0.f;
        // queries, the second operand: whole rows by way of the slots that nothing is in yet, with their pieces as a key's
        F query[KS];
        const S *const q = (const S *)a.q.p + (int64_t)(p.q0 + p.first + row0) * a.q.ts + head * a.q.hs;
        if constexpr (DMA) {
            const int step = (int)(a.q.ts * 2), bytes = own_rows > 0 && a.sign != 0.f ? (own_rows - 1) * step + a.D * 2 : 0;
            const auto r = __builtin_amdgcn_make_buffer_rsrc(const_cast<S *>(q), 0, bytes, 0x00020000);
#pragma unroll
            for (int i = 0; i < 32 * PIECES / 64; ++i) {
                const int at = i * (64 / PIECES) + lane / PIECES, piece = (lane % PIECES ^ (at & 7)) * 8;
                load_to_lds(r, piece < a.D ? at * step + piece * 2 : OUTSIDE, lds_at + here + wave * 32 * ROW + i * 1024);
            }
        } else {
#pragma unroll
            for (int s = 0; s < KS; ++s) query[s] = __builtin_bit_cast(F, col < own_rows && a.sign != 0.f && 16 * s + 8 * half < a.D ? *(const mx4_u4_any *)(q + col * a.q.ts + 16 * s + 8 * half) : (mx4_u4){0u, 0u, 0u, 0u});
        }
        request(true, key_feed, ahead);
        if constexpr (!DMA) enter(true, ahead);
        request(true, key_feed, behind);
        if constexpr (!DMA && CAREFUL) enter(true, behind);
        if constexpr (DMA) {
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * LOADS) : "memory");
#pragma unroll
            for (int s = 0; s < KS; ++s) query[s] = key(here + wave * 32 * ROW, s);
        }
        // of a negative scale they have the sign, so that the largest score has the largest product
        if (a.sign < 0.f) {
#pragma unroll
            for (int s = 0; s < KS; ++s) query[s] = __builtin_bit_cast(F, __builtin_bit_cast(mx4_u4, query[s]) ^ 0x80008000u);
        }
        auto multiply_keys = [&](float16v &score, uint32_t slot) {
#pragma unroll
            for (int i = 0; i < 16; ++i) score[i] = 0.f;
#pragma unroll
            for (int s = 0; s < KS; ++s) score = multiply(key(slot, s), query[s], score);
        };
        int t = all_begin - 1;
        auto meet = [&](bool first) {
            if constexpr (DMA) {
                // what was requested the step before last is there
                if (first) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LOADS) : "memory");
                else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * LOADS) : "memory");
            } else {
                __syncthreads();
                if constexpr (!CAREFUL) {
                    enter(true, behind);
                    if (!first) enter(false, OF_VALUES + here);
                }
            }
            request(true, key_feed, here);
            if constexpr (!DMA && CAREFUL) enter(true, here);   // (a careful pass keeps nothing on its way: registers)
            request(false, value_feed, OF_VALUES + ahead);
            if constexpr (!DMA && CAREFUL) enter(false, OF_VALUES + ahead);
        };
        auto advance = [&]() {
            const uint32_t was = behind;
            behind = here;
            here = ahead;
            ahead = was;
            ++t;
        };
        // The step between two barriers: `score` becomes `later`, the keys ahead `next`, and the values behind are added by `weight`.  Dim above 128 has one wavefront a
        // SIMD, so there its order is laid down: reads from LDS stand four products before their use, two exponentials behind each four (4096 tokens of dim 256 354 -> 337 us).
        auto multiply_both = [&](const float16v &score, float16v &next, const F (&weight)[2], F (&later)[2]) {
            if constexpr (DP <= 128) {
                multiply_keys(next, ahead);
                multiply_values(weight, OF_VALUES + behind);
                exponentials(score, later, careful);
            } else {
                constexpr int FOURS = KS / 4;
                F read[2][4];
                auto fetch = [&](int n) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) read[n & 1][e] = n < FOURS ? key(ahead, 4 * n + e) : value(OF_VALUES + behind, 2 * (n - FOURS) + e / 2, e & 1);
                };
                fetch(0);
#pragma unroll
                for (int i = 0; i < 16; ++i) next[i] = 0.f;
#pragma unroll
                for (int n = 0; n < 2 * FOURS; ++n) {
                    if (n + 1 < 2 * FOURS) fetch(n + 1);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (n < FOURS) next = multiply(read[n & 1][e], query[4 * n + e], next);
                        else {
                            float16v &sum = acc[2 * (n - FOURS) + e / 2];
                            sum = multiply(read[n & 1][e], weight[e & 1], sum);
                        }
                    }
                    two_exponentials(score, later, 2 * n, careful);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        };
        // most of a long prompt: nothing to mask, nothing to look at
        const int hot_begin = begin + 1 > full_begin + 1 ? begin + 1 : full_begin + 1, hot_end = end - 1 < full_end ? end - 1 : full_end;
        while (t <= all_end) {
            if (!CAREFUL && t >= hot_begin && t + 1 < hot_end) {
                do {
                    float16v next;
                    F later[2];
                    meet(false);
                    keep_up(score, weight);
                    multiply_both(score, next, weight, later);
                    advance();
                    meet(false);
                    keep_up(next, later);
                    multiply_both(next, score, later, weight);
                    advance();
                } while (t + 1 < hot_end);
                continue;
            }
            meet(t < all_begin);
            if (DP > 128 && (t + 1 < begin || t > end)) {   // (below, such registers are spilled that a wavefront without queries would wait for every load)
                advance();
                continue;
            }
            const bool ask = t + 1 >= begin && t + 1 < end, weigh = t >= begin && t < end, sum = t - 1 >= begin && t - 1 < end;
            // a careful pass scales and adds in the order of the first, so that results are the same bits
            const bool was_hot = CAREFUL && t >= hot_begin && t - ((t - hot_begin) & 1) + 1 < hot_end;
            if (CAREFUL && was_hot) keep_up(score, weight);
            if (sum) {
                if constexpr (CAREFUL) multiply_odd_values(weight, present, OF_VALUES + behind);
                else multiply_values(weight, OF_VALUES + behind);
            }
            if (weigh) {
                if (edge(t)) {
                    const Seen seen = seen_of(t);
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (!seen(offset_of(i))) score[i] = NONE;
                }
                if (!CAREFUL || !was_hot) keep_up(score, weight);
                if constexpr (CAREFUL) {
                    present = 0;
#pragma unroll
                    for (int i = 0; i < 16; ++i) present |= (uint32_t)(score[i] > NONE) << i;
                }
                exponentials(score, weight, careful);
            }
            if (ask) multiply_keys(score, ahead);
            advance();
        }
        if constexpr (DMA) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    };
    if (all_begin < all_end) {
        __shared__ int found[WAVES];
        pass(std::false_type());
        bool odd = !(total < __builtin_inff()) || fabsf(base) >= LARGE;
#pragma unroll
        for (int j = 0; j < DS; ++j)
#pragma unroll
            for (int i = 0; i < 16; i += 2) odd = odd || __builtin_isunordered(acc[j][i], acc[j][i + 1]);
        const bool any = __any(odd && col < own_rows);
        if (lane == 0) found[wave] = any;
        __syncthreads();
        if (__builtin_expect(__builtin_amdgcn_readfirstlane(found[0] | found[1] | found[2] | found[3]), 0)) {
            clear();
            pass(std::true_type());
            __syncthreads();
        }
    }
    if (active > 1) {
        // Cut: sums, and the base and total, past the XCD's own L2 (device-scope stores, complete before the arrival is counted); whoever is last adds the
        // cuts in their order.  Bases are whole powers of two: so the sums are brought to the largest exactly.
        constexpr int PAIRS = DS * 8 + 1;
        const int64_t who = blockIdx.x / (a.cuts * a.H) * a.H + h;
        uint64_t *const every = a.partial + (who * a.cuts * WAVES + wave) * (PAIRS * 64) + lane;
        uint64_t *const mine = every + (int64_t)cut * WAVES * (PAIRS * 64);
        const auto pair = [](float x, float y) { return as_bits(x) | (uint64_t)as_bits(y) << 32; };
#pragma unroll
        for (int j = 0; j < DS; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) __hip_atomic_store(mine + (j * 8 + i) * 64, pair(acc[j][2 * i], acc[j][2 * i + 1]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(mine + DS * 8 * 64, pair(most == NONE ? NONE : base, total), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        int *const last = (int *)lds;
        if (threadIdx.x == 0) *last = __hip_atomic_fetch_add(a.arrived + who, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == active - 1;
        __syncthreads();
        if (!*last) return;
        if (threadIdx.x == 0) __hip_atomic_store(a.arrived + who, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const auto from = [&](int c, int i) { return __hip_atomic_load(every + ((int64_t)c * WAVES * PAIRS + i) * 64, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
        float highest = NONE;
        for (int c = 0; c < active; ++c) highest = fmaxf(highest, as_float((uint32_t)from(c, DS * 8)));
        highest = highest == NONE ? 0.f : highest;
        total = 0.f;
#pragma unroll
        for (int j = 0; j < DS; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[j][i] = 0.f;
        for (int c = 0; c < active; ++c) {
            const uint64_t of = from(c, PAIRS - 1);
            const float weight = exp2_above_0(as_float((uint32_t)of) - highest);
            total = fmaf(weight, as_float((uint32_t)(of >> 32)), total);
            constexpr int AT_ONCE = DS < 4 ? DS : 4;   // of 32 columns, on their way together
#pragma unroll
            for (int j0 = 0; j0 < DS; j0 += AT_ONCE) {
                uint64_t in[AT_ONCE * 8];
#pragma unroll
                for (int i = 0; i < AT_ONCE * 8; ++i) in[i] = from(c, j0 * 8 + i);
#pragma unroll
                for (int i = 0; i < AT_ONCE * 8; ++i) {
                    float16v &sum = acc[j0 + i / 8];
                    sum[2 * (i % 8)] = fmaf(weight, as_float((uint32_t)in[i]), sum[2 * (i % 8)]);
                    sum[2 * (i % 8) + 1] = fmaf(weight, as_float((uint32_t)(in[i] >> 32)), sum[2 * (i % 8) + 1]);
                }
            }
        }
    }
    float own;
    const float other = other_half(total, own);
    const float all = own + other, by = all == 0.f ? 0.f : 1.f / all;
    if (__any(all == 0.f)) {   // a query that has seen nothing: 0, whatever the values are
#pragma unroll
        for (int j = 0; j < DS; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[j][i] = all == 0.f ? 0.f : acc[j][i];
    }
    // by way of LDS, so that whole rows leave (nothing of the tiles is read any more)
    constexpr int TURN = PIECES < 16 ? PIECES - 1 : 15;
    char *const mine = lds + wave * 32 * ROW;
    if (active > 1) __syncthreads();   // (else one stands behind the last tile)
#pragma unroll
    for (int j = 0; j < DS; ++j)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            typedef S four __attribute__((ext_vector_type(4)));
            *(four *)(mine + col * ROW + ((4 * j + i / 4) ^ (col & TURN)) * 16 + 8 * half) = (four){(S)(acc[j][i] * by), (S)(acc[j][i + 1] * by), (S)(acc[j][i + 2] * by), (S)(acc[j][i + 3] * by)};
        }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");   // the lanes of a wavefront read what others of it wrote
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    S *const out = (S *)a.out.p + (int64_t)(p.q0 + p.first + row0) * a.out.ts + head * a.out.hs;
#pragma unroll
    for (int i = 0; i < 32 * PIECES / 64; ++i) {
        const int row = i * (64 / PIECES) + lane / PIECES, piece = lane % PIECES;
        if (row < own_rows && piece * 8 < a.D) *(mx4_u4_any *)(out + row * a.out.ts + piece * 8) = *(const mx4_u4 *)(mine + row * ROW + (piece ^ (row & TURN)) * 16);
    }
}

template <int T, bool DMA>
void launch(const Prompt &a, int64_t grid, hipStream_t st)
{
    const dim3 g((unsigned)grid), block(64 * WAVES);
    if (a.D <= 64) hlq_attn_prompt_kernel<T, 64, DMA><<<g, block, 0, st>>>(a);
    else if (a.D <= 128) hlq_attn_prompt_kernel<T, 128, DMA><<<g, block, 0, st>>>(a);
    else hlq_attn_prompt_kernel<T, 256, DMA><<<g, block, 0, st>>>(a);
}

struct Shape {
    int abreast, cuts;
    int64_t workgroups;   // of a launch that is not cut
    size_t bytes;         // of the workspace, enough for fewer rows and sequences too
};
hlq_status shape_of(int64_t Tq, int64_t Tk, int32_t B, int32_t q_heads, int32_t heads, int32_t dim, Shape *out)
{
    if (Tq < 0 || Tk < 0 || B < 0 || heads < 1 || q_heads < 1 || q_heads % heads || dim < 8 || dim % 8) return HLQ_ERR_BAD_DESC;
    constexpr int64_t MOST = (int64_t)1 << 30;
    if (Tq >= MOST || Tk >= MOST || B >= MOST || q_heads > KV_MOST_HEADS || dim > KV_MOST_DIM) return HLQ_ERR_UNSUPPORTED;
    Shape s{};
    const int group = q_heads / heads;
    s.abreast = group % 4 == 0 ? 4 : group % 2 == 0 ? 2 : 1;
    // never more tiles than the queries can make, whatever the offsets hold
    const int rows = 32 * (WAVES / s.abreast);
    s.workgroups = (Tq + (Tq < B ? Tq : B) * (rows - 1)) / rows * (q_heads / s.abreast);
    if (s.workgroups > ((int64_t)1 << 24) - 1) return HLQ_ERR_UNSUPPORTED;   // a launch has fewer than 2^32 lanes
    // Few queries over many keys: the keys are cut as many times as the compute unit with most to do then has least (sequences taken as of one length).  In
    // tenths of a step of one of two workgroups of a unit: alone it takes 13 (dim above 128 always), it begins and ends in five steps, a joined tile takes eight and five a cut.
    // (32 heads of 128, 8 of keys: 512 queries over 8192 keys whole 158 us, in 2, 3, 4, 6, 8 cuts 95, 94, 83, 104, 109; 32 over 4096: 77, in 4, 8, 16 cuts 33, 30, 38; over 512: 16, in two 16.5.)
    const int DP = dim <= 64 ? 64 : dim <= 128 ? 128 : 256;
    const int64_t most = (Tk + KEYS * LEAST_STEPS - 1) / (KEYS * LEAST_STEPS), some = Tq < B ? Tq : B;
    const int64_t steps = some > 0 ? (Tk / some + KEYS - 1) / KEYS : 0, likely = some > 0 ? some * ((Tq / some + rows - 1) / rows) * (q_heads / s.abreast) : 0;
    int64_t best = 0;
    s.cuts = 1;
    for (int64_t cuts = 1; cuts <= MOST_CUTS && (cuts == 1 || (cuts <= most && s.workgroups * cuts <= MOST_PARTIALS)); ++cuts) {
        const int64_t each = (likely * cuts + UNITS - 1) / UNITS, pace = DP > 128 ? 13 * each : 10 * each + (each & 1) * 3;
        const int64_t cost = ((steps + cuts - 1) / cuts + 5) * pace + (cuts > 1 ? 80 + 50 * cuts : 0);
        if (cuts == 1 || cost < best) best = cost, s.cuts = (int)cuts;
    }
    const int64_t partials = most < 2 ? 0 : s.workgroups * most < MOST_PARTIALS ? s.workgroups * most : MOST_PARTIALS;
    s.bytes = HLQ_WS_COUNTER_BYTES + (size_t)partials * WAVES * 64 * (DP / 4 + 1) * 8u;
    *out = s;
    return HLQ_OK;
}

}  // namespace

extern "C" {

hlq_status hlq_attn_prompt_workspace_bytes(int64_t Tq, int64_t Tk, int32_t B, int32_t q_heads, int32_t heads, int32_t dim, size_t *bytes)
{
    Shape shape;
    const hlq_status s = shape_of(Tq, Tk, B, q_heads, heads, dim, &shape);
    if (s != HLQ_OK) return s;
    if (!bytes) return HLQ_ERR_NULL;
    *bytes = shape.bytes;
    return HLQ_OK;
}

hlq_status hlq_attn_prompt(int32_t B, int32_t q_heads, int32_t heads, int32_t dim, hlq_dtype type, int64_t Tq, const void *q, int64_t q_ts, int64_t q_hs,
                           int64_t Tk, const void *k, int64_t k_ts, int64_t k_hs, const void *v, int64_t v_ts, int64_t v_hs, const int32_t *q_offsets,
                           const int32_t *k_offsets, int32_t causal, int32_t window, float scale, void *out, int64_t o_ts, int64_t o_hs, void *ws,
                           size_t ws_bytes, void *stream)
{
    Shape shape;
    hlq_status s = shape_of(Tq, Tk, B, q_heads, heads, dim, &shape);
    if (s != HLQ_OK) return s;
    if (type != HLQ_F16 && type != HLQ_BF16) return HLQ_ERR_UNSUPPORTED;
    if (window < 0) return HLQ_ERR_BAD_DESC;
    if (Tq == 0 || B == 0) return HLQ_OK;
    if (!q_offsets || !k_offsets) return HLQ_ERR_NULL;
    if (((uintptr_t)q_offsets | (uintptr_t)k_offsets) & 3u) return HLQ_ERR_BAD_STRIDE;
    if ((s = hlq_check_rows(q, Tq, q_heads, dim, q_ts, q_hs, type, false)) != HLQ_OK) return s;
    if ((s = hlq_check_rows(out, Tq, q_heads, dim, o_ts, o_hs, type, true)) != HLQ_OK) return s;
    if (Tk > 0) {
        if ((s = hlq_check_rows(k, Tk, heads, dim, k_ts, k_hs, type, false)) != HLQ_OK) return s;
        if ((s = hlq_check_rows(v, Tk, heads, dim, v_ts, v_hs, type, false)) != HLQ_OK) return s;
    }
    if (shape.cuts > 1) {
        if (!ws) return HLQ_ERR_NULL;
        if ((uintptr_t)ws & 15u) return HLQ_ERR_BAD_STRIDE;
        if (ws_bytes < shape.bytes) return HLQ_ERR_BUFFER_TOO_SMALL;
    }
    const KvSpan to = hlq_span(out, Tq, q_heads, o_ts, o_hs, type);
    if (hlq_rows_in_the_way(hlq_span(q, Tq, q_heads, q_ts, q_hs, type), to, dim) || hlq_rows_overlap(hlq_span(k, Tk, heads, k_ts, k_hs, type), to, dim) ||
        hlq_rows_overlap(hlq_span(v, Tk, heads, v_ts, v_hs, type), to, dim))
        return HLQ_ERR_BAD_STRIDE;
    Prompt a{};
    a.B = B;
    a.H = heads;
    a.group = q_heads / heads;
    a.D = dim;
    a.Tq = (int)Tq;
    a.Tk = (int)Tk;
    a.q = KvRows{const_cast<void *>(q), q_ts, q_hs};
    a.k = KvRows{const_cast<void *>(k), k_ts, k_hs};
    a.v = KvRows{const_cast<void *>(v), v_ts, v_hs};
    a.out = KvRows{out, o_ts, o_hs};
    a.q_offsets = q_offsets;
    a.k_offsets = k_offsets;
    a.causal = causal != 0;
    a.window = window < Tk ? window : 0;   // no sequence is longer
    a.scale = scale == 0.f ? 1.f : fabsf(scale) * 1.44269504f;
    a.sign = scale < 0.f ? -1.f : scale == 0.f ? 0.f : 1.f;
    a.abreast = shape.abreast;
    a.cuts = shape.cuts;
    a.arrived = (int *)ws;
    a.partial = ws ? (uint64_t *)((char *)ws + HLQ_WS_COUNTER_BYTES) : nullptr;
    const int64_t grid = shape.workgroups * shape.cuts;
    // loads that go to LDS by themselves: rows at multiples of 16 bytes, no nearer than their length, a tile's offsets in 31 bits
    const auto whole = [&](const KvRows &x) { return x.ts >= dim && ((uintptr_t)x.p & 15u) == 0 && x.ts % 8 == 0 && x.hs % 8 == 0 && x.ts < 1 << 23; };
    const bool dma = whole(a.q) && whole(a.k) && whole(a.v);
    const hipStream_t st = (hipStream_t)stream;
    hlq_clear_stale_error();
    if (type == HLQ_F16) dma ? launch<HLQ_F16, true>(a, grid, st) : launch<HLQ_F16, false>(a, grid, st);
    else dma ? launch<HLQ_BF16, true>(a, grid, st) : launch<HLQ_BF16, false>(a, grid, st);
    return hlq_hip_status(hipGetLastError());
}

}  // extern "C"
