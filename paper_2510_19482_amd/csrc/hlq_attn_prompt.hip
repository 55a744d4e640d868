// Attention of packed prompts:  out_i = sum_j p_ij v_j / sum_j p_ij over the keys j that query i sees,  p_ij = exp(scale q_i . k_j - m_i).
//
// One pass over the keys with the running maximum and sum of each query.  A workgroup has 128 queries of one head of one sequence, a wavefront 32 of them;
// keys and values come in tiles of 64 (32 for dim above 128) by way of registers, the next tile's on their way while this one is multiplied.
//   scores    K Q^T with keys the first operand, 32 keys x 32 queries: a lane has 16 keys of one query, so that maximum and sum are the lane's own and
//             one exchange with the lane 32 on
//   weights   are then where the second product, V^T P^T, wants them: its sum over keys may take them in any order
//   values    are turned as they enter LDS, four keys of a column next to each other in the order in which the weights stand
// What is not seen: its score is -infinity, its weight 0.  A value that is infinite or NaN would still enter as 0 times itself, so tiles at the edge of
// what is seen are looked at as they are loaded, and one that holds such a value is multiplied without it; what it does to those that do see it
// is added by counting.
#include "hlq_kv.h"

namespace {

constexpr int WAVES = 4, ROWS = 32 * WAVES;
constexpr float NONE = -__builtin_inff();

typedef __bf16 bf8v __attribute__((ext_vector_type(8)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef float float16v __attribute__((ext_vector_type(16)));

struct Prompt {
    int B, H, group, D;
    int Tq, Tk;
    KvRows q, k, v, out;
    const int32_t *q_offsets, *k_offsets;
    int causal, window;
    float scale;   // times log2(e)
};

template <int T> struct Fragment { using type = bf8v; using scalar = __bf16; static constexpr uint32_t EXPONENT = 0x7f807f80u, ONE = 0x00800080u; };
template <> struct Fragment<HLQ_F16> { using type = half8v; using scalar = _Float16; static constexpr uint32_t EXPONENT = 0x7c007c00u, ONE = 0x04000400u; };

__device__ __forceinline__ float16v multiply(bf8v a, bf8v b, float16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ float16v multiply(half8v a, half8v b, float16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ float other_half(float v, float &own)
{
    const auto s = __builtin_amdgcn_permlane32_swap(as_bits(v), as_bits(v), false, false);
    own = as_float(s[0]);
    return as_float(s[1]);
}
__device__ __forceinline__ float base_of(float m) { return m == NONE ? 0.f : m; }

// sequence and tile of a workgroup; every lane of the wavefront takes part and gets the same answer
struct Place {
    int q0, n_q, k0, n_k;   // rows of the sequence
    int first;              // query of the tile's first row; n_q = 0: there are fewer tiles
};
__device__ __forceinline__ Place place_of(const Prompt &a, int tile)
{
    const int lane = (int)(threadIdx.x & 63u);
    // offsets are device data: whatever they hold, rows stay inside
    auto offset = [](const int32_t *o, int i, int most) { const int v = o[i]; return v < 0 ? 0 : v > most ? most : v; };
    int before = 0;
    for (int at = 0; at < a.B; at += 64) {
        const int b = at + lane;
        int lo = 0, n = 0;
        if (b < a.B) {
            lo = offset(a.q_offsets, b, a.Tq);
            n = offset(a.q_offsets, b + 1, a.Tq) - lo;
            n = n < 0 ? 0 : n;
        }
        const int mine = n / ROWS + (n % ROWS > 0);
        int upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
        }
        const int all = __builtin_amdgcn_readlane(upto, 63);
        if (tile - before < all) {
            const int f = (int)__builtin_ctzll(__ballot(upto > tile - before));
            Place p;
            p.q0 = __builtin_amdgcn_readlane(lo, f);
            p.n_q = __builtin_amdgcn_readlane(n, f);
            const int past = __builtin_amdgcn_readlane(upto, f);
            // of a sequence the last tile first: it sees most keys
            p.first = (past - 1 - (tile - before)) * ROWS;
            p.k0 = offset(a.k_offsets, at + f, a.Tk);
            const int n_k = offset(a.k_offsets, at + f + 1, a.Tk) - p.k0;
            p.n_k = __builtin_amdgcn_readfirstlane(n_k < 0 ? 0 : n_k);
            p.k0 = __builtin_amdgcn_readfirstlane(p.k0);
            return p;
        }
        before += all;
    }
    return {0, 0, 0, 0, 0};
}

template <int T, int DP>
__global__ void __launch_bounds__(64 * WAVES, DP > 128 ? 1 : 2)
hlq_attn_prompt_kernel(const Prompt a)
{
    using F = typename Fragment<T>::type;
    using S = typename Fragment<T>::scalar;
    constexpr int KEYS = DP > 128 ? 32 : 64, BLOCKS = KEYS / 32;
    constexpr int KP = DP * 2 + 16, VP = KEYS * 2 + 16;                 // bytes of a row in LDS: of a key, of a column of values
    constexpr int KEY_LOADS = KEYS * DP / 8 / (64 * WAVES);             // 16 bytes each
    constexpr int UNITS = KEYS / 4 * (DP / 8);                          // of values: four keys, eight columns
    constexpr int VALUE_UNITS = (UNITS + 64 * WAVES - 1) / (64 * WAVES);
    __shared__ __attribute__((aligned(16))) char key_rows[KEYS * KP], value_rows[DP * VP];
    __shared__ int strange[2];                                          // the tile has values that are no numbers

    const int lane = (int)(threadIdx.x & 63u), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int col = lane & 31, half = lane >> 5;
    int id = (int)blockIdx.x;
    const int h = id % a.H;   // kv heads in turn: one each XCD where there are eight
    id /= a.H;
    const int head = h * a.group + id % a.group;
    const Place p = place_of(a, id / a.group);
    if (p.n_q == 0) return;

    const int shift = p.n_k - p.n_q;                                    // place of query 0
    const int rows = p.n_q - p.first < ROWS ? p.n_q - p.first : ROWS;
    // keys that some query of the workgroup sees
    int key_end = p.n_k, key_first = 0;
    if (a.causal) key_end = shift + p.first + rows < key_end ? shift + p.first + rows : key_end;
    if (a.window > 0) {
        const int64_t lowest = (int64_t)shift + p.first - a.window + 1;
        key_first = lowest > 0 ? (int)lowest & ~(KEYS - 1) : 0;
    }

    // queries, the second operand
    const int row = wave * 32 + col, my_place = shift + p.first + row;
    F query[DP / 16];
    {
        const S *q = (const S *)a.q.p + (int64_t)(p.q0 + p.first + (row < rows ? row : 0)) * a.q.ts + head * a.q.hs;
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) {
            S v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (S)0.f;
            if (row < rows && 16 * s + 8 * half < a.D) mx4_read8<false>(q + 16 * s + 8 * half, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) query[s][i] = v[i];
        }
    }

    mx4_u4 key_in[KEY_LOADS], value_in[VALUE_UNITS][4];
    const S *const k = (const S *)a.k.p + (int64_t)p.k0 * a.k.ts + h * a.k.hs, *const v = (const S *)a.v.p + (int64_t)p.k0 * a.v.ts + h * a.v.hs;
    const mx4_u4 zero = {0u, 0u, 0u, 0u};
    auto load = [&](int key0) {
#pragma unroll
        for (int i = 0; i < KEY_LOADS; ++i) {
            const int at = i * 64 * WAVES + (int)threadIdx.x, key = key0 + at / (DP / 8), d = at % (DP / 8) * 8;
            key_in[i] = key < p.n_k && d < a.D ? *(const mx4_u4_any *)(k + key * a.k.ts + d) : zero;
        }
#pragma unroll
        for (int i = 0; i < VALUE_UNITS; ++i) {
            const int at = i * 64 * WAVES + (int)threadIdx.x, key = key0 + at / (DP / 8) * 4, d = at % (DP / 8) * 8;
#pragma unroll
            for (int e = 0; e < 4; ++e) value_in[i][e] = at < UNITS && key + e < p.n_k && d < a.D ? *(const mx4_u4_any *)(v + (key + e) * a.v.ts + d) : zero;
        }
    };
    auto enter = [&](bool look, int turn) {
#pragma unroll
        for (int i = 0; i < KEY_LOADS; ++i) {
            const int at = i * 64 * WAVES + (int)threadIdx.x;
            *(mx4_u4 *)(key_rows + at / (DP / 8) * KP + at % (DP / 8) * 16) = key_in[i];
        }
#pragma unroll
        for (int i = 0; i < VALUE_UNITS; ++i) {
            const int at = i * 64 * WAVES + (int)threadIdx.x, four = at / (DP / 8), d = at % (DP / 8) * 8;
            const int place = (four & ~3) | (four & 1) << 1 | (four >> 1 & 1);   // of the four keys in the order of the weights
            if (UNITS % (64 * WAVES) && at >= UNITS) continue;
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const uint32_t pick = c & 1 ? 0x07060302u : 0x05040100u;
                *(mx4_u2 *)(value_rows + (d + c) * VP + place * 8) = (mx4_u2){__builtin_amdgcn_perm(value_in[i][1][c >> 1], value_in[i][0][c >> 1], pick),
                                                                              __builtin_amdgcn_perm(value_in[i][3][c >> 1], value_in[i][2][c >> 1], pick)};
            }
        }
        if (look) {
            uint32_t found = 0;
#pragma unroll
            for (int i = 0; i < VALUE_UNITS; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int w = 0; w < 4; ++w) found |= (value_in[i][e][w] & Fragment<T>::EXPONENT) + Fragment<T>::ONE;
            if (found & 0x80008000u) strange[turn] = 1;
        }
    };

    float16v acc[DP / 32];
#pragma unroll
    for (int j = 0; j < DP / 32; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[j][i] = 0.f;
    float top = NONE, total = 0.f;
    // places of the wavefront's first and last query
    const int wave_first = shift + p.first + wave * 32, wave_last = shift + p.first + (wave * 32 + 31 < rows ? wave * 32 + 31 : rows - 1);
    // whether some query of the workgroup (or wavefront) does not see all of a tile's keys
    auto edge = [&](int key0, int first, int last) {
        return key0 + KEYS > p.n_k || (a.causal && key0 + KEYS - 1 > first) || (a.window > 0 && key0 <= last - a.window);
    };

    if (threadIdx.x < 2) strange[threadIdx.x] = 0;
    int turn = 0;
    if (key_first < key_end) load(key_first);
    for (int key0 = key_first; key0 < key_end; key0 += KEYS) {
        __syncthreads();
        enter(edge(key0, shift + p.first, shift + p.first + rows - 1), turn);
        __syncthreads();
        if (key0 + KEYS < key_end) load(key0 + KEYS);
        const bool odd = strange[turn];
        if (threadIdx.x == 0) strange[turn ^ 1] = 0;
        turn ^= 1;
        if (wave * 32 >= rows || (a.causal && key0 > wave_last) || (a.window > 0 && key0 + KEYS <= wave_first - a.window + 1)) continue;   // nothing to see
        const bool part = edge(key0, wave_first, wave_last);

        float x[BLOCKS][16];
#pragma unroll
        for (int t = 0; t < BLOCKS; ++t) {
            float16v s;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) s = multiply(*(const F *)(key_rows + (t * 32 + col) * KP + i * 32 + half * 16), query[i], s);
#pragma unroll
            for (int i = 0; i < 16; ++i) x[t][i] = s[i] * a.scale;
        }
        auto seen = [&](int t, int i) {
            const int key = key0 + t * 32 + 8 * (i >> 2) + 4 * half + (i & 3);
            return key < p.n_k && (!a.causal || key <= my_place) && (a.window == 0 || key > my_place - a.window);
        };
        if (part) {
#pragma unroll
            for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (!seen(t, i)) x[t][i] = NONE;
        }
        float m = x[0][0];
#pragma unroll
        for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) m = fmaxf(m, x[t][i]);
        float own;
        const float other = other_half(m, own);
        m = fmaxf(top, fmaxf(own, other));
        const float base = base_of(m);
        if (__any(m > top)) {
            const float keep = __builtin_amdgcn_exp2f(top - base);
            total *= keep;
#pragma unroll
            for (int j = 0; j < DP / 32; ++j)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[j][i] *= keep;
            top = m;
        }
        F weight[BLOCKS][2];
#pragma unroll
        for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float w = __builtin_amdgcn_exp2f(x[t][i] - base);
                total += w;
                weight[t][i >> 3][i & 7] = (S)w;
            }
        auto value = [&](int j, int t, int u) { return *(const F *)(value_rows + (j * 32 + col) * VP + t * 64 + u * 32 + half * 16); };
        if (!(part && odd)) {
#pragma unroll
            for (int j = 0; j < DP / 32; ++j)
#pragma unroll
                for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
                    for (int u = 0; u < 2; ++u) acc[j] = multiply(value(j, t, u), weight[t][u], acc[j]);
        } else {
            // values that are numbers as above; +infinity, and -infinity, and NaN as both, once for each query that sees one
            F sees[BLOCKS][2];
#pragma unroll
            for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    sees[t][i >> 3][i & 7] = (S)(seen(t, i) ? 1.f : 0.f);
                    if (!seen(t, i)) weight[t][i >> 3][i & 7] = (S)0.f;
                }
#pragma unroll
            for (int j = 0; j < DP / 32; ++j) {
                float16v plus, minus;
#pragma unroll
                for (int i = 0; i < 16; ++i) plus[i] = minus[i] = 0.f;
#pragma unroll
                for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        F c = value(j, t, u), up, down;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float f = (float)c[e];
                            up[e] = (S)(f < __builtin_inff() ? 0.f : 1.f);
                            down[e] = (S)(f > NONE ? 0.f : 1.f);
                            if (!(fabsf(f) < __builtin_inff())) c[e] = (S)0.f;
                        }
                        acc[j] = multiply(c, weight[t][u], acc[j]);
                        plus = multiply(up, sees[t][u], plus);
                        minus = multiply(down, sees[t][u], minus);
                    }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    if (plus[i] > 0.f) acc[j][i] += __builtin_inff();
                    if (minus[i] > 0.f) acc[j][i] -= __builtin_inff();
                }
            }
        }
    }
    float own;
    const float other = other_half(total, own);
    total = own + other;
    if (row >= rows) return;
    const float by = total == 0.f ? 0.f : 1.f / total;
    const int64_t at = (int64_t)(p.q0 + p.first + row) * a.out.ts + head * a.out.hs;
#pragma unroll
    for (int j = 0; j < DP / 32; ++j)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int d = 32 * j + 2 * i + 4 * half;
            const float v4[4] = {acc[j][i] * by, acc[j][i + 1] * by, acc[j][i + 2] * by, acc[j][i + 3] * by};
            if (d < a.D) mx4_store4(a.out.p, T, at + d, v4, 4);
        }
}

template <int T>
void launch(const Prompt &a, int64_t grid, hipStream_t st)
{
    const dim3 g((unsigned)grid), block(64 * WAVES);
    if (a.D <= 64) hlq_attn_prompt_kernel<T, 64><<<g, block, 0, st>>>(a);
    else if (a.D <= 128) hlq_attn_prompt_kernel<T, 128><<<g, block, 0, st>>>(a);
    else hlq_attn_prompt_kernel<T, 256><<<g, block, 0, st>>>(a);
}

hlq_status check(int64_t Tq, int64_t Tk, int32_t B, int32_t q_heads, int32_t heads, int32_t dim)
{
    if (Tq < 0 || Tk < 0 || B < 0 || heads < 1 || q_heads < 1 || q_heads % heads || dim < 8 || dim % 8) return HLQ_ERR_BAD_DESC;
    constexpr int64_t MOST = (int64_t)1 << 30;
    return Tq > MOST || Tk > MOST || B > MOST || q_heads > KV_MOST_HEADS || dim > KV_MOST_DIM ? HLQ_ERR_UNSUPPORTED : HLQ_OK;
}

}  // namespace

extern "C" {

hlq_status hlq_attn_prompt_workspace_bytes(int64_t Tq, int64_t Tk, int32_t B, int32_t q_heads, int32_t heads, int32_t dim, size_t *bytes)
{
    const hlq_status s = check(Tq, Tk, B, q_heads, heads, dim);
    if (s != HLQ_OK) return s;
    if (!bytes) return HLQ_ERR_NULL;
    *bytes = HLQ_WS_COUNTER_BYTES;
    return HLQ_OK;
}

hlq_status hlq_attn_prompt(int32_t B, int32_t q_heads, int32_t heads, int32_t dim, hlq_dtype type, int64_t Tq, const void *q, int64_t q_ts, int64_t q_hs,
                           int64_t Tk, const void *k, int64_t k_ts, int64_t k_hs, const void *v, int64_t v_ts, int64_t v_hs, const int32_t *q_offsets,
                           const int32_t *k_offsets, int32_t causal, int32_t window, float scale, void *out, int64_t o_ts, int64_t o_hs, void *ws,
                           size_t ws_bytes, void *stream)
{
    hlq_status s = check(Tq, Tk, B, q_heads, heads, dim);
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
    (void)ws;
    (void)ws_bytes;
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
    a.window = window < 1 << 30 ? window : 0;   // no sequence is longer
    a.scale = scale * 1.44269504f;
    // never more tiles than the queries can make, whatever the offsets hold
    const int64_t tiles = Tq / ROWS + (Tq < B ? Tq : B), grid = tiles * q_heads;
    if (grid > ((int64_t)1 << 24) - 1) return HLQ_ERR_UNSUPPORTED;   // a launch has fewer than 2^32 lanes
    const hipStream_t st = (hipStream_t)stream;
    hlq_clear_stale_error();
    if (type == HLQ_F16) launch<HLQ_F16>(a, grid, st);
    else launch<HLQ_BF16>(a, grid, st);
    return hlq_hip_status(hipGetLastError());
}

}  // extern "C"
