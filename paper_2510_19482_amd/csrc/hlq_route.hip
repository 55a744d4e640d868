// Experts: the router (k largest logits of a token, their softmax weights, tokens grouped by expert) and the weighted sum of the
// experts' outputs.
//
// Router.  A logit becomes a key: its order as a number (0: masked, never chosen), then the expert, the lowest largest, so that keys
// differ and the largest key is the next choice.  26 bits for logits of 16; 42 for f32, as the bits of positive doubles, whose
// maximum is one instruction.  Sixteen lanes hold a token's keys and take the largest k times.  Weights: softmax in fp32, over the
// chosen ones or over all.
// Grouping is a counting sort, stable and without atomics whose order could matter: a token takes an expert at most once, so
// for the 32 tokens of a chunk an expert's rows are a 32-bit mask, its count the bits of it, and a row's place among them the
// bits below its own.  Chunks' counts are added up by each workgroup that places rows (up to 512 chunks) or by a scan in between.
// Exponentials are fp32's own: of an argument rounded once they put a weight 60 half units off; for f32 and all experts' sum 5 % of the time.
// 8192 tokens, 256 experts, k = 8, f32: choices 9.4 us (8 MB; two wavefronts a SIMD in dependent maxima; with 64 lanes a token and
// ballots 19), places 6.7; 32 tokens, 64 experts: 4.3 in one launch; 131072 tokens, 128 experts, bf16: 30.6, the scan 13.2, places 15.9.
#include "hlq_mx4.h"

namespace {

constexpr int CHUNK = 32;           // tokens, bits of a mask; of one workgroup
constexpr int DIRECT_CHUNKS = 512;  // up to here each workgroup of the second kernel adds the counts by itself, in 16 bits
constexpr int PLACE_THREADS = 512;
constexpr int64_t MOST_TOKENS = (int64_t)1 << 27;   // a launch stays below 2^32 threads

struct Route {
    int64_t T;
    int E, k, pitch;                // pitch: bytes of a chunk's counts, E up to 4
    int renorm;
    const void *logits;
    int64_t ld;
    int32_t *ids;
    float *weights;
    int32_t *offsets, *rows, *slots;
    uint8_t *counts;                // [chunks][pitch]
    int32_t *before;                // [chunks + 1][pitch]: rows of an expert in earlier chunks
    int chunks;
};

// what one lane holds of a logit: the key, and what it says
constexpr float LARGEST = 3.402823466e38f;
template <int T>
struct RouteKey {   // f16, bf16
    using type = uint32_t;
    using V = typename Mx4Type<T>::type;
    static constexpr uint32_t INF = T == HLQ_F16 ? 0x7c00u : 0x7f80u;
    static __device__ __forceinline__ type make(V v, int e)
    {
        uint32_t b = __builtin_bit_cast(uint16_t, v);
        if ((b & 0x7fffu) > INF || b == (0x8000u | INF)) return 0u;   // NaN, -inf
        if (b == 0x8000u) b = 0u;                                       // -0
        return ((b ^ (b & 0x8000u ? 0xffffu : 0x8000u)) << 16) | (uint32_t)(HLQ_MAX_EXPERTS - 1 - e);
    }
    static __device__ __forceinline__ bool present(type k) { return k >= 0x10000u; }
    static __device__ __forceinline__ type without(type k, type taken) { return k == taken ? 0u : k; }
    static __device__ __forceinline__ float value(type k)
    {
        const uint32_t o = k >> 16;
        const float v = (float)__builtin_bit_cast(V, (uint16_t)(o ^ (o & 0x8000u ? 0x8000u : 0xffffu)));
        return v < LARGEST ? v : LARGEST;
    }
    static __device__ __forceinline__ type max(type a, type b) { return a > b ? a : b; }
    template <int CTRL>
    static __device__ __forceinline__ type rotated(type k) { return (type)__builtin_amdgcn_mov_dpp((int)k, CTRL, 0xf, 0xf, true); }
};
template <>
struct RouteKey<HLQ_F32> {
    using type = uint64_t;
    static constexpr uint64_t NORMAL = 1ull << 62;   // a key that is not masked is a normal double
    static __device__ __forceinline__ type make(float v, int e)
    {
        if (!(v > -INFINITY)) return 0ull;
        v = (v < LARGEST ? v : LARGEST) + 0.0f;   // -0 is 0
        const uint32_t b = __builtin_bit_cast(uint32_t, v);
        return NORMAL | (uint64_t)(b & 0x80000000u ? ~b : b | 0x80000000u) << 10 | (uint32_t)(HLQ_MAX_EXPERTS - 1 - e);
    }
    static __device__ __forceinline__ bool present(type k) { return k >= NORMAL; }
    static __device__ __forceinline__ type without(type k, type taken)
    {
        // the lower words differ, by the expert's number; without its upper word a key is below all that are left
        const uint32_t low = (uint32_t)k;
        return low | (uint64_t)(low == (uint32_t)taken ? 0u : (uint32_t)(k >> 32)) << 32;
    }
    static __device__ __forceinline__ float value(type k)
    {
        const uint32_t o = (uint32_t)(k >> 10);
        return __builtin_bit_cast(float, o & 0x80000000u ? o & 0x7fffffffu : ~o);
    }
    static __device__ __forceinline__ type max(type a, type b)
    {
        uint64_t m;
        asm("v_max_f64 %0, %1, %2" : "=v"(m) : "v"(a), "v"(b));
        return m;
    }
    template <int CTRL>
    static __device__ __forceinline__ type rotated(type k)
    {
        return (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)k, CTRL, 0xf, 0xf, true) |
               (uint64_t)(uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)(k >> 32), CTRL, 0xf, 0xf, true) << 32;
    }
};
// of N keys, as a tree
template <class K, int N>
__device__ __forceinline__ typename K::type max_of(const typename K::type *key)
{
    if constexpr (N == 1) return key[0];
    else return K::max(max_of<K, N / 2>(key), max_of<K, N - N / 2>(key + N / 2));
}
// of the sixteen lanes of a row, in each of them: from 8, 4, 2, 1 lanes on
template <class K>
__device__ __forceinline__ typename K::type row_max(typename K::type v)
{
    v = K::max(v, K::template rotated<0x128>(v));
    v = K::max(v, K::template rotated<0x124>(v));
    v = K::max(v, K::template rotated<0x122>(v));
    return K::max(v, K::template rotated<0x121>(v));
}
template <int CTRL>
__device__ __forceinline__ float rotated(float v) { return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true)); }
__device__ __forceinline__ float row_sum(float v)
{
    v += rotated<0x128>(v);
    v += rotated<0x124>(v);
    v += rotated<0x122>(v);
    return v + rotated<0x121>(v);
}

// masks of a chunk's rows by expert from its choices, staged in LDS as [token][k]
__device__ __forceinline__ void set_masks(const Route &a, const int *picks, uint32_t *masks, int tokens)
{
    for (int i = (int)threadIdx.x; i < tokens * a.k; i += (int)blockDim.x)
        if (picks[i] >= 0) atomicOr(&masks[picks[i]], 1u << (i / a.k));
}
// slots and rows of a chunk; base: first row of each expert's share of it
__device__ __forceinline__ void place(const Route &a, const int *picks, const uint32_t *masks, const int *base, int64_t t0, int tokens)
{
    for (int i = (int)threadIdx.x; i < tokens * a.k; i += (int)blockDim.x) {
        const int e = picks[i], t = i / a.k;
        int slot = -1;
        if (e >= 0) {
            slot = base[e] + __popc(masks[e] & ((1u << t) - 1u));
            a.rows[slot] = (int32_t)(t0 + t);
        }
        a.slots[t0 * a.k + i] = slot;
    }
}
// exclusive prefix of n <= 1024 counts in LDS, by one wavefront; returns their sum
__device__ __forceinline__ int prefix(const int *count, int *first, int n)
{
    const int lane = (int)(threadIdx.x & 63u);
    int before = 0;
    for (int b = 0; b < n; b += 64) {
        const int mine = b + lane < n ? count[b + lane] : 0;
        int upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
        }
        if (b + lane < n) first[b + lane] = before + upto - mine;
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return before;
}

// V: logits a lane holds
template <int T, int V>
__global__ void __launch_bounds__(16 * CHUNK)
hlq_route_top_kernel(const Route a)
{
    extern __shared__ int lds[];
    uint32_t *masks = (uint32_t *)lds;               // [E]
    int *count = lds + a.E, *first = count + a.E;    // [E] each
    int *picks = first + a.E;                        // [CHUNK][k]
    float *values = (float *)(picks + CHUNK * a.k);  // [CHUNK][k]
    const int lane = (int)(threadIdx.x & 63u), wave = (int)(threadIdx.x >> 6), l = lane & 15, t = (int)(threadIdx.x >> 4);
    const int64_t t0 = (int64_t)blockIdx.x * CHUNK;
    const int tokens = (int)(a.T - t0 < CHUNK ? a.T - t0 : CHUNK);
    for (int e = (int)threadIdx.x; e < a.E; e += (int)blockDim.x) masks[e] = 0u;
    if (t < tokens) {
        using K = RouteKey<T>;
        const typename Mx4Type<T>::type *row = (const typename Mx4Type<T>::type *)a.logits + (t0 + t) * a.ld;
        typename K::type key[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int e = 16 * j + l;
            key[j] = e < a.E ? K::make(row[e], e) : (typename K::type)0;
        }
        float top = 0.f, sum = 0.f;
        int found = 0;
        for (; found < a.k; ++found) {
            const typename K::type best = row_max<K>(max_of<K, V>(key));
            if (!K::present(best)) break;
            const float v = K::value(best);
            if (found == 0) {
                top = v;
                if (!a.renorm) {
#pragma unroll
                    for (int j = 0; j < V; ++j) sum += K::present(key[j]) ? expf(K::value(key[j]) - top) : 0.f;
                }
            }
            if (l == 0) {
                picks[t * a.k + found] = HLQ_MAX_EXPERTS - 1 - (int)(best & (HLQ_MAX_EXPERTS - 1));
                values[t * a.k + found] = v;
            }
#pragma unroll
            for (int j = 0; j < V; ++j) key[j] = K::without(key[j], best);
        }
        // what lane 0 of the row wrote is there for the others: they are of one wavefront, whose LDS accesses keep their order
        __builtin_amdgcn_wave_barrier();
        if (a.renorm) {
            for (int i = l; i < found; i += 16) sum += expf(values[t * a.k + i] - top);
        }
        sum = row_sum(sum);
        for (int i = l; i < a.k; i += 16) {
            const int id = i < found ? picks[t * a.k + i] : -1;
            if (i >= found) picks[t * a.k + i] = -1;
            a.ids[(t0 + t) * a.k + i] = id;
            a.weights[(t0 + t) * a.k + i] = i < found ? expf(values[t * a.k + i] - top) / sum : 0.f;
        }
    }
    __syncthreads();
    set_masks(a, picks, masks, tokens);
    __syncthreads();
    if (a.chunks > 1) {
        for (int e = (int)threadIdx.x; e < a.pitch; e += (int)blockDim.x)
            a.counts[(int64_t)blockIdx.x * a.pitch + e] = e < a.E ? (uint8_t)__popc(masks[e]) : (uint8_t)0;
        return;
    }
    for (int e = (int)threadIdx.x; e < a.E; e += (int)blockDim.x) count[e] = __popc(masks[e]);
    __syncthreads();
    if (wave == 0) {
        const int all = prefix(count, first, a.E);
        for (int e = lane; e < a.E; e += 64) a.offsets[e] = first[e];
        if (lane == 0) a.offsets[a.E] = all;
        for (int i = all + lane; i < tokens * a.k; i += 64) a.rows[i] = -1;
    }
    __syncthreads();
    place(a, picks, masks, first, t0, tokens);
}

// Rows of an expert in earlier chunks, and in all.  A workgroup has four experts, a thread a share of the chunks.  131072 tokens, 128 experts:
// 13 us (with 16 experts a workgroup and 4-byte stores 39: one compute unit put out 64 addresses for each of 1024 stores); 16500, 256: 4.1.
__global__ void __launch_bounds__(1024)
hlq_route_scan_kernel(const Route a)
{
    __shared__ mx4_int4 waves[16];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, e0 = (int)blockIdx.x * 4;
    const int share = (a.chunks + 1023) / 1024, c0 = tid * share, c1 = c0 + share < a.chunks ? c0 + share : a.chunks;
    auto each = [&](auto f) {   // words are loaded together: a load waits for no store
        for (int c = c0; c < c1; c += 8) {
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = c + j < c1 ? *(const uint32_t *)(a.counts + (int64_t)(c + j) * a.pitch + e0) : 0u;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c + j < c1) f(c + j, w[j]);
        }
    };
    mx4_int4 mine = {0, 0, 0, 0};
    each([&](int, uint32_t w) {
#pragma unroll
        for (int i = 0; i < 4; ++i) mine[i] += (int)(w >> (8 * i) & 255u);
    });
    mx4_int4 upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int o = __shfl_up(upto[i], d);
            upto[i] += lane >= d ? o : 0;
        }
    if (lane == 63) waves[wave] = upto;
    __syncthreads();
    for (int v = 0; v < wave; ++v) upto += waves[v];
    if (tid == 1023) *(mx4_int4 *)(a.before + (int64_t)a.chunks * a.pitch + e0) = upto;
    mx4_int4 before = upto - mine;
    each([&](int c, uint32_t w) {
        *(mx4_int4 *)(a.before + (int64_t)c * a.pitch + e0) = before;
#pragma unroll
        for (int i = 0; i < 4; ++i) before[i] += (int)(w >> (8 * i) & 255u);
    });
}

__global__ void __launch_bounds__(PLACE_THREADS)
hlq_route_place_kernel(const Route a)
{
    extern __shared__ int lds[];
    uint32_t *masks = (uint32_t *)lds;                                         // [pitch] each
    int *count = lds + a.pitch, *first = count + a.pitch, *before = first + a.pitch;
    int *picks = before + a.pitch;                                             // [CHUNK][k]
    __shared__ int total;
    const int64_t t0 = (int64_t)blockIdx.x * CHUNK;
    const int tokens = (int)(a.T - t0 < CHUNK ? a.T - t0 : CHUNK), me = (int)blockIdx.x, tid = (int)threadIdx.x;
    for (int i = tid; i < tokens * a.k; i += PLACE_THREADS) picks[i] = a.ids[t0 * a.k + i];
    const bool scanned = a.chunks > DIRECT_CHUNKS;
    for (int e = tid; e < a.pitch; e += PLACE_THREADS) {
        masks[e] = 0u;
        count[e] = scanned && e < a.E ? a.before[(int64_t)a.chunks * a.pitch + e] : 0;
        before[e] = scanned && e < a.E ? a.before[(int64_t)me * a.pitch + e] : 0;
    }
    __syncthreads();
    set_masks(a, picks, masks, tokens);
    if (!scanned) {
        // a thread has four experts over a share of the chunks, their counts in the bytes of a word
        const int quads = a.pitch / 4, shares = quads < PLACE_THREADS ? PLACE_THREADS / quads : 1;
        for (int i = tid; i < quads * shares; i += PLACE_THREADS) {
            const int quad = i % quads, share = i / quads;
            uint32_t all[2] = {0u, 0u}, less[2] = {0u, 0u};   // experts 0 and 2, 1 and 3, in 16 bits
#pragma unroll 8
            for (int c = share; c < a.chunks; c += shares) {
                const uint32_t w = *(const uint32_t *)(a.counts + (int64_t)c * a.pitch + quad * 4);
                const uint32_t even = w & 0x00ff00ffu, odd = (w >> 8) & 0x00ff00ffu;
                all[0] += even;
                all[1] += odd;
                less[0] += c < me ? even : 0u;
                less[1] += c < me ? odd : 0u;
            }
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                atomicAdd(&count[quad * 4 + n], (int)(all[n & 1] >> (16 * (n >> 1)) & 0xffffu));
                atomicAdd(&before[quad * 4 + n], (int)(less[n & 1] >> (16 * (n >> 1)) & 0xffffu));
            }
        }
    }
    __syncthreads();
    if (tid < 64) {
        const int all = prefix(count, first, a.E);
        if (tid == 0) total = all;
    }
    __syncthreads();
    if (me == 0) {
        for (int e = tid; e < a.E; e += PLACE_THREADS) a.offsets[e] = first[e];
        if (tid == 0) a.offsets[a.E] = total;
    }
    for (int e = tid; e < a.E; e += PLACE_THREADS) before[e] += first[e];
    // rows that no token took
    for (int64_t i = total + (int64_t)me * PLACE_THREADS + tid; i < a.T * a.k; i += (int64_t)gridDim.x * PLACE_THREADS) a.rows[i] = -1;
    __syncthreads();
    place(a, picks, masks, before, t0, tokens);
}

template <int T>
void launch_top(const Route &a, hipStream_t st)
{
    const dim3 grid((unsigned)a.chunks), block(16 * CHUNK);
    const size_t lds = (size_t)a.E * 12u + (size_t)CHUNK * a.k * 8u;
    if (a.E <= 64) hlq_route_top_kernel<T, 4><<<grid, block, lds, st>>>(a);
    else if (a.E <= 128) hlq_route_top_kernel<T, 8><<<grid, block, lds, st>>>(a);
    else if (a.E <= 256) hlq_route_top_kernel<T, 16><<<grid, block, lds, st>>>(a);
    else if (a.E <= 384) hlq_route_top_kernel<T, 24><<<grid, block, lds, st>>>(a);
    else if (a.E <= 512) hlq_route_top_kernel<T, 32><<<grid, block, lds, st>>>(a);
    else hlq_route_top_kernel<T, 64><<<grid, block, lds, st>>>(a);
}

struct Combine {
    int64_t T;
    int k, D, eights;
    int64_t R;
    const void *y;
    int64_t ld;
    const int32_t *slots;
    const float *weights;
    void *out;
    int otype;
    int64_t ldo;
};

// y[t, d] = sum_i weights[t, i] Y[slots[t, i], d], i ascending, fp32: a thread has eight successive d of a token.  Bound by the
// bytes of Y; the loads of four experts are in flight together, and pass the caches by.  8192 tokens, 8 of 4096, bf16: 119 us
// (605 MB, 5.1 TB/s; through the caches 131).
template <int T>
__global__ void __launch_bounds__(256)
hlq_expert_combine_kernel(const Combine a, int64_t items)
{
    using V = typename Mx4Type<T>::type;
    for (int64_t it = (int64_t)blockIdx.x * 256 + threadIdx.x; it < items; it += (int64_t)gridDim.x * 256) {
        const int64_t t = it / a.eights;
        const int d = (int)(it - t * a.eights) * 8;
        float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int i = 0; i < a.k; i += 4) {
            V v[4][8];
            float w[4];
            bool has[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                has[j] = false;
                if (i + j < a.k) {
                    const int s = a.slots[t * a.k + i + j];
                    has[j] = s >= 0 && s < a.R;
                    w[j] = a.weights[t * a.k + i + j];
                    if (has[j]) mx4_load8<true>((const V *)a.y + s * a.ld + d, a.D - d, v[j]);
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (has[j])
#pragma unroll
                    for (int c = 0; c < 8; ++c) sum[c] = fmaf(w[j], (float)v[j][c], sum[c]);
        }
        mx4_store8(a.out, a.otype, t * a.ldo + d, sum, a.D - d);
    }
}

template <int T>
void launch_combine(const Combine &a, hipStream_t st)
{
    const int64_t items = a.T * a.eights, blocks = (items + 255) / 256;
    const unsigned grid = (unsigned)(blocks < (1 << 20) ? blocks : 1 << 20);
    hlq_expert_combine_kernel<T><<<grid, 256, 0, st>>>(a, items);
}

hlq_status check_route(int64_t T, int32_t E, int32_t k)
{
    if (T < 0 || E < 1 || k < 1 || k > E) return HLQ_ERR_BAD_DESC;
    if (E > HLQ_MAX_EXPERTS || k > HLQ_MAX_CHOICES || T > MOST_TOKENS || T > (((int64_t)1 << 31) - 256) / k) return HLQ_ERR_UNSUPPORTED;
    return HLQ_OK;
}
size_t counts_bytes(int64_t T, int32_t E) { return ((size_t)((T + CHUNK - 1) / CHUNK) * (size_t)((E + 3) & ~3) + 15u) & ~(size_t)15u; }
size_t route_need(int64_t T, int32_t E)
{
    const int64_t chunks = (T + CHUNK - 1) / CHUNK;
    if (chunks <= 1) return 0;
    return counts_bytes(T, E) + (chunks > DIRECT_CHUNKS ? (size_t)(chunks + 1) * (size_t)((E + 3) & ~3) * 4u : 0u);
}

}  // namespace

extern "C" {

hlq_status hlq_route_workspace_bytes(int64_t T, int32_t E, int32_t k, size_t *bytes)
{
    const hlq_status s = check_route(T, E, k);
    if (s != HLQ_OK) return s;
    if (!bytes) return HLQ_ERR_NULL;
    *bytes = route_need(T, E);
    return HLQ_OK;
}

hlq_status hlq_route(int64_t T, int32_t E, int32_t k, const void *logits, hlq_dtype type, int64_t ld, int renorm, int32_t *ids,
                     float *weights, int32_t *offsets, int32_t *rows, int32_t *slots, void *ws, size_t ws_bytes, void *stream)
{
    const hlq_status s = check_route(T, E, k);
    if (s != HLQ_OK) return s;
    if (!hlq_is_float(type)) return HLQ_ERR_UNSUPPORTED;
    if (T > 1 && ld < E) return HLQ_ERR_BAD_STRIDE;
    if (!offsets || (T > 0 && (!logits || !ids || !weights || !rows || !slots))) return HLQ_ERR_NULL;
    if ((uintptr_t)logits % (unsigned)hlq_dtype_bytes(type) || (((uintptr_t)ids | (uintptr_t)weights | (uintptr_t)offsets | (uintptr_t)rows | (uintptr_t)slots) & 3u))
        return HLQ_ERR_BAD_STRIDE;
    const size_t need = route_need(T, E);
    if (need) {
        if (!ws) return HLQ_ERR_NULL;
        if (ws_bytes < need) return HLQ_ERR_BUFFER_TOO_SMALL;
        if ((uintptr_t)ws & 15u) return HLQ_ERR_BAD_STRIDE;
    }
    Route a{};
    a.T = T;
    a.E = E;
    a.k = k;
    a.pitch = (E + 3) & ~3;
    a.renorm = renorm;
    a.logits = logits;
    a.ld = ld;
    a.ids = ids;
    a.weights = weights;
    a.offsets = offsets;
    a.rows = rows;
    a.slots = slots;
    a.chunks = T == 0 ? 1 : (int)((T + CHUNK - 1) / CHUNK);   // without tokens one workgroup writes the offsets
    a.counts = (uint8_t *)ws;
    a.before = ws ? (int32_t *)((char *)ws + counts_bytes(T, E)) : nullptr;
    const hipStream_t st = (hipStream_t)stream;
    hlq_clear_stale_error();
    if (type == HLQ_F16) launch_top<HLQ_F16>(a, st);
    else if (type == HLQ_BF16) launch_top<HLQ_BF16>(a, st);
    else launch_top<HLQ_F32>(a, st);
    if (a.chunks > DIRECT_CHUNKS) hlq_route_scan_kernel<<<(E + 3) / 4, 1024, 0, st>>>(a);
    if (a.chunks > 1) hlq_route_place_kernel<<<(unsigned)a.chunks, PLACE_THREADS, (size_t)a.pitch * 16u + (size_t)CHUNK * k * 4u, st>>>(a);
    return hlq_hip_status(hipGetLastError());
}

hlq_status hlq_expert_combine(int64_t T, int32_t k, int32_t D, int64_t R, const void *Y, hlq_dtype ytype, int64_t ldy, const int32_t *slots,
                              const float *weights, void *out, hlq_dtype otype, int64_t ldo, void *stream)
{
    if (T < 0 || k < 1 || D < 1 || R < 0) return HLQ_ERR_BAD_DESC;
    if (!hlq_is_float(ytype) || !hlq_is_float(otype) || k > HLQ_MAX_CHOICES || D > HLQ_MAX_N || T >= ((int64_t)1 << 31)) return HLQ_ERR_UNSUPPORTED;
    if ((R > 1 && ldy < D) || (T > 1 && ldo < D)) return HLQ_ERR_BAD_STRIDE;
    if (T == 0) return HLQ_OK;
    if ((R > 0 && !Y) || !slots || !weights || !out) return HLQ_ERR_NULL;
    if ((uintptr_t)Y % (unsigned)hlq_dtype_bytes(ytype) || (uintptr_t)out % (unsigned)hlq_dtype_bytes(otype) || (((uintptr_t)slots | (uintptr_t)weights) & 3u))
        return HLQ_ERR_BAD_STRIDE;
    Combine a{T, k, D, (D + 7) / 8, R, Y, ldy, slots, weights, out, otype, ldo};
    const hipStream_t st = (hipStream_t)stream;
    hlq_clear_stale_error();
    if (ytype == HLQ_F16) launch_combine<HLQ_F16>(a, st);
    else if (ytype == HLQ_BF16) launch_combine<HLQ_BF16>(a, st);
    else launch_combine<HLQ_F32>(a, st);
    return hlq_hip_status(hipGetLastError());
}

}  // extern "C"
