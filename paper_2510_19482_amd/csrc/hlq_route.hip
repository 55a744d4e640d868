// Experts: the router (k largest logits of a token, their softmax weights, tokens grouped by expert) and the weighted sum of the
// experts' outputs.
//
// Router.  Logits become unsigned keys whose order is the numbers' (0: masked, never chosen); a wavefront holds a token's logits,
// lane l those of experts l, l + 64, ..., and takes the largest k times: a maximum over the lanes, then the lowest expert that
// has it.  Weights: softmax in fp32, over the chosen ones or over all.
// Grouping is a counting sort, stable and without atomics whose order could matter: a token takes an expert at most once, so
// for the 64 tokens of a chunk an expert's rows are a 64-bit mask, its count the bits of it, and a row's place among them the
// bits below its own.  Chunks' counts are summed by whoever needs them (up to 256 chunks) or by a scan in between.
#include "hlq_mx4.h"

namespace {

constexpr int CHUNK = 64;           // tokens, bits of a mask
constexpr int DIRECT_CHUNKS = 256;  // up to here each workgroup of the second kernel adds the counts by itself
constexpr int TOP_WAVES = 16;

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
    int32_t *before;                // [chunks + 1][E]: rows of an expert in earlier chunks
    int chunks;
};

// largest of 64 unsigned values, in every lane's hands as a scalar
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
    auto step = [&](uint32_t o) { v = o > v ? o : v; };
    step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, true));   // from 1, 2, 4, 8 lanes below in a row of 16
    step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, true));
    step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, true));
    step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, true));
    step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false));  // a row's last lane to the next row
    step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false));  // the lower half's last lane to the upper half
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
    return v;
}

__device__ __forceinline__ uint32_t key_of(float v)
{
    if (!(v > -INFINITY)) return 0u;                 // masked: -inf and NaN
    v = (v < 3.402823466e38f ? v : 3.402823466e38f) + 0.0f;   // +inf is the largest float; -0 is 0
    const uint32_t b = __builtin_bit_cast(uint32_t, v);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key)
{
    return __builtin_bit_cast(float, key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

// masks of a chunk's rows by expert from its choices, staged in LDS as [token][k]
__device__ __forceinline__ void set_masks(const Route &a, const int *picks, unsigned long long *masks, int tokens)
{
    for (int i = (int)threadIdx.x; i < tokens * a.k; i += (int)blockDim.x)
        if (picks[i] >= 0) atomicOr(&masks[picks[i]], 1ull << (i / a.k));
}
// slots and rows of a chunk; base: first row of each expert's share of it
__device__ __forceinline__ void place(const Route &a, const int *picks, const unsigned long long *masks, const int *base, int64_t t0, int tokens)
{
    for (int i = (int)threadIdx.x; i < tokens * a.k; i += (int)blockDim.x) {
        const int e = picks[i], t = i / a.k;
        int slot = -1;
        if (e >= 0) {
            slot = base[e] + __popcll(masks[e] & ((1ull << t) - 1ull));
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
__global__ void __launch_bounds__(64 * TOP_WAVES)
hlq_route_top_kernel(const Route a)
{
    extern __shared__ unsigned long long lds[];
    unsigned long long *masks = lds;                 // [E]
    int *picks = (int *)(masks + a.E);               // [CHUNK][k]
    int *count = picks + CHUNK * a.k, *first = count + a.E;   // [E] each
    const int lane = (int)(threadIdx.x & 63u), wave = (int)(threadIdx.x >> 6);
    const int64_t t0 = (int64_t)blockIdx.x * CHUNK;
    const int tokens = (int)(a.T - t0 < CHUNK ? a.T - t0 : CHUNK);
    for (int e = (int)threadIdx.x; e < a.E; e += (int)blockDim.x) masks[e] = 0ull;
    for (int t = wave; t < tokens; t += TOP_WAVES) {
        const typename Mx4Type<T>::type *row = (const typename Mx4Type<T>::type *)a.logits + (t0 + t) * a.ld;
        uint32_t key[V], all[V];
#pragma unroll
        for (int j = 0; j < V; ++j) key[j] = all[j] = 64 * j + lane < a.E ? key_of((float)row[64 * j + lane]) : 0u;
        uint32_t mine = 0u;      // lane i: the i-th choice
        int id = -1;
        for (int i = 0; i < a.k; ++i) {
            uint32_t best = key[0];
#pragma unroll
            for (int j = 1; j < V; ++j) best = key[j] > best ? key[j] : best;
            best = wave_max(best);
            if (best == 0u) break;
            int e = -1;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const uint64_t has = __ballot(key[j] == best);
                if (e < 0 && has) {
                    e = 64 * j + (int)__builtin_ctzll(has);
                    if (lane == (e & 63)) key[j] = 0u;
                }
            }
            if (lane == i) {
                mine = best;
                id = e;
            }
        }
        const float top = value_of((uint32_t)__builtin_amdgcn_readfirstlane((int)mine));
        const float p = mine ? expf(value_of(mine) - top) : 0.f;
        float sum = p;
        if (!a.renorm) {
            sum = 0.f;
#pragma unroll
            for (int j = 0; j < V; ++j) sum += all[j] ? expf(value_of(all[j]) - top) : 0.f;
        }
        sum = wave_sum(sum);
        if (lane < a.k) {
            a.ids[(t0 + t) * a.k + lane] = id;
            a.weights[(t0 + t) * a.k + lane] = mine ? p / sum : 0.f;
            picks[t * a.k + lane] = id;
        }
    }
    __syncthreads();
    set_masks(a, picks, masks, tokens);
    __syncthreads();
    if (a.chunks > 1) {
        for (int e = (int)threadIdx.x; e < a.pitch; e += (int)blockDim.x)
            a.counts[(int64_t)blockIdx.x * a.pitch + e] = e < a.E ? (uint8_t)__popcll(masks[e]) : (uint8_t)0;
        return;
    }
    for (int e = (int)threadIdx.x; e < a.E; e += (int)blockDim.x) count[e] = __popcll(masks[e]);
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

// rows of an expert in earlier chunks; a workgroup has 16 experts, a thread four of them over a share of the chunks
__global__ void __launch_bounds__(1024)
hlq_route_scan_kernel(const Route a)
{
    __shared__ int sums[256][16];
    const int quad = (int)(threadIdx.x & 3u), part = (int)(threadIdx.x >> 2);
    const int e0 = (int)blockIdx.x * 16 + quad * 4;
    const int share = (a.chunks + 255) / 256, c0 = part * share, c1 = c0 + share < a.chunks ? c0 + share : a.chunks;
    int s[4] = {0, 0, 0, 0};
    if (e0 < a.pitch)
        for (int c = c0; c < c1; ++c) {
            const uint32_t w = *(const uint32_t *)(a.counts + (int64_t)c * a.pitch + e0);
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] += (int)(w >> (8 * i) & 255u);
        }
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[part][quad * 4 + i] = s[i];
    __syncthreads();
    if (threadIdx.x < 16) {
        int before = 0;
        for (int p = 0; p < 256; ++p) {
            const int v = sums[p][threadIdx.x];
            sums[p][threadIdx.x] = before;
            before += v;
        }
        const int e = (int)blockIdx.x * 16 + (int)threadIdx.x;
        if (e < a.E) a.before[(int64_t)a.chunks * a.E + e] = before;
    }
    __syncthreads();
    if (e0 < a.pitch) {
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = sums[part][quad * 4 + i];
        for (int c = c0; c < c1; ++c) {
            const uint32_t w = *(const uint32_t *)(a.counts + (int64_t)c * a.pitch + e0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (e0 + i < a.E) a.before[(int64_t)c * a.E + e0 + i] = s[i];
                s[i] += (int)(w >> (8 * i) & 255u);
            }
        }
    }
}

__global__ void __launch_bounds__(256)
hlq_route_place_kernel(const Route a)
{
    extern __shared__ unsigned long long lds[];
    unsigned long long *masks = lds;
    int *picks = (int *)(masks + a.E);
    int *count = picks + CHUNK * a.k, *first = count + a.E, *before = first + a.E;
    __shared__ int total;
    const int64_t t0 = (int64_t)blockIdx.x * CHUNK;
    const int tokens = (int)(a.T - t0 < CHUNK ? a.T - t0 : CHUNK), me = (int)blockIdx.x;
    for (int i = (int)threadIdx.x; i < tokens * a.k; i += 256) picks[i] = a.ids[t0 * a.k + i];
    for (int e = (int)threadIdx.x; e < a.E; e += 256) {
        masks[e] = 0ull;
        if (a.chunks > DIRECT_CHUNKS) {
            count[e] = a.before[(int64_t)a.chunks * a.E + e];
            before[e] = a.before[(int64_t)me * a.E + e];
        }
    }
    if (a.chunks <= DIRECT_CHUNKS)
        for (int e = 4 * (int)threadIdx.x; e < a.pitch; e += 4 * 256) {
            int all[4] = {0, 0, 0, 0}, less[4] = {0, 0, 0, 0};
#pragma unroll 8
            for (int c = 0; c < a.chunks; ++c) {
                const uint32_t w = *(const uint32_t *)(a.counts + (int64_t)c * a.pitch + e);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int n = (int)(w >> (8 * i) & 255u);
                    all[i] += n;
                    less[i] += c < me ? n : 0;
                }
            }
            for (int i = 0; i < 4 && e + i < a.E; ++i) {
                count[e + i] = all[i];
                before[e + i] = less[i];
            }
        }
    __syncthreads();
    set_masks(a, picks, masks, tokens);
    if (threadIdx.x < 64) {
        const int all = prefix(count, first, a.E);
        if (threadIdx.x == 0) total = all;
    }
    __syncthreads();
    if (me == 0) {
        for (int e = (int)threadIdx.x; e < a.E; e += 256) a.offsets[e] = first[e];
        if (threadIdx.x == 0) a.offsets[a.E] = total;
    }
    for (int e = (int)threadIdx.x; e < a.E; e += 256) before[e] += first[e];
    // rows that no token took
    for (int64_t i = total + (int64_t)me * 256 + threadIdx.x; i < a.T * a.k; i += (int64_t)gridDim.x * 256) a.rows[i] = -1;
    __syncthreads();
    place(a, picks, masks, before, t0, tokens);
}

template <int T>
void launch_top(const Route &a, size_t lds, hipStream_t st)
{
    const dim3 grid((unsigned)a.chunks), block(64 * TOP_WAVES);
    if (a.E <= 64) hlq_route_top_kernel<T, 1><<<grid, block, lds, st>>>(a);
    else if (a.E <= 128) hlq_route_top_kernel<T, 2><<<grid, block, lds, st>>>(a);
    else if (a.E <= 256) hlq_route_top_kernel<T, 4><<<grid, block, lds, st>>>(a);
    else if (a.E <= 512) hlq_route_top_kernel<T, 8><<<grid, block, lds, st>>>(a);
    else hlq_route_top_kernel<T, 16><<<grid, block, lds, st>>>(a);
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
    bool out_aligned;
};

// y[t, d] = sum_i weights[t, i] Y[slots[t, i], d], i ascending, fp32: a thread has eight successive d of a token.  Bound by the
// bytes of Y; the loads of four experts are in flight together.
template <int T, bool ALIGNED>
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
                    if (has[j]) mx4_load8<ALIGNED>((const V *)a.y + s * a.ld + d, a.D - d, v[j]);
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (has[j])
#pragma unroll
                    for (int c = 0; c < 8; ++c) sum[c] = fmaf(w[j], (float)v[j][c], sum[c]);
        }
        const int left = a.D - d;
        mx4_store(a.out, a.otype, t * a.ldo + d, sum, left < 4 ? left : 4, left >= 4 && a.out_aligned);
        if (left > 4) mx4_store(a.out, a.otype, t * a.ldo + d + 4, sum + 4, left < 8 ? left - 4 : 4, left >= 8 && a.out_aligned);
    }
}

template <int T>
void launch_combine(const Combine &a, bool aligned, hipStream_t st)
{
    const int64_t items = a.T * a.eights, blocks = (items + 255) / 256;
    const unsigned grid = (unsigned)(blocks < (1 << 20) ? blocks : 1 << 20);
    if (aligned) hlq_expert_combine_kernel<T, true><<<grid, 256, 0, st>>>(a, items);
    else hlq_expert_combine_kernel<T, false><<<grid, 256, 0, st>>>(a, items);
}

hlq_status check_route(int64_t T, int32_t E, int32_t k)
{
    if (T < 0 || E < 1 || k < 1 || k > E) return HLQ_ERR_BAD_DESC;
    if (E > HLQ_MAX_EXPERTS || k > HLQ_MAX_CHOICES || T > (((int64_t)1 << 31) - 256) / k) return HLQ_ERR_UNSUPPORTED;
    return HLQ_OK;
}
size_t counts_bytes(int64_t T, int32_t E) { return ((size_t)((T + CHUNK - 1) / CHUNK) * (size_t)((E + 3) & ~3) + 15u) & ~(size_t)15u; }
size_t route_need(int64_t T, int32_t E)
{
    const int64_t chunks = (T + CHUNK - 1) / CHUNK;
    if (chunks <= 1) return 0;
    return counts_bytes(T, E) + (chunks > DIRECT_CHUNKS ? (size_t)(chunks + 1) * (size_t)E * 4u : 0u);
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
    const size_t lds = (size_t)E * 16u + (size_t)CHUNK * k * 4u;
    hlq_clear_stale_error();
    if (type == HLQ_F16) launch_top<HLQ_F16>(a, lds, st);
    else if (type == HLQ_BF16) launch_top<HLQ_BF16>(a, lds, st);
    else launch_top<HLQ_F32>(a, lds, st);
    if (a.chunks > DIRECT_CHUNKS) hlq_route_scan_kernel<<<(E + 15) / 16, 1024, 0, st>>>(a);
    if (a.chunks > 1) hlq_route_place_kernel<<<(unsigned)a.chunks, 256, lds + (size_t)E * 4u, st>>>(a);
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
    Combine a{T, k, D, (D + 7) / 8, R, Y, ldy, slots, weights, out, otype, ldo, false};
    a.out_aligned = (uintptr_t)out % (4u * (unsigned)hlq_dtype_bytes(otype)) == 0 && (T == 1 || ldo % 4 == 0);
    const bool aligned = ((uintptr_t)Y & 15u) == 0 && (R <= 1 || ldy * hlq_dtype_bytes(ytype) % 16 == 0);
    const hipStream_t st = (hipStream_t)stream;
    hlq_clear_stale_error();
    if (ytype == HLQ_F16) launch_combine<HLQ_F16>(a, aligned, st);
    else if (ytype == HLQ_BF16) launch_combine<HLQ_BF16>(a, aligned, st);
    else launch_combine<HLQ_F32>(a, aligned, st);
    return hlq_hip_status(hipGetLastError());
}

}  // extern "C"
