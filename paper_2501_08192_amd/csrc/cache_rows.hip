// Rows into and out of the block-structured cache (psv_cache_append, psv_cache_gather).
//
// Bound by memory: rows are read and written once, 16 bytes a lane; the angles are shared by the heads of a row through LDS.
#include "rows.h"

namespace psv {

constexpr int kAppendThreads = 256, kAppendTileRows = 16;

// Where the channel 0 of a token's key and value lies in a pool of 2-byte elements, and the distance from channel to channel of a value.
struct Place {
    size_t k, v;
    uint32_t v_step;
};
__device__ __forceinline__ Place place16(int64_t slot, uint32_t h, uint32_t nkv, bool token_major)
{
    const size_t blk = (size_t)slot >> 4;
    const uint32_t off = (uint32_t)slot & 15;
    if (token_major) {
        const size_t at = ((blk * 16 + off) * nkv + h) * 128;
        return {at, at, 1};
    }
    return {((blk * nkv + h) * 16 + off) * 128, (blk * nkv + h) * 2048 + off, 16};
}

struct AppendArgs {
    psv_append_args a;
    psv_cache c;
    psv_rope rope;          // dims 0: not rotated
};

// A head is shared by 128 / 2N lanes; a lane has two vectors of N channels: of rotated halves the two partners, else neighbours.
template <uint32_t DT, bool HALF, bool Q8>
__global__ __launch_bounds__(kAppendThreads) void k_cache_append(AppendArgs g)
{
    using T = typename Elem<DT>::T;
    constexpr int N = Elem<DT>::N, LANES = 64 / N, HEADS = kAppendThreads / LANES;
    __shared__ float2 cs[kAppendTileRows * 64];
    const psv_append_args &a = g.a;
    const uint32_t row0 = blockIdx.x * kAppendTileRows, n_rows = min((uint32_t)kAppendTileRows, a.rows - row0), n = g.rope.dims / 2;
    const double m = g.rope.magnitude;
    for (uint32_t i = threadIdx.x; i < n_rows * n; i += kAppendThreads) {
        const uint32_t r = i / n, p = i % n;
        cs[r * 64 + p] = turn((double)a.positions[row0 + r] * g.rope.freq[p], m);
    }
    __syncthreads();
    const uint32_t lane = threadIdx.x % LANES, nq = a.n_q_heads, nkv = g.c.n_kv_heads, heads = nq + 2 * nkv;
    const bool turned = lane * 2 * N < 2 * n;
    const uint32_t lo = HALF && turned ? lane * N : lane * 2 * N, hi = HALF && turned ? n + lane * N : lo + N;
    const uint64_t n_slots = (uint64_t)g.c.num_pool_blocks * 16;
    for (uint32_t s = threadIdx.x / LANES; s < n_rows * heads; s += HEADS) {
        const uint32_t r = s / heads, h = s % heads;
        const int64_t row = row0 + r;
        const bool query = h < nq, key = !query && h < nq + nkv;
        const uint32_t kvh = key ? h - nq : h - nq - nkv;
        const T *x = query ? static_cast<const T *>(a.q) + row * a.q_row + h * 128
                   : key ? static_cast<const T *>(a.k) + row * a.k_row + kvh * 128
                         : static_cast<const T *>(a.v) + row * a.v_row + kvh * 128;
        float u[N], v[N];
        load_row<DT, N>(x + lo, u);
        load_row<DT, N>(x + hi, v);
        if ((query || key) && turned) {
            const float2 *c = cs + r * 64;
            if (HALF) {
#pragma unroll
                for (int e = 0; e < N; ++e) turn_pair(u[e], v[e], c[lo + e]);
            } else {
#pragma unroll
                for (int e = 0; e < N; e += 2) {
                    turn_pair(u[e], u[e + 1], c[(lo + e) / 2]);
                    turn_pair(v[e], v[e + 1], c[(hi + e) / 2]);
                }
            }
        }
        if (query) {
            T *y = static_cast<T *>(a.q_out) + row * a.q_out_row + h * 128;
            store_row<DT, N>(y + lo, u);
            store_row<DT, N>(y + hi, v);
            continue;
        }
        const int64_t slot = a.slots[row];
        if ((uint64_t)slot >= n_slots) continue;
        if constexpr (Q8) {
            float most = 0.f;
#pragma unroll
            for (int e = 0; e < N; ++e) most = fmaxf(most, fmaxf(fabsf(u[e]), fabsf(v[e])));
#pragma unroll
            for (int off = 1; off < LANES; off <<= 1) most = fmaxf(most, __shfl_xor(most, off, 64));
            const float scale = most > 0.f ? most / 127.0f : 1.0f;
            const uint32_t off = (uint32_t)slot & 15;
            uint8_t *unit = static_cast<uint8_t *>(key ? g.c.k_pool : g.c.v_pool) + ((size_t)(slot >> 4) * nkv + kvh) * PSV_KV_UNIT_BYTES_INT8;
            const uint32_t step = key ? 1 : 16;
            uint8_t *d = unit + (key ? off * 128 : off);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                d[(lo + e) * step] = quant_i8(u[e], scale);
                d[(hi + e) * step] = quant_i8(v[e], scale);
            }
            if (lane == 0) reinterpret_cast<float *>(unit + 2048)[off] = scale;
        } else {
            const Place at = place16(slot, kvh, nkv, g.c.kv_layout == PSV_KV_TOKEN_MAJOR);
            if (key || at.v_step == 1) {
                uint16_t *d = static_cast<uint16_t *>(key ? g.c.k_pool : g.c.v_pool) + (key ? at.k : at.v);
                store_row<PSV_BF16, N>(d + lo, u);
                store_row<PSV_BF16, N>(d + hi, v);
            } else {
                uint16_t *d = static_cast<uint16_t *>(g.c.v_pool) + at.v;
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    d[(lo + e) * 16] = (uint16_t)f32_to_bf16(u[e]);
                    d[(hi + e) * 16] = (uint16_t)f32_to_bf16(v[e]);
                }
            }
        }
    }
}

template <uint32_t DT, bool HALF>
static void launch_append_as(const AppendArgs &g, hipStream_t s)
{
    const dim3 grid((g.a.rows + kAppendTileRows - 1) / kAppendTileRows), block(kAppendThreads);
    if (g.c.kv_format == PSV_FMT_INT8) PSV_LAUNCH((k_cache_append<DT, HALF, true>), grid, block, 0, s, g);
    else PSV_LAUNCH((k_cache_append<DT, HALF, false>), grid, block, 0, s, g);
}

hipError_t launch_cache_append(const psv_append_args &a, const psv_cache &cache, const psv_rope *rope, hipStream_t s)
{
    AppendArgs g{};
    g.a = a;
    g.c = cache;
    if (rope) g.rope = *rope;
    const bool half = !rope || rope->pairing == PSV_ROPE_HALF;
    if (a.dtype == PSV_F32) half ? launch_append_as<PSV_F32, true>(g, s) : launch_append_as<PSV_F32, false>(g, s);
    else if (a.dtype == PSV_BF16) half ? launch_append_as<PSV_BF16, true>(g, s) : launch_append_as<PSV_BF16, false>(g, s);
    else half ? launch_append_as<PSV_F16, true>(g, s) : launch_append_as<PSV_F16, false>(g, s);
    return hipGetLastError();
}

struct GatherArgs {
    psv_gather_args a;
    psv_cache c;
};

template <uint32_t DT, bool Q8>
__global__ __launch_bounds__(kAppendThreads) void k_cache_gather(GatherArgs g)
{
    using T = typename Elem<DT>::T;
    constexpr int LANES = 16, HEADS = kAppendThreads / LANES;      // 8 channels a lane
    const psv_gather_args &a = g.a;
    const uint32_t row0 = blockIdx.x * kAppendTileRows, n_rows = min((uint32_t)kAppendTileRows, a.rows - row0);
    const uint32_t ch = threadIdx.x % LANES * 8, nkv = g.c.n_kv_heads;
    const uint64_t n_slots = (uint64_t)g.c.num_pool_blocks * 16;
    for (uint32_t s = threadIdx.x / LANES; s < n_rows * 2 * nkv; s += HEADS) {
        const uint32_t r = s / (2 * nkv), h = s % (2 * nkv);
        const int64_t row = row0 + r, slot = a.slots[row];
        if ((uint64_t)slot >= n_slots) continue;
        const bool key = h < nkv;
        const uint32_t kvh = key ? h : h - nkv;
        float v[8];
        if constexpr (Q8) {
            const uint32_t off = (uint32_t)slot & 15;
            const uint8_t *unit = static_cast<const uint8_t *>(key ? g.c.k_pool : g.c.v_pool) + ((size_t)(slot >> 4) * nkv + kvh) * PSV_KV_UNIT_BYTES_INT8;
            const float scale = reinterpret_cast<const float *>(unit + 2048)[off];
            const int8_t *d = reinterpret_cast<const int8_t *>(unit) + (key ? off * 128 : off);
            const uint32_t step = key ? 1 : 16;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (float)d[(ch + e) * step] * scale;
        } else {
            const Place at = place16(slot, kvh, nkv, g.c.kv_layout == PSV_KV_TOKEN_MAJOR);
            const uint16_t *d = static_cast<const uint16_t *>(key ? g.c.k_pool : g.c.v_pool) + (key ? at.k : at.v);
            const uint32_t step = key ? 1 : at.v_step;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = __uint_as_float((uint32_t)d[(ch + e) * step] << 16);
        }
        T *y = (key ? static_cast<T *>(a.k) + row * a.k_row : static_cast<T *>(a.v) + row * a.v_row) + kvh * 128;
        store_row<DT, 8>(y + ch, v);
    }
}

template <uint32_t DT>
static void launch_gather_as(const GatherArgs &g, hipStream_t s)
{
    const dim3 grid((g.a.rows + kAppendTileRows - 1) / kAppendTileRows), block(kAppendThreads);
    if (g.c.kv_format == PSV_FMT_INT8) PSV_LAUNCH((k_cache_gather<DT, true>), grid, block, 0, s, g);
    else PSV_LAUNCH((k_cache_gather<DT, false>), grid, block, 0, s, g);
}

hipError_t launch_cache_gather(const psv_gather_args &a, const psv_cache &cache, hipStream_t s)
{
    const GatherArgs g{a, cache};
    if (a.dtype == PSV_F32) launch_gather_as<PSV_F32>(g, s);
    else if (a.dtype == PSV_BF16) launch_gather_as<PSV_BF16>(g, s);
    else launch_gather_as<PSV_F16>(g, s);
    return hipGetLastError();
}

}  // namespace psv
