// Rows into and out of the block-structured cache (psv_cache_append, psv_cache_gather).
//
// Bound by memory: rows are read and written once, 16 bytes a lane; a row's angles are made once, by the workgroup that has it, and lie in
// LDS for all of its heads.  A value of the head-major layouts is a column of its block ([channel][16 tokens]): two bytes (int8: one) in each
// of 128 lines.  Its rows go through LDS, and where eight of them follow one another from a slot that is a multiple of eight on -- all of a
// prompt but its ends -- a lane moves one channel of the eight at once.  Such an octet belongs to the workgroup that has its first row, so that
// where tiles of rows end does not matter.  The two kinds of work are workgroups of their own, side by side in one launch.
// (Append of 9500 rows of 8 query and 2 kv heads, 58 MB: 11.8 us, 4.9 TB/s, with two-byte stores of values 22.6; of 3 x 1024 rows of 16 and 2 into
// an int8 cache, 30 MB: 10.1 us; gather of 24400 rows of 2 kv heads, 50 MB: 9.7 us, of 18000 int8 rows, 28 MB: 8.3 us.)
#include "rows.h"

namespace psv {

constexpr int kRowThreads = 256;
constexpr int kTurnTile = 8;         // most rows of a workgroup that rotates (9500 rows of 8 query and 2 kv heads: 12.0 us, with 16 rows 13.3)
constexpr int kColumnTile = 32;      // most rows of a workgroup that transposes values; and up to 7 more, of its last octet
constexpr int kColumnRows = kColumnTile + 7;

struct Place {
    size_t k, v;                     // elements to channel 0 of a token's key and value in pools of 2-byte elements
};
__device__ __forceinline__ Place place16(int64_t slot, uint32_t h, uint32_t nkv, bool token_major)
{
    const size_t blk = (size_t)slot >> 4;
    const uint32_t off = (uint32_t)slot & 15;
    if (token_major) {
        const size_t at = ((blk * 16 + off) * nkv + h) * 128;
        return {at, at};
    }
    return {((blk * nkv + h) * 16 + off) * 128, (blk * nkv + h) * 2048 + off};
}
// A token's (block, kv head) in an int8 pool
template <class P>
__device__ __forceinline__ P *unit8(P *pool, int64_t slot, uint32_t h, uint32_t nkv)
{
    return pool + ((size_t)(slot >> 4) * nkv + h) * PSV_KV_UNIT_BYTES_INT8;
}

// The rows [row0, row0 + tile) as a wave sees them: lane l has row row0 - 8 + l and its slot.
struct Columns {
    int64_t slot;
    uint64_t octets;                 // lanes whose row is the first of an octet of this tile
    uint64_t singles;                // ... or of this tile and in no octet
    uint64_t rows;                   // all rows that the tile's workgroup has
};
__device__ __forceinline__ Columns columns_of(const int64_t *slots, uint32_t rows, uint32_t row0, uint32_t tile, uint64_t n_slots)
{
    const int lane = threadIdx.x & 63;
    const int64_t r = (int64_t)row0 - 8 + lane;
    Columns c;
    c.slot = r >= 0 && r < (int64_t)rows && lane < (int)tile + 16 ? slots[r] : -1;
    const bool valid = (uint64_t)c.slot < n_slots;
    const uint64_t ok = __ballot(valid), first = __ballot(valid && (c.slot & 7) == 0), next = __ballot(valid && c.slot == __shfl_up(c.slot, 1, 64) + 1);
    const uint64_t a = next >> 1, b = a & (a >> 1), d = b & (b >> 2), whole = first & d & (d >> 3);      // the seven rows behind it follow
    const uint64_t mine = ((1ull << tile) - 1) << 8;
    auto spread = [](uint64_t x) { x |= x << 1; x |= x << 2; return x | x << 4; };
    c.octets = whole & mine;
    c.singles = ok & mine & ~spread(whole);
    c.rows = spread(c.octets) | c.singles;
    return c;
}
// The n-th set bit of x (n below their number).
__device__ __forceinline__ int nth_bit(uint64_t x, uint32_t n)
{
    for (uint32_t i = 0; i < n; ++i) x &= x - 1;
    return __builtin_ctzll(x);
}

struct AppendArgs {
    psv_append_args a;
    psv_cache c;
    uint32_t dims;                   // rotated channels; 0: not rotated
    double magnitude, freq[PSV_HEAD_DIM / 2];
    uint32_t turn_tile, turn_groups;             // workgroups [0, turn_groups): rotate
    uint32_t column_tile, column_groups;         // the others: values by columns, column_groups of them a kv head
    uint32_t heads;                              // of a row in a rotating workgroup: queries, keys and, where they are rows, values
};

// Codes of N values of a row, clamp(rint(v / scale), -127, 127).  A correctly rounded division is some ten instructions; the product with 1 / scale
// is within 127 * 2^-22 of it, so that both round to the same code unless the product is that near the middle between two: then, for
// scales whose reciprocal overflows, and where a product is no number (a NaN, an infinity times zero; the maximum hands it on), the division decides.  (Appending 8192 rows of 8 query and 8 kv heads: 21.3 us, with divisions 23.8.)
template <int N>
__device__ __forceinline__ void store_codes(uint8_t *p, const float (&v)[N], float scale)
{
    const float kMagic = 12582912.0f, r = 1.0f / scale;      // 1.5 * 2^23: adding it rounds to an integer (ties to even), which its low byte holds
    uint32_t w[N / 4];
    float far = 0.f;
#pragma unroll
    for (int e = 0; e < N; e += 4) {
        float m[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            m[k] = fmaf(v[e + k], r, kMagic);
            far = __builtin_elementwise_maximum(far, fabsf(fmaf(v[e + k], r, -(m[k] - kMagic))));
        }
        w[e / 4] = pack_magic_bytes(m[0], m[1], m[2], m[3]);
    }
    if (!(far < 0.4999f) || !(scale > 1e-30f)) {
#pragma unroll
        for (int e = 0; e < N; e += 4)
            w[e / 4] = quant_i8(v[e], scale) | (uint32_t)quant_i8(v[e + 1], scale) << 8 | (uint32_t)quant_i8(v[e + 2], scale) << 16 | (uint32_t)quant_i8(v[e + 3], scale) << 24;
    }
#pragma unroll
    for (int e = 0; e < N / 4; ++e) reinterpret_cast<uint32_t *>(p)[e] = w[e];
}

// Queries, keys and row-stored values: a head is shared by 128 / 2N lanes; a lane has two vectors of N channels: of rotated halves the two
// partners, else neighbours.
template <uint32_t DT, bool HALF, bool Q8>
__device__ __forceinline__ void append_rows(const AppendArgs &g, float2 *cs, int64_t *slots)
{
    using T = typename Elem<DT>::T;
    constexpr int N = Elem<DT>::N, LANES = 64 / N, HEADS = kRowThreads / LANES;
    const psv_append_args &a = g.a;
    const uint32_t row0 = blockIdx.x * g.turn_tile, n_rows = min(g.turn_tile, a.rows - row0), n = g.dims / 2;
    const double m = g.magnitude;
    const uint32_t lane = threadIdx.x % LANES, nq = a.n_q_heads, nkv = g.c.n_kv_heads, heads = g.heads;
    const bool turned = lane * 2 * N < 2 * n;
    const uint32_t lo = HALF && turned ? lane * N : lane * 2 * N, hi = HALF && turned ? n + lane * N : lo + N;
    const uint64_t n_slots = (uint64_t)g.c.num_pool_blocks * 16;
    const uint32_t step_r = HEADS / heads, step_h = HEADS % heads;
    uint32_t r = threadIdx.x / LANES / heads, h = threadIdx.x / LANES % heads;
    Pack<DT, N> next_u, next_v;
    auto request = [&]() {
        const int64_t row = row0 + r;
        const T *x = h < nq ? static_cast<const T *>(a.q) + row * a.q_row + h * 128
                   : h < nq + nkv ? static_cast<const T *>(a.k) + row * a.k_row + (h - nq) * 128
                                  : static_cast<const T *>(a.v) + row * a.v_row + (h - nq - nkv) * 128;
        next_u = fetch_row<DT, N>(x + lo);
        next_v = fetch_row<DT, N>(x + hi);
    };
    if (r < n_rows) request();
    for (int i = threadIdx.x; i < (int)n_rows; i += kRowThreads) slots[i] = a.slots[row0 + i];
    for (uint32_t i = threadIdx.x; i < n_rows * 64; i += kRowThreads) {
        const uint32_t p = i & 63;
        if (p < n) cs[i] = turn((double)a.positions[row0 + (i >> 6)] * g.freq[p], m);
    }
    __syncthreads();
    while (r < n_rows) {
        const uint32_t at_r = r, at_h = h;
        const int64_t row = row0 + at_r;
        const bool query = at_h < nq, key = !query && at_h < nq + nkv;
        const uint32_t kvh = key ? at_h - nq : at_h - nq - nkv;
        float u[N], v[N];
        unpack_row<DT, N>(next_u, u);
        unpack_row<DT, N>(next_v, v);
        r += step_r;
        h += step_h;
        if (h >= heads) {
            h -= heads;
            ++r;
        }
        if (r < n_rows) request();
        if ((query || key) && turned) {
            const float2 *c = cs + at_r * 64;
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
            T *y = static_cast<T *>(a.q_out) + row * a.q_out_row + at_h * 128;
            store_row<DT, N>(y + lo, u);
            store_row<DT, N>(y + hi, v);
            continue;
        }
        const int64_t slot = slots[at_r];
        if ((uint64_t)slot >= n_slots) continue;
        if constexpr (Q8) {
            float most = 0.f;
#pragma unroll
            for (int e = 0; e < N; ++e) most = fmaxf(most, fmaxf(fabsf(u[e]), fabsf(v[e])));
#pragma unroll
            for (int off = 1; off < LANES; off <<= 1) most = fmaxf(most, __shfl_xor(most, off, 64));
            const float scale = most > 0.f ? most / 127.0f : 1.0f;
            const uint32_t off = (uint32_t)slot & 15;
            uint8_t *unit = unit8(static_cast<uint8_t *>(g.c.k_pool), slot, kvh, nkv);
            store_codes<N>(unit + off * 128 + lo, u, scale);
            store_codes<N>(unit + off * 128 + hi, v, scale);
            if (lane == 0) reinterpret_cast<float *>(unit + 2048)[off] = scale;
        } else {
            const Place at = place16(slot, kvh, nkv, g.c.kv_layout == PSV_KV_TOKEN_MAJOR);
            uint16_t *d = static_cast<uint16_t *>(key ? g.c.k_pool : g.c.v_pool) + (key ? at.k : at.v);
            store_row<PSV_BF16, N>(d + lo, u);
            store_row<PSV_BF16, N>(d + hi, v);
        }
    }
}

// Values of one kv head by columns.  Rows in LDS are 17 (int8: 9) pieces of 16 bytes apart, so that the two halves of a block that a wave reads
// at once, eight rows apart, lie in different banks.
constexpr int kColumnStride = 272, kColumnStride8 = 144;

template <uint32_t DT, bool Q8>
__device__ __forceinline__ void append_columns(const AppendArgs &g, uint8_t *rows)
{
    using T = typename Elem<DT>::T;
    constexpr int N = Elem<DT>::N, LANES = 128 / N, ROWS = kRowThreads / LANES, STRIDE = Q8 ? kColumnStride8 : kColumnStride;
    const psv_append_args &a = g.a;
    const uint32_t at = blockIdx.x - g.turn_groups, kvh = at / g.column_groups, row0 = at % g.column_groups * g.column_tile, nkv = g.c.n_kv_heads;
    const Columns c = columns_of(a.slots, a.rows, row0, g.column_tile, (uint64_t)g.c.num_pool_blocks * 16);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t ch = threadIdx.x % LANES * N;
#pragma unroll
    for (int i = 0; i < (kColumnRows + ROWS - 1) / ROWS; ++i) {
        const uint32_t r = i * ROWS + threadIdx.x / LANES;           // row row0 + r, lane 8 + r of the wave's view
        const int64_t slot = __shfl(c.slot, (int)min(8 + r, 63u), 64);
        if (8 + r > 63 || !(c.rows >> (8 + r) & 1)) continue;
        float v[N];
        load_row<DT, N>(static_cast<const T *>(a.v) + (int64_t)(row0 + r) * a.v_row + kvh * 128 + ch, v);
        if constexpr (Q8) {
            float most = 0.f;
#pragma unroll
            for (int e = 0; e < N; ++e) most = fmaxf(most, fabsf(v[e]));
#pragma unroll
            for (int off = 1; off < LANES; off <<= 1) most = fmaxf(most, __shfl_xor(most, off, 64));
            const float scale = most > 0.f ? most / 127.0f : 1.0f;
            store_codes<N>(rows + r * STRIDE + ch, v, scale);
            if (ch == 0) reinterpret_cast<float *>(unit8(static_cast<uint8_t *>(g.c.v_pool), slot, kvh, nkv) + 2048)[slot & 15] = scale;
        } else {
            store_row<PSV_BF16, N>(reinterpret_cast<uint16_t *>(rows + r * STRIDE) + ch, v);
        }
    }
    __syncthreads();
    // octets, two at a time so that both halves of a block leave together: a wave has 32 channels of them
    const uint32_t n = __popcll(c.octets), odd = n && (__shfl(c.slot, n ? __builtin_ctzll(c.octets) : 0, 64) & 8) ? 1 : 0;
    const uint32_t half = lane & 1, chan = wave * 32 + lane / 2;
    for (uint32_t pair = 0; pair * 2 < n + odd; ++pair) {
        const uint32_t k = pair * 2 + half - odd;                    // wraps far beyond n where there is none
        const int first = k < n ? nth_bit(c.octets, k) : 8;
        const int64_t slot = __shfl(c.slot, first, 64);
        if (k >= n) continue;
        const uint8_t *src = rows + (first - 8) * STRIDE;
        if constexpr (Q8) {
            uint32_t w[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i / 4] |= (uint32_t)src[i * STRIDE + chan] << (i % 4 * 8);
            *reinterpret_cast<uint2 *>(unit8(static_cast<uint8_t *>(g.c.v_pool), slot, kvh, nkv) + chan * 16 + (slot & 15)) = make_uint2(w[0], w[1]);
        } else {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[i] = (uint32_t)reinterpret_cast<const uint16_t *>(src + 2 * i * STRIDE)[chan] |
                       (uint32_t)reinterpret_cast<const uint16_t *>(src + (2 * i + 1) * STRIDE)[chan] << 16;
            *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(g.c.v_pool) + place16(slot, kvh, nkv, false).v + chan * 16) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    uint64_t left = c.singles;
    for (int k = 0; left; ++k, left &= left - 1) {
        if ((k & 3) != wave) continue;
        const int l = __builtin_ctzll(left);
        const int64_t slot = __shfl(c.slot, l, 64);
        const uint8_t *src = rows + (l - 8) * STRIDE;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t channel = i * 64 + lane;
            if constexpr (Q8) unit8(static_cast<uint8_t *>(g.c.v_pool), slot, kvh, nkv)[channel * 16 + (slot & 15)] = src[channel];
            else static_cast<uint16_t *>(g.c.v_pool)[place16(slot, kvh, nkv, false).v + channel * 16] = reinterpret_cast<const uint16_t *>(src)[channel];
        }
    }
}

template <uint32_t DT, bool HALF, bool Q8>
__global__ __launch_bounds__(kRowThreads) void k_cache_append(AppendArgs g)
{
    static_assert(kTurnTile * (512 + 8) <= kColumnRows * kColumnStride, "a tile's angles and slots");
    __shared__ __align__(16) uint8_t lds[kColumnRows * kColumnStride];
    if (blockIdx.x < g.turn_groups) append_rows<DT, HALF, Q8>(g, reinterpret_cast<float2 *>(lds), reinterpret_cast<int64_t *>(lds + kTurnTile * 512));
    else append_columns<DT, Q8>(g, lds);
}

template <uint32_t DT, bool HALF>
static void launch_append_as(const AppendArgs &g, hipStream_t s)
{
    const dim3 grid(g.turn_groups + g.column_groups * g.c.n_kv_heads), block(kRowThreads);
    if (g.c.kv_format == PSV_FMT_INT8) PSV_LAUNCH((k_cache_append<DT, HALF, true>), grid, block, 0, s, g);
    else PSV_LAUNCH((k_cache_append<DT, HALF, false>), grid, block, 0, s, g);
}

// Rows a workgroup takes: the most, or fewer until every compute unit has a workgroup.
static uint32_t tile_of(uint32_t rows, uint32_t most)
{
    while (most > 1 && rows / most < 256) most /= 2;
    return most;
}

hipError_t launch_cache_append(const psv_append_args &a, const psv_cache &cache, const psv_rope *rope, hipStream_t s)
{
    AppendArgs g{};
    g.a = a;
    g.c = cache;
    if (rope) {
        g.dims = rope->dims;
        g.magnitude = rope->magnitude;
        for (uint32_t i = 0; i < rope->dims / 2; ++i) g.freq[i] = rope->freq[i];
    }
    const bool columns = cache.kv_layout == PSV_KV_HEAD_MAJOR;
    g.heads = a.n_q_heads + cache.n_kv_heads * (columns ? 1 : 2);
    // three heads a lane (2 / 3 / 4: 9500 rows of 10 heads 12.8 / 11.5 / 11.5 us, 16384 of 18 34.1 / 35.3 / 37.3, 16384 of 24 in 32 bits 63.7 /
    // 65.2 / 65.4; with twelve 71.4)
    const uint32_t most = 3 * (a.dtype == PSV_F32 ? kRowThreads / 16 : kRowThreads / 8) / g.heads;
    g.turn_tile = tile_of(a.rows, most < 1 ? 1 : most < (uint32_t)kTurnTile ? most : kTurnTile);
    g.turn_groups = (a.rows + g.turn_tile - 1) / g.turn_tile;
    g.column_tile = tile_of(a.rows * cache.n_kv_heads, kColumnTile);
    g.column_groups = columns ? (a.rows + g.column_tile - 1) / g.column_tile : 0;
    // Both kinds together in one grid: with 2^24 rows and 2^28 kv heads at most, 2^22 of four rows and 2^23 + 128 of columns fit.
    while (g.turn_groups + g.column_groups * cache.n_kv_heads > kMostGroups) {
        g.turn_tile *= 2;
        g.turn_groups = (a.rows + g.turn_tile - 1) / g.turn_tile;
    }
    const bool half = !rope || rope->pairing == PSV_ROPE_HALF;
    if (a.dtype == PSV_F32) half ? launch_append_as<PSV_F32, true>(g, s) : launch_append_as<PSV_F32, false>(g, s);
    else if (a.dtype == PSV_BF16) half ? launch_append_as<PSV_BF16, true>(g, s) : launch_append_as<PSV_BF16, false>(g, s);
    else half ? launch_append_as<PSV_F16, true>(g, s) : launch_append_as<PSV_F16, false>(g, s);
    return hipGetLastError();
}

struct GatherArgs {
    psv_gather_args a;
    psv_cache c;
    uint32_t row_tile, row_groups;               // workgroups [0, row_groups): what lies in the cache as rows
    uint32_t column_tile, column_groups;         // the others: values by columns, column_groups of them a kv head
};

template <uint32_t DT, bool Q8>
__device__ __forceinline__ void gather_rows(const GatherArgs &g, int64_t *slots)
{
    using T = typename Elem<DT>::T;
    constexpr int LANES = 16, HEADS = kRowThreads / LANES;      // 8 channels a lane
    const psv_gather_args &a = g.a;
    const uint32_t row0 = blockIdx.x * g.row_tile, n_rows = min(g.row_tile, a.rows - row0);
    const uint32_t ch = threadIdx.x % LANES * 8, nkv = g.c.n_kv_heads, heads = g.column_groups ? nkv : 2 * nkv;
    const uint64_t n_slots = (uint64_t)g.c.num_pool_blocks * 16;
    const uint32_t step_r = HEADS / heads, step_h = HEADS % heads;
    uint32_t r = threadIdx.x / LANES / heads, h = threadIdx.x / LANES % heads;
    for (int i = threadIdx.x; i < (int)n_rows; i += kRowThreads) slots[i] = a.slots[row0 + i];
    __syncthreads();
    constexpr uint32_t kBytes = Q8 ? 8 : 16;
    struct alignas(kBytes) Piece { uint32_t w[kBytes / 4]; };
    Piece next{};
    float next_scale = 1.f;
    auto request = [&]() {
        const int64_t slot = slots[r];
        if ((uint64_t)slot >= n_slots) return;
        const bool key = h < nkv;
        if constexpr (Q8) {
            const uint8_t *unit = unit8(static_cast<const uint8_t *>(g.c.k_pool), slot, h, nkv);
            next_scale = reinterpret_cast<const float *>(unit + 2048)[slot & 15];
            next = *reinterpret_cast<const Piece *>(unit + (slot & 15) * 128 + ch);
        } else {
            const Place at = place16(slot, key ? h : h - nkv, nkv, g.c.kv_layout == PSV_KV_TOKEN_MAJOR);
            next = *reinterpret_cast<const Piece *>(static_cast<const uint16_t *>(key ? g.c.k_pool : g.c.v_pool) + (key ? at.k : at.v) + ch);
        }
    };
    if (r < n_rows) request();
    while (r < n_rows) {
        const uint32_t at_r = r, at_h = h;
        const Piece p = next;
        const float scale = next_scale;
        r += step_r;
        h += step_h;
        if (h >= heads) {
            h -= heads;
            ++r;
        }
        if (r < n_rows) request();
        if ((uint64_t)slots[at_r] >= n_slots) continue;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (Q8) v[e] = (float)(int8_t)(p.w[e / 4] >> (e % 4 * 8)) * scale;
            else v[e] = e & 1 ? bf16_hi(p.w[e / 2]) : bf16_lo(p.w[e / 2]);
        }
        const int64_t row = row0 + at_r;
        T *y = at_h < nkv ? static_cast<T *>(a.k) + row * a.k_row + at_h * 128 : static_cast<T *>(a.v) + row * a.v_row + (at_h - nkv) * 128;
        store_row<DT, 8>(y + ch, v);
    }
}

// append_columns the other way round
template <uint32_t DT, bool Q8>
__device__ __forceinline__ void gather_columns(const GatherArgs &g, uint8_t *rows)
{
    using T = typename Elem<DT>::T;
    constexpr int LANES = 16, ROWS = kRowThreads / LANES, STRIDE = Q8 ? kColumnStride8 : kColumnStride;
    const psv_gather_args &a = g.a;
    const uint32_t at = blockIdx.x - g.row_groups, kvh = at / g.column_groups, row0 = at % g.column_groups * g.column_tile, nkv = g.c.n_kv_heads;
    const Columns c = columns_of(a.slots, a.rows, row0, g.column_tile, (uint64_t)g.c.num_pool_blocks * 16);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t n = __popcll(c.octets), odd = n && (__shfl(c.slot, n ? __builtin_ctzll(c.octets) : 0, 64) & 8) ? 1 : 0;
    const uint32_t half = lane & 1, chan = wave * 32 + lane / 2;
    for (uint32_t pair = 0; pair * 2 < n + odd; ++pair) {
        const uint32_t k = pair * 2 + half - odd;
        const int first = k < n ? nth_bit(c.octets, k) : 8;
        const int64_t slot = __shfl(c.slot, first, 64);
        if (k >= n) continue;
        uint8_t *dst = rows + (first - 8) * STRIDE;
        if constexpr (Q8) {
            const uint2 w = *reinterpret_cast<const uint2 *>(unit8(static_cast<const uint8_t *>(g.c.v_pool), slot, kvh, nkv) + chan * 16 + (slot & 15));
#pragma unroll
            for (int i = 0; i < 8; ++i) dst[i * STRIDE + chan] = (uint8_t)((i < 4 ? w.x : w.y) >> (i % 4 * 8));
        } else {
            const uint4 q = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(g.c.v_pool) + place16(slot, kvh, nkv, false).v + chan * 16);
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) reinterpret_cast<uint16_t *>(dst + i * STRIDE)[chan] = (uint16_t)(w[i / 2] >> (i % 2 * 16));
        }
    }
    uint64_t left = c.singles;
    for (int k = 0; left; ++k, left &= left - 1) {
        if ((k & 3) != wave) continue;
        const int l = __builtin_ctzll(left);
        const int64_t slot = __shfl(c.slot, l, 64);
        uint8_t *dst = rows + (l - 8) * STRIDE;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t channel = i * 64 + lane;
            if constexpr (Q8) dst[channel] = unit8(static_cast<const uint8_t *>(g.c.v_pool), slot, kvh, nkv)[channel * 16 + (slot & 15)];
            else reinterpret_cast<uint16_t *>(dst)[channel] = static_cast<const uint16_t *>(g.c.v_pool)[place16(slot, kvh, nkv, false).v + channel * 16];
        }
    }
    __syncthreads();
    const uint32_t ch = threadIdx.x % LANES * 8;
#pragma unroll
    for (int i = 0; i < (kColumnRows + ROWS - 1) / ROWS; ++i) {
        const uint32_t r = i * ROWS + threadIdx.x / LANES;
        const int64_t slot = __shfl(c.slot, (int)min(8 + r, 63u), 64);
        if (8 + r > 63 || !(c.rows >> (8 + r) & 1)) continue;
        float v[8];
        if constexpr (Q8) {
            const float scale = reinterpret_cast<const float *>(unit8(static_cast<const uint8_t *>(g.c.v_pool), slot, kvh, nkv) + 2048)[slot & 15];
            const uint2 w = *reinterpret_cast<const uint2 *>(rows + r * STRIDE + ch);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (float)(int8_t)((e < 4 ? w.x : w.y) >> (e % 4 * 8)) * scale;
        } else {
            load_row<PSV_BF16, 8>(reinterpret_cast<const uint16_t *>(rows + r * STRIDE) + ch, v);
        }
        store_row<DT, 8>(static_cast<T *>(a.v) + (int64_t)(row0 + r) * a.v_row + kvh * 128 + ch, v);
    }
}

template <uint32_t DT, bool Q8>
__global__ __launch_bounds__(kRowThreads) void k_cache_gather(GatherArgs g)
{
    __shared__ __align__(16) uint8_t lds[kColumnRows * (Q8 ? kColumnStride8 : kColumnStride)];
    if (blockIdx.x < g.row_groups) gather_rows<DT, Q8>(g, reinterpret_cast<int64_t *>(lds));
    else gather_columns<DT, Q8>(g, lds);
}

template <uint32_t DT>
static void launch_gather_as(const GatherArgs &g, hipStream_t s)
{
    const dim3 grid(g.row_groups + g.column_groups * g.c.n_kv_heads), block(kRowThreads);
    if (g.c.kv_format == PSV_FMT_INT8) PSV_LAUNCH((k_cache_gather<DT, true>), grid, block, 0, s, g);
    else PSV_LAUNCH((k_cache_gather<DT, false>), grid, block, 0, s, g);
}

hipError_t launch_cache_gather(const psv_gather_args &a, const psv_cache &cache, hipStream_t s)
{
    const bool columns = cache.kv_layout == PSV_KV_HEAD_MAJOR;
    // (A grid of all of them fits: one row a workgroup are 2^28 / 17 groups at most, token-major, or 2^28 / 33 and 2^23 + 33 of columns.)  Four
    // heads a lane of what lies as rows (16384 rows of 8 kv heads, token-major: 28.7 us, with 32 heads a lane 39.5)
    const uint32_t most = 4 * (kRowThreads / 16) / (cache.n_kv_heads * (columns ? 1 : 2));
    GatherArgs g{a, cache, tile_of(a.rows, most < 1 ? 1 : most < (uint32_t)kColumnTile ? most : kColumnTile), 0, tile_of(a.rows * cache.n_kv_heads, kColumnTile), 0};
    g.row_groups = (a.rows + g.row_tile - 1) / g.row_tile;
    g.column_groups = columns ? (a.rows + g.column_tile - 1) / g.column_tile : 0;
    if (a.dtype == PSV_F32) launch_gather_as<PSV_F32>(g, s);
    else if (a.dtype == PSV_BF16) launch_gather_as<PSV_BF16>(g, s);
    else launch_gather_as<PSV_F16>(g, s);
    return hipGetLastError();
}

}  // namespace psv
