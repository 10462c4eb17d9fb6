// Log probabilities of given tokens, entropy and the most likely tokens (psv_logprobs_part, psv_logprobs_join).
//
// With M the largest logit of a row, d = x - M (exact, or one rounding) and e = exp(s d):  ln p = s d - ln(sum e), entropy = ln(sum e) -
// s (sum e d) / (sum e).  A workgroup reduces a piece of a row, its record, to (M, sum e, sum e d), the given tokens' logits and its largest
// `top`; records are joined by rescaling their sums to the common M.  All sums are 32 bits; e d <= 0, so that nothing cancels.
//
// Bound by memory: a piece is read once, into registers, all loads at once, and everything else -- the maximum, the sums, the
// alternatives -- is made from there.
//
// Alternatives without sorting: the top-th largest of the lanes' maxima is a bound T that at least `top` logits reach, and of every lane
// but `top` none exceeds it; so at most top * (columns a lane) logits exceed T, usually about `top`.  Those that reach it are collected in LDS and
// each one's rank counted.  Where more equal ones reach T than the list holds, the same bound on the ids of those equal to T
// cuts them to top * (columns a lane) in all, which the list holds.
#include "rows.h"

namespace psv {

constexpr int kWaves = kLogprobThreads / 64;
constexpr uint32_t kList = PSV_LOGPROBS_MAX_TOP * 64;

// Order of floats as unsigned integers (-0 counts as 0; no NaN)
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t b = __float_as_uint(x + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_order(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o); }
constexpr uint32_t kOrderNone = 0x007fffffu;      // of -infinity

// The k-th largest of the workgroup's kLogprobThreads values (k <= threads), or a lower value that exactly k of them reach: bit by bit
// from the top, counted by the lanes of one wave.
__device__ __forceinline__ uint32_t kth_largest(uint32_t v, uint32_t k, uint32_t *tmp)
{
    tmp[threadIdx.x] = v;
    __syncthreads();
    if (threadIdx.x < 64) {
        uint32_t w[kWaves], t = 0;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) w[i] = tmp[i * 64 + threadIdx.x];
        for (uint32_t bit = 1u << 31; bit; bit >>= 1) {
            uint32_t n = 0;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) n += __popcll(__ballot(w[i] >= (t | bit)));
            if (n >= k) t |= bit;
            if (n == k) break;
        }
        if (threadIdx.x == 0) tmp[kLogprobThreads] = t;
    }
    __syncthreads();
    return tmp[kLogprobThreads];
}

// Ranks of the n listed (order, id) among themselves; the first `top` go to values and ids, what is missing is filled up.
__device__ __forceinline__ void write_ranked(const uint2 *list, uint32_t n, uint32_t top, float *values, int32_t *ids)
{
    for (uint32_t i = threadIdx.x; i < n; i += kLogprobThreads) {
        const uint2 me = list[i];
        uint32_t rank = 0;
        for (uint32_t j = 0; j < n; ++j) {
            const uint2 o = list[j];
            rank += o.x > me.x || (o.x == me.x && o.y < me.y);
        }
        if (rank < top) {
            values[rank] = of_order(me.x);
            ids[rank] = (int32_t)me.y;
        }
    }
    for (uint32_t i = n + threadIdx.x; i < top; i += kLogprobThreads) {
        values[i] = -INFINITY;
        ids[i] = -1;
    }
}

__device__ __forceinline__ float block_sum(float v, float *tmp)
{
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
    __syncthreads();
    const float t = (tmp[0] + tmp[1]) + (tmp[2] + tmp[3]);
    __syncthreads();
    return t;
}
__device__ __forceinline__ float block_max(float v, float *tmp)
{
    v = wave_max(v);
    if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
    __syncthreads();
    const float t = fmaxf(fmaxf(tmp[0], tmp[1]), fmaxf(tmp[2], tmp[3]));
    __syncthreads();
    return t;
}

struct PartArgs {
    psv_logprobs_args a;
    float *records;
    uint32_t chunk;
    float to_log2;          // scale * log2(e)
};

// A record: M, sum e, sum e d, unused; the given tokens' logits (-infinity: not in this piece); the largest logits; their ids.
__host__ __device__ inline uint32_t record_floats(uint32_t given, uint32_t top) { return 4 + given + 2 * top; }

template <uint32_t DT, int E>
__global__ __launch_bounds__(kLogprobThreads) void k_logprobs_part(PartArgs g)
{
    using T = typename Elem<DT>::T;
    constexpr int N = Elem<DT>::N;
    struct __attribute__((packed, aligned(sizeof(T)))) Loose { Pack<DT, N> p; };      // rows of any alignment
    __shared__ float tmp[kWaves];
    __shared__ uint32_t lanes[kLogprobThreads + 1], count;
    __shared__ uint2 list[kList];
    const psv_logprobs_args &a = g.a;
    const uint32_t row = blockIdx.x / a.records, rec = blockIdx.x % a.records;
    const uint32_t c0 = min(rec * g.chunk, a.columns), c1 = min(c0 + g.chunk, a.columns);
    const T *px = static_cast<const T *>(a.logits) + (int64_t)row * a.row;
    float *out = g.records + (size_t)blockIdx.x * record_floats(a.given, a.top);
    if (threadIdx.x < a.given) {
        const int64_t t = (int64_t)a.tokens[(size_t)row * a.given + threadIdx.x] - a.first_token;
        out[4 + threadIdx.x] = t >= c0 && t < c1 ? Elem<DT>::get(px[t]) : -INFINITY;
    }
    float x[E];
#pragma unroll
    for (int j = 0; j < E / N; ++j) {
        const uint32_t c = c0 + (j * kLogprobThreads + threadIdx.x) * N;
        if (c + N <= c1) {
            const Pack<DT, N> p = reinterpret_cast<const Loose *>(px + c)->p;
#pragma unroll
            for (int e = 0; e < N; ++e) x[j * N + e] = Elem<DT>::get(p.e[e]);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) x[j * N + e] = c + e < c1 ? Elem<DT>::get(px[c + e]) : -INFINITY;
        }
    }
    float mine = -INFINITY;
#pragma unroll
    for (int e = 0; e < E; ++e) mine = fmaxf(mine, x[e]);
    const float M = block_max(mine, tmp), ref = M == -INFINITY ? 0.f : M;
    float s = 0.f, w = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float d = x[e] - ref, p = exp2_raw(d * g.to_log2);
        s += p;
        w = fmaf(p, p > 0.f ? d : 0.f, w);      // a masked logit has no part
    }
    s = block_sum(s, tmp);
    w = block_sum(w, tmp);
    if (threadIdx.x == 0) {
        out[0] = M;
        out[1] = s;
        out[2] = w;
        out[3] = 0.f;
    }
    if (a.top == 0) return;

    float *values = out + 4 + a.given;
    int32_t *ids = reinterpret_cast<int32_t *>(values + a.top);
    if (!(s == s)) {                            // a NaN or +infinity: no alternatives
        write_ranked(list, 0, a.top, values, ids);
        return;
    }
    auto id_of = [&](int e) { return c0 + ((e / N) * kLogprobThreads + threadIdx.x) * N + e % N; };
    uint32_t bound = kth_largest(order_of(mine), a.top, lanes);
    if (bound <= kOrderNone) bound = kOrderNone + 1;
    const float least = of_order(bound);
    uint32_t last = ~0u;                        // highest id taken of those equal to `least`
    for (int pass = 0;; ++pass) {
        if (threadIdx.x == 0) count = 0;
        __syncthreads();
        if (mine >= least) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (x[e] >= least) {
                    const uint32_t id = id_of(e);
                    if (x[e] > least || id <= last) {
                        const uint32_t at = atomicAdd(&count, 1u);
                        if (at < kList) list[at] = make_uint2(order_of(x[e]), id);
                    }
                }
        }
        __syncthreads();
        if (count <= kList || pass) break;
        // too many equal ones: those lanes that exceed the bound count first, then the lanes by their first id
        uint32_t key = 0;
        if (mine > least) key = ~0u;
        else if (mine == least) {
            uint32_t first = ~0u;
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (x[e] == least) first = min(first, id_of(e));
            key = ~first;
        }
        __syncthreads();
        last = ~kth_largest(key, a.top, lanes);
    }
    const uint32_t n = min(count, kList);
    for (uint32_t i = threadIdx.x; i < n; i += kLogprobThreads) list[i].y += a.first_token;
    __syncthreads();
    write_ranked(list, n, a.top, values, ids);
}

template <uint32_t DT>
static void launch_part_as(const PartArgs &g, hipStream_t s)
{
    const dim3 grid(g.a.rows * g.a.records), block(kLogprobThreads);
    if (g.chunk <= kLogprobThreads * 8) PSV_LAUNCH((k_logprobs_part<DT, 8>), grid, block, 0, s, g);
    else if (g.chunk <= kLogprobThreads * 16) PSV_LAUNCH((k_logprobs_part<DT, 16>), grid, block, 0, s, g);
    else if (g.chunk <= kLogprobThreads * 32) PSV_LAUNCH((k_logprobs_part<DT, 32>), grid, block, 0, s, g);
    else PSV_LAUNCH((k_logprobs_part<DT, 64>), grid, block, 0, s, g);
}

hipError_t launch_logprobs_part(const psv_logprobs_args &a, float *records, hipStream_t s)
{
    const PartArgs g{a, records, logprob_chunk(a.columns, a.records), a.scale * 1.4426950408889634f};
    if (a.dtype == PSV_F32) launch_part_as<PSV_F32>(g, s);
    else if (a.dtype == PSV_BF16) launch_part_as<PSV_BF16>(g, s);
    else launch_part_as<PSV_F16>(g, s);
    return hipGetLastError();
}

struct JoinArgs {
    psv_logprobs_args a;
    const float *records;   // [shards][rows][records] of them
    uint32_t shards;
    psv_logprobs_out out;
};

__global__ __launch_bounds__(kLogprobThreads) void k_logprobs_join(JoinArgs g)
{
    __shared__ float tmp[kWaves], values[PSV_LOGPROBS_MAX_TOP];
    __shared__ int32_t ids[PSV_LOGPROBS_MAX_TOP];
    __shared__ uint32_t lanes[kLogprobThreads + 1], count;
    __shared__ uint2 list[kList];
    const psv_logprobs_args &a = g.a;
    const uint32_t row = blockIdx.x, size = record_floats(a.given, a.top), n_rec = g.shards * a.records;
    auto record = [&](uint32_t i) { return g.records + (((size_t)(i / a.records) * a.rows + row) * a.records + i % a.records) * size; };
    float m = -INFINITY, s = 0.f, w = 0.f;
    if (threadIdx.x < n_rec) {
        const float *r = record(threadIdx.x);
        m = r[0];
        s = r[1];
        w = r[2];
    }
    const float M = block_max(m, tmp);
    if (m > -INFINITY || s != s) {
        const float d = m - M, f = exp2_raw(d * a.scale * 1.4426950408889634f);
        w = f * (w + (f > 0.f ? s * d : 0.f));
        s *= f;
    }
    const float S = block_sum(s, tmp), W = block_sum(w, tmp);
    const bool bad = !(S == S), none = S == 0.f;
    const float ln_s = logf(S);
    auto answer = [&](float x) { return bad ? __uint_as_float(0x7fc00000u) : none || x == -INFINITY ? -INFINITY : (x - M) * a.scale - ln_s; };
    if (g.out.entropy && threadIdx.x == 0) g.out.entropy[row] = bad ? __uint_as_float(0x7fc00000u) : none ? 0.f : ln_s - W * a.scale / S;
    if (g.out.logprobs && threadIdx.x < a.given) {
        const int32_t t = a.tokens[(size_t)row * a.given + threadIdx.x];
        float x = -INFINITY;
        for (uint32_t i = 0; i < n_rec; ++i) x = fmaxf(x, record(i)[4 + threadIdx.x]);
        g.out.logprobs[(size_t)row * a.given + threadIdx.x] = t < 0 ? 0.f : (uint32_t)t >= a.vocab ? __uint_as_float(0x7fc00000u) : answer(x);
    }
    if (!g.out.top_ids || a.top == 0) return;
    const uint32_t n_all = bad ? 0 : n_rec * a.top;
    auto entry = [&](uint32_t i, uint2 &v) {
        const float *r = record(i / a.top) + 4 + a.given + i % a.top;
        v = make_uint2(order_of(r[0]), __float_as_uint(r[a.top]));
    };
    // the lanes' largest, then all that reach the top-th of them: ids differ, so that an (order, id) is held by one
    uint2 v, best = make_uint2(0, 0);
    for (uint32_t i = threadIdx.x; i < n_all; i += kLogprobThreads) {
        entry(i, v);
        if (v.x > best.x || (v.x == best.x && v.y < best.y)) best = v;
    }
    uint32_t bound = kth_largest(best.x, a.top, lanes), last = ~0u;
    if (bound <= kOrderNone) bound = kOrderNone + 1;
    for (int pass = 0;; ++pass) {
        if (threadIdx.x == 0) count = 0;
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < n_all; i += kLogprobThreads) {
            entry(i, v);
            if (v.x > bound || (v.x == bound && v.y <= last)) {
                const uint32_t at = atomicAdd(&count, 1u);
                if (at < kList) list[at] = v;
            }
        }
        __syncthreads();
        if (count <= kList || pass) break;
        const uint32_t key = best.x > bound ? ~0u : best.x == bound ? ~best.y : 0u;
        __syncthreads();
        last = ~kth_largest(key, a.top, lanes);
    }
    write_ranked(list, min(count, kList), a.top, values, ids);
    __syncthreads();
    if (threadIdx.x < a.top) {
        g.out.top_ids[(size_t)row * a.top + threadIdx.x] = ids[threadIdx.x];
        g.out.top_logprobs[(size_t)row * a.top + threadIdx.x] = bad ? __uint_as_float(0x7fc00000u) : answer(values[threadIdx.x]);
    }
}

hipError_t launch_logprobs_join(const psv_logprobs_args &a, const float *records, uint32_t shards, const psv_logprobs_out &out, hipStream_t s)
{
    const JoinArgs g{a, records, shards, out};
    PSV_LAUNCH(k_logprobs_join, dim3(a.rows), dim3(kLogprobThreads), 0, s, g);
    return hipGetLastError();
}

}  // namespace psv
