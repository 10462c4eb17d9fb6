// Log probabilities of given tokens, entropy and the most likely tokens (psv_logprobs_part, psv_logprobs_join).
//
// With M the largest logit of a row, d = x - M (exact, or one rounding) and e = exp(s d):  ln p = s d - ln(sum e), entropy = ln(sum e) -
// s (sum e d) / (sum e).  A workgroup reduces a piece of a row, its record, to (M, sum e, sum e d), the given tokens' logits and its largest
// `top`; records are joined by rescaling their sums to the common M.  All sums are 32 bits.  No term e d is positive, so that nothing cancels but the
// common rounding of the exponents, at most a quarter of a unit (below).
//
// A piece is read once, into registers, all loads at once, and everything else -- the maximum, the sums, the alternatives -- is made from
// there.  Large calls in 32 bits are bound by memory (1024 rows of 128256, 525 MB: 92 us, 5.7 TB/s), in 16 bits by instructions, 11.3 a column of
// which the exponential takes the time of four (2048 rows, the same bytes: 102 us, the vector units busy 89 % of it; both for 8 alternatives, without the
// join, in a stream of calls).  Small ones are bound by
// the chain load -> bound -> candidates -> ranks, 5 us, and the same in the join.
//
// Alternatives without sorting: the top-th largest of the lanes' maxima is a bound T that at least `top` logits reach, and of every lane
// but `top` none exceeds it; so at most top * (columns a lane) logits exceed T, usually about `top`.  Those that reach it are collected in LDS and
// each one's rank counted.  Where more equal ones reach T than the list holds, the same bound on the ids of those equal to T
// cuts them to top * (columns a lane) in all, which the list holds.
#include "rows.h"

namespace psv {

constexpr int kThreads = kLogprobThreads, kWaves = kThreads / 64;
constexpr uint32_t kJoinList = PSV_LOGPROBS_MAX_TOP * 64;

// Order of floats as unsigned integers (-0 counts as 0, every NaN is above infinity)
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t b = __float_as_uint(x + 0.f);
    return x != x ? ~0u : b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_order(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o); }
constexpr uint32_t kOrderNone = 0x007fffffu, kOrderInf = 0xff800000u;      // of -infinity and infinity
constexpr float kLowest = -3.402823466e38f;

__device__ __forceinline__ float nan32() { return __uint_as_float(0x7fc00000u); }

// The k-th largest of the workgroup's values (k <= threads), or a lower one that at most `enough` of them reach: bit by bit, from the first
// in which the largest and the smallest differ down to bit LOW (below it an order has zeros, or ones where the value is negative).  A wave has
// all of them, one of each wave a lane, and counts for itself.  Bound by the way from the comparisons to the scalar unit and back, some
// 0.06 us a bit, so that it stops early; two bits a step took as long.
template <int LOW, int W>
__device__ __forceinline__ uint32_t kth_largest(const uint32_t (&w)[W], uint32_t k, uint32_t enough)
{
    uint32_t most = w[0], least = ~w[0];
#pragma unroll
    for (int i = 1; i < W; ++i) {
        most = max(most, w[i]);
        least = max(least, ~w[i]);
    }
    most = wave_max_u32(most);
    least = ~wave_max_u32(least);
    if (k == 1 || most == least) return most;
    uint32_t bit = 0x80000000u >> __builtin_clz(most ^ least), t = least & ~(2 * bit - 1);
    for (; bit >= 1u << LOW; bit >>= 1) {
        uint32_t n = 0;
#pragma unroll
        for (int i = 0; i < W; ++i) n += __popcll(__ballot(w[i] >= (t | bit)));
        if (n >= k) {
            t |= bit;
            if (n <= enough) break;
        }
    }
    return t & 0x80000000u ? t : t | ((1u << LOW) - 1);
}
// How many lanes may reach the bound: as many as the list has room for, but not so many that ranking them takes longer than the bits would.
__host__ __device__ constexpr uint32_t enough_lanes(uint32_t k, uint32_t more, uint32_t room) { return k + more < room ? k + more : room; }

// Places for a lane's `n` entries in the list.  The address looks like the lane's own, or the compiler would make one addition of the wave's, by a
// loop over its lanes: longer than what the additions take in LDS.
__device__ __forceinline__ uint32_t list_places(uint32_t *count, uint32_t n)
{
    uint32_t own = 0;
    asm volatile("" : "+v"(own));
    return atomicAdd(count + own, n);
}

// Ranks of the n listed among themselves, an entry a lane; put(rank, entry) for the first `top`.  The others come to a wave by lane reads: an entry
// read from LDS instead costs its latency (joining 61 rows of 160 entries for 20 of them: 5.6 us against 7.5).
template <int THREADS, class Put>
__device__ __forceinline__ void rank_list(const uint64_t *list, uint32_t n, uint32_t top, Put put)
{
    const uint32_t lane = threadIdx.x & 63;
    for (uint32_t i = threadIdx.x - lane; i < n; i += THREADS) {
        const uint64_t me = list[min(i + lane, n - 1)];
        uint32_t rank = 0;
        for (uint32_t j0 = 0; j0 < n; j0 += 64) {
            const uint64_t o = list[min(j0 + lane, n - 1)];
            const uint32_t m = min(n - j0, 64u);
            for (uint32_t j = 0; j < m; ++j) {
                const uint64_t other = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(o >> 32), (int)j) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)o, (int)j);
                rank += other > me;
            }
        }
        if (i + lane < n && rank < top) put(rank, me);
    }
}
// An entry: the order of a logit, and its id so that the lower one counts as the larger.
__device__ __forceinline__ uint64_t list_entry(uint32_t order, uint32_t id) { return (uint64_t)order << 32 | (uint32_t)~id; }
__device__ __forceinline__ float entry_value(uint64_t v) { return of_order((uint32_t)(v >> 32)); }
__device__ __forceinline__ uint32_t entry_id(uint64_t v) { return ~(uint32_t)v; }

// What a workgroup shares: the lanes' largest, then the waves' sums, and the candidates.
template <int THREADS, uint32_t LIST>
struct Shared {
    uint32_t lanes[THREADS];
    float2 sums[THREADS / 64];
    uint32_t count;
    uint64_t list[LIST];
};

struct PartArgs {
    psv_logprobs_args a;
    float *records;
    uint32_t chunk;
    float to_log2;          // scale * log2(e)
};

// A record: M, sum e, sum e d, unused; the given tokens' logits (-infinity: not in this piece); the largest logits; their ids.
__host__ __device__ inline uint32_t record_floats(uint32_t given, uint32_t top) { return 4 + given + 2 * top; }

// A lane's E columns as they were read, 16-bit ones two to a register.
template <uint32_t DT, int E>
struct Held {
    static constexpr bool kHalves = DT != PSV_F32;
    uint32_t w[kHalves ? E / 2 : E];
    __device__ float get(int e) const
    {
        if constexpr (!kHalves) return __uint_as_float(w[e]);
        else if constexpr (DT == PSV_BF16) return e & 1 ? bf16_hi(w[e / 2]) : bf16_lo(w[e / 2]);
        else return (float)__builtin_bit_cast(_Float16, (uint16_t)(e & 1 ? w[e / 2] >> 16 : w[e / 2]));
    }
    // Column e, known only when it runs, of one group.  The empty asm keeps the selections in registers: without it the
    // compiler may make the words an array in scratch.
    __device__ float pick(uint32_t e) const
    {
        constexpr int W = kHalves ? E / 2 : E;
        static_assert(E == 8, "one group");   // four or eight words: a chain of selections is short
        const uint32_t k = kHalves ? e >> 1 : e;
        uint32_t v = w[0];
        asm volatile("" : "+v"(v));
#pragma unroll
        for (uint32_t j = 1; j < (uint32_t)W; ++j) {
            v = k == j ? w[j] : v;
            asm volatile("" : "+v"(v));
        }
        if constexpr (!kHalves) return __uint_as_float(v);
        v = e & 1 ? v >> 16 : v & 0xffffu;
        if constexpr (DT == PSV_BF16) return __uint_as_float(v << 16);
        else return (float)__builtin_bit_cast(_Float16, (uint16_t)v);
    }
    // Columns 8 i to 8 i + 7
    __device__ Held<DT, 8> group(uint32_t i) const
    {
        constexpr int GW = kHalves ? 4 : 8;
        Held<DT, 8> h;
#pragma unroll
        for (int j = 0; j < GW; ++j) {
            h.w[j] = w[j];
#pragma unroll
            for (int k = 1; k < E / 8; ++k) h.w[j] = i == (uint32_t)k ? w[k * GW + j] : h.w[j];
        }
        return h;
    }
    // Conversions are made again after this, not carried over in as many registers.
    __device__ void forget()
    {
#pragma unroll
        for (uint32_t &v : w) asm volatile("" : "+v"(v));
    }
};

template <uint32_t DT, int E>
__global__ __launch_bounds__(kLogprobThreads, DT == PSV_F32 ? (E == 128 ? 2 : E == 64 ? 4 : 6) : (E == 128 ? 4 : E == 64 ? 6 : 8)) void k_logprobs_part(PartArgs g)
{
    using T = typename Elem<DT>::T;
    constexpr int N = Elem<DT>::N, G = 8;
    constexpr uint32_t kList = PSV_LOGPROBS_MAX_TOP * E;
    struct __attribute__((packed, aligned(sizeof(T)))) Loose { uint32_t w[4]; };      // rows of any alignment
    __shared__ Shared<kThreads, kList> sh;
    const psv_logprobs_args &a = g.a;
    const uint32_t row = blockIdx.x / a.records, rec = blockIdx.x % a.records;
    const uint32_t c0 = min(rec * g.chunk, a.columns), c1 = min(c0 + g.chunk, a.columns);
    const T *px = static_cast<const T *>(a.logits) + (int64_t)row * a.row;
    float *out = g.records + (size_t)blockIdx.x * record_floats(a.given, a.top);
    // the lane's vector j of the piece; masked past its end
    auto fetch = [&](uint32_t j, uint32_t (&w)[4]) {
        const uint32_t c = c0 + (j * kLogprobThreads + threadIdx.x) * N;
        if (c + N <= c1) {
            const Loose p = *reinterpret_cast<const Loose *>(px + c);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = p.w[i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (DT == PSV_F32) {
                    w[i] = c + i < c1 ? __float_as_uint(px[c + i]) : 0xff800000u;
                } else {
                    const uint16_t *ph = reinterpret_cast<const uint16_t *>(px);
                    const uint32_t none = DT == PSV_BF16 ? 0xff80u : 0xfc00u;
                    const uint32_t lo = c + 2 * i < c1 ? ph[c + 2 * i] : none, hi = c + 2 * i + 1 < c1 ? ph[c + 2 * i + 1] : none;
                    w[i] = lo | hi << 16;
                }
            }
        }
    };
    Held<DT, E> x;
#pragma unroll
    for (int j = 0; j < E / N; ++j) {
        uint32_t w[4];
        fetch(j, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) x.w[j * 4 + i] = w[i];
    }
    if (threadIdx.x < a.given) {
        const int64_t t = (int64_t)a.tokens[(size_t)row * a.given + threadIdx.x] - a.first_token;
        out[4 + threadIdx.x] = t >= c0 && t < c1 ? Elem<DT>::get(px[t]) : -INFINITY;
    }
    // the largest of every group of eight columns, of the lane, and -- with the bound of the alternatives -- of the workgroup
    float most[E / G], mine = -INFINITY;
#pragma unroll
    for (int i = 0; i < E / G; ++i) {
        float m = x.get(i * G);
#pragma unroll
        for (int e = 1; e < G; ++e) m = __builtin_elementwise_maximum(m, x.get(i * G + e));
        most[i] = m;
        mine = __builtin_elementwise_maximum(mine, m);
    }
    sh.lanes[threadIdx.x] = order_of(mine);
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    uint32_t w4[kWaves], top_order = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        w4[i] = sh.lanes[i * 64 + (threadIdx.x & 63)];
        top_order = max(top_order, w4[i]);
    }
    top_order = wave_max_u32(top_order);
    const bool bad = top_order >= kOrderInf;          // a NaN or +infinity
    const float M = of_order(top_order), ref = top_order == kOrderNone ? 0.f : M;
    // In units of log 2, t = x c - M c as one multiply-add: M c is rounded, which moves every t by the same `shift`, known exactly and taken out of
    // the sums at their end.  (With the difference first a column costs an instruction more: this kernel, 2048 rows of 128256 in bf16 108.8 us
    // against 100.6.)
    // Below 2^23 the rounding is at most 1/4, which scales the sums by 2^(1/4) at most and costs the second a quarter of the first's error.  From there
    // on -- a large scale, or a piece of nothing but far values -- it would leave the exponential's range: the difference first, of columns read again.
    const float c = g.to_log2;
    const bool near = fabsf(ref * c) < 0x1p23f;
    const float Mc = near ? ref * c : 0.f, shift = near ? fmaf(ref, c, -Mc) : 0.f;
    float s = 0.f, w = 0.f;
    auto add = [&](float t) {
        t = fmaxf(t, kLowest);          // a masked logit: p = 0 and a finite t
        const float p = exp2_raw(t);
        s += p;
        w = fmaf(p, t, w);
    };
    x.forget();
    if (near) {
#pragma unroll
        for (int e = 0; e < E; ++e) add(fmaf(x.get(e), c, -Mc));
    } else {
#pragma unroll 1
        for (int j = 0; j < E / N; ++j) {
            Held<DT, N> h;
            fetch(j, h.w);
#pragma unroll
            for (int e = 0; e < N; ++e) add((h.get(e) - ref) * c);
        }
    }
    s = wave_sum(s);
    w = wave_sum(w);
    if ((threadIdx.x & 63) == 0) sh.sums[threadIdx.x >> 6] = make_float2(s, w);
    float *values = out + 4 + a.given;
    int32_t *ids = reinterpret_cast<int32_t *>(values + a.top);
    uint32_t n = 0;
    if (a.top == 0 || bad) {
        __syncthreads();
    } else {
        const float least = of_order(max(kth_largest<DT == PSV_F32 ? 0 : DT == PSV_BF16 ? 16 : 13>(w4, a.top, enough_lanes(a.top, a.top / 2, kList / E)), kOrderNone + 1));
        uint32_t last = ~0u;                        // highest id taken of those equal to `least`
        uint32_t groups = 0;                        // the few that reach it are looked through one by one
#pragma unroll
        for (int i = 0; i < E / G; ++i) groups |= most[i] >= least ? 1u << i : 0u;
        auto id_of = [&](uint32_t i, uint32_t e) { return c0 + threadIdx.x * N + i * (G * kThreads) + e / N * (kThreads * N) + e % N; };
        // Taken from the registers, a group costs a selection a word and group: large pieces, which are bound by their instructions, read it
        // again instead (this kernel, 2048 rows of 32000 in bf16, 20 alternatives: 38.0 us against 40.2); small ones would wait for the trip.
        auto group = [&](uint32_t i) {
            if constexpr (E < 64) {
                return x.group(i);
            } else {
                Held<DT, G> h;
#pragma unroll
                for (int j = 0; j < G / N; ++j) {
                    uint32_t w[4];
                    fetch(i * (G / N) + j, w);
#pragma unroll
                    for (int k = 0; k < 4; ++k) h.w[j * 4 + k] = w[k];
                }
                return h;
            }
        };
        if (E < 64) x.forget();
        for (int pass = 0;; ++pass) {
            for (uint32_t left = groups; left; left &= left - 1) {
                const uint32_t i = __builtin_ctz(left);
                const Held<DT, G> h = group(i);
                uint32_t hits = 0;
#pragma unroll
                for (int e = G - 1; e >= 0; --e) hits = 2 * hits + (h.get(e) >= least);
                if (pass)
#pragma unroll
                    for (int e = 0; e < G; ++e)
                        if (h.get(e) == least && id_of(i, e) > last) hits &= ~(1u << e);
                uint32_t at = list_places(&sh.count, (uint32_t)__popc(hits));
                // A step a hit, mostly one, not a test a column (for 20, this kernel, 61 rows of 32003: 7.0 us against 7.4; with the join, 2048 of 128256: 114 against 117)
                for (; hits && at < kList; hits &= hits - 1) {
                    const uint32_t e = __builtin_ctz(hits);
                    sh.list[at++] = list_entry(order_of(h.pick(e)), id_of(i, e));
                }
            }
            __syncthreads();
            n = sh.count;
            if (n <= kList) break;
            if (pass) { n = kList; break; }         // not reached: no read behind the list all the same
            // too many equal ones: those lanes that exceed the bound count first, then the lanes by their first id
            uint32_t key = 0;
            if (mine > least) {
                key = ~0u;
            } else if (groups) {
                const uint32_t i = __builtin_ctz(groups);
                const Held<DT, G> h = group(i);
#pragma unroll
                for (int e = G - 1; e >= 0; --e)
                    if (h.get(e) == least) key = ~id_of(i, e);
            }
            sh.lanes[threadIdx.x] = key;
            __syncthreads();
            if (threadIdx.x == 0) sh.count = 0;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) w4[i] = sh.lanes[i * 64 + (threadIdx.x & 63)];
            last = ~kth_largest<0>(w4, a.top, a.top);
            __syncthreads();
        }
        rank_list<kThreads>(sh.list, n, a.top, [&](uint32_t rank, uint64_t v) {
            values[rank] = entry_value(v);
            ids[rank] = (int32_t)(entry_id(v) + a.first_token);
        });
    }
    for (uint32_t i = n + threadIdx.x; i < a.top; i += kLogprobThreads) {
        values[i] = -INFINITY;
        ids[i] = -1;
    }
    if (threadIdx.x == 0) {
        const float2 a0 = sh.sums[0], a1 = sh.sums[1], a2 = sh.sums[2], a3 = sh.sums[3];
        const float S = (a0.x + a1.x) + (a2.x + a3.x), D = (a0.y + a1.y) + (a2.y + a3.y), back = exp2_raw(-shift);
        out[0] = M;
        out[1] = bad ? nan32() : S * back;
        out[2] = fmaf(-shift, S, D) * back / c;         // of d = t / c
        out[3] = 0.f;
    }
}

template <uint32_t DT>
static void launch_part_as(const PartArgs &g, hipStream_t s)
{
    const dim3 grid(g.a.rows * g.a.records), block(kLogprobThreads);
    if (g.chunk <= kLogprobThreads * 8) PSV_LAUNCH((k_logprobs_part<DT, 8>), grid, block, 0, s, g);
    else if (g.chunk <= kLogprobThreads * 16) PSV_LAUNCH((k_logprobs_part<DT, 16>), grid, block, 0, s, g);
    else if (g.chunk <= kLogprobThreads * 32) PSV_LAUNCH((k_logprobs_part<DT, 32>), grid, block, 0, s, g);
    else if (g.chunk <= kLogprobThreads * 64) PSV_LAUNCH((k_logprobs_part<DT, 64>), grid, block, 0, s, g);
    else PSV_LAUNCH((k_logprobs_part<DT, 128>), grid, block, 0, s, g);
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
    uint32_t by_top, by_records;      // divisions as products: i / top = i * by_top >> 21 for i < 256 top, k / records = k * by_records >> 16 for k < 256
};

// One workgroup a row.  64 threads, where a row has no more records than those and at most kHeld alternatives a lane: a
// wave needs no barriers, and a compute unit has room for as many rows as it has wave slots.  (8 records of 8 alternatives, 2048
// rows: 6.4 us, with 256 threads 13.4.)
constexpr uint32_t kHeld = 8;
template <int THREADS>
__global__ __launch_bounds__(THREADS) void k_logprobs_join(JoinArgs g)
{
    constexpr int W = THREADS / 64;
    constexpr uint32_t LIST = THREADS == 64 ? PSV_LOGPROBS_MAX_TOP * kHeld : kJoinList;
    __shared__ Shared<THREADS, LIST> sh;
    __shared__ float given_s[PSV_LOGPROBS_MAX_GIVEN];
    __shared__ uint32_t most_s[W];
    const psv_logprobs_args &a = g.a;
    const uint32_t row = blockIdx.x, size = record_floats(a.given, a.top), n_rec = g.shards * a.records;
    auto record = [&](uint32_t k) {
        const uint32_t shard = k * g.by_records >> 16;
        return g.records + ((size_t)(shard * (a.rows - 1) + row) * a.records + k) * size;      // ((shard * rows + row) * records + k - shard * records)
    };
    float m = -INFINITY, s = 0.f, w = 0.f, x0 = -INFINITY;
    if (threadIdx.x < n_rec) {
        const float *r = record(threadIdx.x);
        m = r[0];
        s = r[1];
        w = r[2];
        if (a.given) x0 = r[4];
    }
    // The alternatives of all records; a wave keeps its lanes' in registers.  Ids differ, so that an (order, id) is held by one lane.
    const uint32_t n_all = g.out.top_ids ? n_rec * a.top : 0;
    auto entry = [&](uint32_t i) {
        const uint32_t k = i * g.by_top >> 21;
        const float *r = record(k) + 4 + a.given + (i - k * a.top);
        return make_uint2(THREADS == 64 ? __float_as_uint(r[0]) : order_of(r[0]), __float_as_uint(r[a.top]));
    };
    uint2 held[kHeld];
    if constexpr (THREADS == 64)
#pragma unroll
        for (int j = 0; j < kHeld; ++j) {          // all requested at once; their orders are made when they have arrived
            held[j] = make_uint2(0, 0);
            if (j * THREADS < n_all) held[j] = entry(min(j * THREADS + threadIdx.x, n_all - 1));
        }
    uint2 best = make_uint2(0, 0);
    auto look = [&](uint2 v) {
        if (v.x > best.x || (v.x == best.x && v.y < best.y)) best = v;
    };
    if constexpr (THREADS == 64) {
        if (n_all)
#pragma unroll
        for (int j = 0; j < kHeld; ++j) {
            held[j].x = j * THREADS + threadIdx.x < n_all ? order_of(__uint_as_float(held[j].x)) : 0;
            look(held[j]);
        }
    } else {
        for (uint32_t i = threadIdx.x; i < n_all; i += THREADS) look(entry(i));
    }
    static_assert(PSV_LOGPROBS_MAX_GIVEN <= THREADS && PSV_LOGPROBS_MAX_TOP <= THREADS, "one lane each");
    if (threadIdx.x < PSV_LOGPROBS_MAX_GIVEN) given_s[threadIdx.x] = -INFINITY;
    if (threadIdx.x == 0) sh.count = 0;
    sh.lanes[threadIdx.x] = best.x;
    const uint32_t most = wave_max_u32(s != s ? ~0u : order_of(m));
    if ((threadIdx.x & 63) == 0) most_s[threadIdx.x >> 6] = most;
    __syncthreads();
    uint32_t top_order = most_s[0];
#pragma unroll
    for (int i = 1; i < W; ++i) top_order = max(top_order, most_s[i]);
    const bool bad = top_order >= kOrderInf;
    const float M = of_order(top_order);
    // a given token's logit lies in one record
    if (x0 > -INFINITY) given_s[0] = x0;
    if (threadIdx.x < n_rec)
        for (uint32_t k = 1; k < a.given; ++k) {
            const float x = record(threadIdx.x)[4 + k];
            if (x > -INFINITY) given_s[k] = x;
        }
    if (m > -INFINITY) {
        const float d = m - M, f = exp2_raw(d * a.scale * 1.4426950408889634f);
        w = f * (w + (f > 0.f ? s * d : 0.f));
        s *= f;
    }
    s = wave_sum(s);
    w = wave_sum(w);
    if ((threadIdx.x & 63) == 0) sh.sums[threadIdx.x >> 6] = make_float2(s, w);
    uint32_t n = 0;
    if (n_all == 0 || bad) {
        __syncthreads();
    } else {
        uint32_t w4[W], last = ~0u;
#pragma unroll
        for (int i = 0; i < W; ++i) w4[i] = sh.lanes[i * 64 + (threadIdx.x & 63)];
        const uint32_t bound = max(kth_largest<0>(w4, a.top, enough_lanes(a.top, a.top / 4, LIST / (THREADS == 64 ? kHeld : 32))), kOrderNone + 1);
        for (int pass = 0;; ++pass) {
            auto reaches = [&](uint2 v) { return v.x > bound || (v.x == bound && v.y <= last); };
            if constexpr (THREADS == 64) {          // the wave's places by counting: nothing to wait for
                n = 0;
#pragma unroll
                for (int j = 0; j < kHeld; ++j) {
                    const bool hit = reaches(held[j]);
                    const uint64_t hits = __ballot(hit);
                    const uint32_t at = __builtin_amdgcn_mbcnt_hi((uint32_t)(hits >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)hits, n));
                    if (hit && at < LIST) sh.list[at] = list_entry(held[j].x, held[j].y);
                    n += __popcll(hits);
                }
                __syncthreads();
            } else {
                for (uint32_t i = threadIdx.x; i < n_all; i += THREADS) {
                    const uint2 v = entry(i);
                    if (!reaches(v)) continue;
                    const uint32_t at = list_places(&sh.count, 1);
                    if (at < LIST) sh.list[at] = list_entry(v.x, v.y);
                }
                __syncthreads();
                n = sh.count;
            }
            if (n <= LIST) break;
            if (pass) { n = LIST; break; }
            sh.lanes[threadIdx.x] = best.x > bound ? ~0u : best.x == bound ? ~best.y : 0u;
            __syncthreads();
            if (threadIdx.x == 0) sh.count = 0;
#pragma unroll
            for (int i = 0; i < W; ++i) w4[i] = sh.lanes[i * 64 + (threadIdx.x & 63)];
            last = ~kth_largest<0>(w4, a.top, a.top);
            __syncthreads();
        }
    }
    float S = 0.f, D = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        S += sh.sums[i].x;
        D += sh.sums[i].y;
    }
    const float ln_s = logf(S);
    const bool none = top_order == kOrderNone;
    // by halves, whose difference is the exact half where that of the logits passes what 32 bits hold
    auto answer = [&](float x) { return bad ? nan32() : none || x == -INFINITY ? -INFINITY : (0.5f * x - 0.5f * M) * (2.f * a.scale) - ln_s; };
    if (g.out.entropy && threadIdx.x == 0) g.out.entropy[row] = bad ? nan32() : none ? 0.f : ln_s - D * a.scale / S;
    if (g.out.logprobs && threadIdx.x < a.given) {
        const int32_t t = a.tokens[(size_t)row * a.given + threadIdx.x];
        g.out.logprobs[(size_t)row * a.given + threadIdx.x] = t < 0 ? 0.f : (uint32_t)t >= a.vocab ? nan32() : answer(given_s[threadIdx.x]);
    }
    if (!g.out.top_ids) return;
    int32_t *ids = g.out.top_ids + (size_t)row * a.top;
    float *values = g.out.top_logprobs + (size_t)row * a.top;
    rank_list<THREADS>(sh.list, n, a.top, [&](uint32_t rank, uint64_t v) {
        ids[rank] = (int32_t)entry_id(v);
        values[rank] = answer(entry_value(v));
    });
    for (uint32_t i = n + threadIdx.x; i < a.top; i += THREADS) {
        ids[i] = -1;
        values[i] = bad ? nan32() : -INFINITY;
    }
}

hipError_t launch_logprobs_join(const psv_logprobs_args &a, const float *records, uint32_t shards, const psv_logprobs_out &out, hipStream_t s)
{
    const JoinArgs g{a, records, shards, out, a.top ? ((1u << 21) + a.top - 1) / a.top : 0, (65536 + a.records - 1) / a.records};
    const uint32_t n = shards * a.records;
    if (n <= 64 && n * a.top <= 64 * kHeld) PSV_LAUNCH(k_logprobs_join<64>, dim3(a.rows), dim3(64), 0, s, g);
    else PSV_LAUNCH(k_logprobs_join<kThreads>, dim3(a.rows), dim3(kThreads), 0, s, g);
    return hipGetLastError();
}

}  // namespace psv
