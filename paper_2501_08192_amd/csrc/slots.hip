// Block tables and slot maps from the lengths of requests (psv_cache_slots).
//
// Two prefix sums over the requests (rows and blocks), which also say who is refused, then 16 bytes a row.  The sums are a few
// thousand additions: every workgroup makes them for itself, so that one launch does all and no workgroup waits for another; its
// rows are then spread over the lanes, four neighbours each, their request found by bisection of the row starts in LDS.  Bound by the launch
// and the chain lengths -> sums -> row starts -> block -> slot: 64 requests of one token 3.4 us, 509 of 400 tokens (3.3 MB)
// 7.0.
//
// Why both sums can be made at once, though a request whose rows do not fit takes no blocks: the rows before it only grow, so that one
// that fits has none before it that does not.
#include "rows.h"

namespace psv {

constexpr int kSlotsThreads = 256;

__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

// Inclusive prefix sum over a wave, held at 2^32 - 1 (associative, as nothing is negative).
__device__ __forceinline__ uint32_t wave_scan(uint32_t v)
{
    v = add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, true));     // row_shr:1, 2, 4, 8
    v = add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, true));
    v = add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, true));
    v = add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, true));
    const uint32_t r0 = (uint32_t)__builtin_amdgcn_readlane((int)v, 15), r1 = (uint32_t)__builtin_amdgcn_readlane((int)v, 31),
                   r2 = (uint32_t)__builtin_amdgcn_readlane((int)v, 47);
    const int row = (threadIdx.x & 63) >> 4;
    const uint32_t before = row > 2 ? add_sat(add_sat(r0, r1), r2) : row > 1 ? add_sat(r0, r1) : row > 0 ? r0 : 0;
    return add_sat(v, before);
}

// PER: requests of a lane, requested at once.  ROWS: rows of a lane and step.
template <int PER, int ROWS>
__global__ __launch_bounds__(kSlotsThreads) void k_cache_slots(psv_slots_args a)
{
    // first_s: place in the free list of the request's first new block, -1: refused
    __shared__ int32_t start_s[PER * kSlotsThreads], len_s[PER * kSlotsThreads], first_s[PER * kSlotsThreads], new_s[PER * kSlotsThreads];
    __shared__ uint32_t wave_s[2][kSlotsThreads / 64];
    const uint32_t b0 = threadIdx.x * PER;
    int64_t lens[PER], news[PER];
    // read and written in the order of memory, worked on in the order of requests: through LDS
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const uint32_t b = i * kSlotsThreads + threadIdx.x;
        len_s[b] = b < a.batch ? a.lens[b] : 0;
        new_s[b] = b < a.batch ? a.new_lens[b] : 0;
    }
    if (PER > 1) __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        lens[i] = len_s[b0 + i];
        news[i] = new_s[b0 + i];
    }
    const int64_t most = (int64_t)a.max_blocks * 16;
    const bool table = a.block_table != nullptr;
    int32_t head = 0, free_n = 0;
    if (table) {
        const int32_t lo = a.free_range[0], hi = a.free_range[1];
        if (lo >= 0 && hi > lo && (uint32_t)hi <= a.free_capacity) {
            head = lo;
            free_n = hi - lo;
        }
    }
    auto need_of = [&](int64_t len, int64_t n) -> uint32_t {      // 0 where the lengths are out of range
        return len >= 0 && n >= 0 && len + n <= most ? (uint32_t)((len + n + 15) / 16 - (len + 15) / 16) : 0;
    };
    uint32_t rows = 0, blocks = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        rows = add_sat(rows, (uint32_t)max(news[i], (int64_t)0));
        blocks = add_sat(blocks, need_of(lens[i], news[i]));
    }
    const uint32_t rows_to = wave_scan(rows), blocks_to = wave_scan(blocks);
    if ((threadIdx.x & 63) == 63) {
        wave_s[0][threadIdx.x >> 6] = rows_to;
        wave_s[1][threadIdx.x >> 6] = blocks_to;
    }
    __syncthreads();
    uint32_t row = __shfl_up(rows_to, 1, 64), taken = __shfl_up(blocks_to, 1, 64), total_rows = 0;      // not by subtraction: a held sum has lost what it was
    if ((threadIdx.x & 63) == 0) row = taken = 0;
    uint32_t rows_before = 0, blocks_before = 0;
#pragma unroll
    for (int w = 0; w < kSlotsThreads / 64; ++w) {
        if (w < (int)(threadIdx.x >> 6)) {
            rows_before = add_sat(rows_before, wave_s[0][w]);
            blocks_before = add_sat(blocks_before, wave_s[1][w]);
        }
        total_rows = add_sat(total_rows, wave_s[0][w]);
    }
    uint32_t refused = 0, used = 0;
    row = add_sat(row, rows_before);
    taken = add_sat(taken, blocks_before);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const uint32_t b = b0 + i;
        if (b >= a.batch) break;
        const int64_t len = lens[i], n = news[i];
        const uint32_t need = need_of(len, n);
        bool good = len >= 0 && n >= 0 && len + n <= most && (int64_t)row + n <= (int64_t)a.rows;
        const uint32_t before = taken;
        taken = add_sat(taken, need);
        if (table && need && taken > (uint32_t)free_n) good = false;
        start_s[b] = (int32_t)min(row, a.rows);
        first_s[b] = !good ? -1 : table && need ? head + (int32_t)before : 0;
        refused += !good;
        if (good && need) used = taken;                           // those that are not refused come first: the last one's end is their sum
        row = add_sat(row, (uint32_t)max(n, (int64_t)0));
    }
    const int32_t end = (int32_t)min(total_rows, a.rows);
    __shared__ uint32_t refused_s[kSlotsThreads / 64], used_s[kSlotsThreads / 64];
    if (blockIdx.x == 0) {
        refused = (uint32_t)wave_sum((float)refused);             // exact: at most 16 a lane
        used = wave_max_u32(used);
        if ((threadIdx.x & 63) == 0) {
            refused_s[threadIdx.x >> 6] = refused;
            used_s[threadIdx.x >> 6] = used;
        }
    }
    __syncthreads();
    if (blockIdx.x == 0)
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const uint32_t b = i * kSlotsThreads + threadIdx.x;
            if (b >= a.batch) break;
            a.row_starts[b] = start_s[b];
            a.seq_lens[b] = first_s[b] < 0 ? len_s[b] : len_s[b] + new_s[b];
        }
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        a.row_starts[a.batch] = end;
        *a.refused = (int32_t)(refused_s[0] + refused_s[1] + refused_s[2] + refused_s[3]);
        if (table) {
            a.free_range_out[0] = a.free_range[0] + (int32_t)max(max(used_s[0], used_s[1]), max(used_s[2], used_s[3]));
            a.free_range_out[1] = a.free_range[1];
        }
    }
    struct __attribute__((packed, aligned(8))) Slots { int64_t v[ROWS]; };
    struct __attribute__((packed, aligned(4))) Words { int32_t v[ROWS]; };
    for (uint64_t r0 = ((uint64_t)blockIdx.x * kSlotsThreads + threadIdx.x) * ROWS; r0 < a.rows; r0 += (uint64_t)gridDim.x * kSlotsThreads * ROWS) {
        uint32_t lo = 0;
        if ((int64_t)r0 < end) {
            uint32_t hi = a.batch;                  // the last request that starts at or before r0: one without rows shares its start with the next
            while (hi - lo > 1) {
                const uint32_t mid = (lo + hi) / 2;
                if (start_s[mid] <= (int32_t)r0) lo = mid;
                else hi = mid;
            }
        }
        Slots slots;
        Words positions, requests;
        const int32_t *where[ROWS];
        int32_t *entry[ROWS];
        int64_t at[ROWS];
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {      // where each row's block id stands
            const int64_t r = (int64_t)r0 + i;
            where[i] = nullptr;
            entry[i] = nullptr;
            slots.v[i] = -1;
            positions.v[i] = 0;
            requests.v[i] = -1;
            at[i] = 0;
            if (r >= end) continue;
            while (lo + 1 < a.batch && start_s[lo + 1] <= r) ++lo;
            const int64_t p = (int64_t)len_s[lo] + (r - start_s[lo]);
            positions.v[i] = (int32_t)p;
            requests.v[i] = (int32_t)lo;
            at[i] = p;
            if (first_s[lo] < 0) continue;
            const int32_t blk = (int32_t)(p >> 4), held = (len_s[lo] + 15) >> 4;
            if (!table) {
                const uint64_t id = (uint64_t)lo * a.max_blocks + blk;
                if (id < a.num_pool_blocks) slots.v[i] = (int64_t)(id << 4) | (p & 15);
            } else if (blk < held) {
                where[i] = a.block_table + (size_t)lo * a.max_blocks + blk;
            } else {
                where[i] = a.free_blocks + first_s[lo] + (blk - held);
                if ((p & 15) == 0) entry[i] = a.block_table + (size_t)lo * a.max_blocks + blk;
            }
        }
        int32_t id[ROWS];
#pragma unroll
        for (int i = 0; i < ROWS; ++i) id[i] = where[i] ? *where[i] : -1;
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            if (entry[i]) *entry[i] = id[i];
            if (id[i] >= 0 && (uint32_t)id[i] < a.num_pool_blocks) slots.v[i] = (int64_t)id[i] * 16 + (at[i] & 15);
        }
        if (r0 + ROWS <= a.rows) {
            *reinterpret_cast<Slots *>(a.slots + r0) = slots;
            *reinterpret_cast<Words *>(a.positions + r0) = positions;
            *reinterpret_cast<Words *>(a.requests + r0) = requests;
        } else {
#pragma unroll
            for (int i = 0; i < ROWS; ++i)
                if (r0 + i < a.rows) {
                    a.slots[r0 + i] = slots.v[i];
                    a.positions[r0 + i] = positions.v[i];
                    a.requests[r0 + i] = requests.v[i];
                }
        }
    }
}

template <int PER>
static void launch_slots_as(const psv_slots_args &a, hipStream_t s)
{
    // Four rows a lane share a bisection and leave in wide stores; one row a lane where those are fewer workgroups than compute units.
    const int rows = a.rows >= kSlotsThreads * 256 ? 4 : 1;
    uint64_t blocks = ((uint64_t)a.rows + kSlotsThreads * rows - 1) / (kSlotsThreads * rows);
    if (blocks < 1) blocks = 1;
    if (blocks > 256) blocks = 256;
    if (rows == 4) PSV_LAUNCH((k_cache_slots<PER, 4>), dim3((unsigned)blocks), dim3(kSlotsThreads), 0, s, a);
    else PSV_LAUNCH((k_cache_slots<PER, 1>), dim3((unsigned)blocks), dim3(kSlotsThreads), 0, s, a);
}

hipError_t launch_cache_slots(const psv_slots_args &a, hipStream_t s)
{
    if (a.batch <= kSlotsThreads) launch_slots_as<1>(a, s);
    else if (a.batch <= 4 * kSlotsThreads) launch_slots_as<4>(a, s);
    else launch_slots_as<PSV_SLOTS_MAX_BATCH / kSlotsThreads>(a, s);
    return hipGetLastError();
}

}  // namespace psv
