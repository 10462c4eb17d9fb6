// Block tables and slot maps from the lengths of requests (psv_cache_slots).
//
// Three prefix sums over the requests (rows, blocks, and with them who is refused), then 16 bytes a row.  The sums are a few
// thousand additions: every workgroup makes them for itself, so that one launch does all and no workgroup waits for another;
// its rows are then spread over the lanes, a row's request found by bisection of the row starts in LDS.
#include "rows.h"

namespace psv {

constexpr int kSlotsThreads = 256;

// Exclusive prefix sum over the workgroup's threads and the total; `tmp` is free to use again after the call.
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t *tmp, int64_t &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t s = v;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int64_t t = __shfl_up(s, off, 64);
        if (lane >= off) s += t;
    }
    if (lane == 63) tmp[wave] = s;
    __syncthreads();
    int64_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kSlotsThreads / 64; ++w) {
        if (w < wave) before += tmp[w];
        total += tmp[w];
    }
    __syncthreads();
    return before + s - v;
}

__global__ __launch_bounds__(kSlotsThreads) void k_cache_slots(psv_slots_args a)
{
    __shared__ int32_t start_s[PSV_SLOTS_MAX_BATCH], len_s[PSV_SLOTS_MAX_BATCH], first_s[PSV_SLOTS_MAX_BATCH];      // first_s: place in the free list of the request's first new block, -1 refused
    __shared__ int64_t tmp[kSlotsThreads / 64];
    const uint32_t per = (a.batch + kSlotsThreads - 1) / kSlotsThreads, b0 = threadIdx.x * per;
    const int64_t most = (int64_t)a.max_blocks * 16;
    const bool table = a.block_table != nullptr;
    int64_t head = 0, free_n = 0;
    if (table) {
        const int32_t lo = a.free_range[0], hi = a.free_range[1];
        if (lo >= 0 && hi > lo && (uint32_t)hi <= a.free_capacity) { head = lo; free_n = hi - lo; }
    }
    // rows
    int64_t rows = 0, total_rows = 0;
    for (uint32_t i = 0; i < per; ++i)
        if (b0 + i < a.batch) rows += max(a.new_lens[b0 + i], 0);
    int64_t row = block_scan(rows, tmp, total_rows);
    // blocks: what the requests that are not refused for their lengths need
    auto length = [&](uint32_t b, int64_t at, int64_t &len, int64_t &n, int64_t &need) {
        len = a.lens[b];
        n = a.new_lens[b];
        const bool good = len >= 0 && n >= 0 && len + n <= most && at + n <= (int64_t)a.rows;
        need = good ? (len + n + 15) / 16 - (len + 15) / 16 : 0;
        return good;
    };
    int64_t blocks = 0, total_blocks = 0, at = row, len, n, need;
    for (uint32_t i = 0; i < per && b0 + i < a.batch; ++i) {
        (void)length(b0 + i, at, len, n, need);
        at += max(n, (int64_t)0);
        blocks += need;
    }
    int64_t taken = block_scan(blocks, tmp, total_blocks);
    int64_t refused = 0, used = 0, total_refused = 0, total_used = 0;
    for (uint32_t i = 0; i < per && b0 + i < a.batch; ++i) {
        const uint32_t b = b0 + i;
        bool good = length(b, row, len, n, need);
        taken += need;
        if (table && need && taken > free_n) good = false;
        start_s[b] = (int32_t)min(row, (int64_t)a.rows);
        len_s[b] = (int32_t)len;
        first_s[b] = good ? (int32_t)(table ? head + taken - need : 0) : -1;
        if (good) used += need;
        else ++refused;
        if (blockIdx.x == 0) {
            a.row_starts[b] = start_s[b];
            a.seq_lens[b] = (int32_t)(good ? len + n : len);
        }
        row += max(n, (int64_t)0);
    }
    (void)block_scan(refused, tmp, total_refused);
    (void)block_scan(used, tmp, total_used);
    const int32_t end = (int32_t)min(total_rows, (int64_t)a.rows);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        a.row_starts[a.batch] = end;
        *a.refused = (int32_t)total_refused;
        if (table) {
            a.free_range_out[0] = (int32_t)(free_n ? head + total_used : a.free_range[0]);
            a.free_range_out[1] = a.free_range[1];
        }
    }
    __syncthreads();
    for (uint64_t r64 = (uint64_t)blockIdx.x * kSlotsThreads + threadIdx.x; r64 < a.rows; r64 += (uint64_t)gridDim.x * kSlotsThreads) {
        const int32_t r = (int32_t)r64;
        int64_t slot = -1;
        int32_t pos = 0, req = -1;
        if (r < end) {
            uint32_t lo = 0, hi = a.batch;              // the last request that starts at or before r: one without rows shares its start with the next
            while (hi - lo > 1) {
                const uint32_t mid = (lo + hi) / 2;
                if (start_s[mid] <= r) lo = mid;
                else hi = mid;
            }
            req = (int32_t)lo;
            const int64_t p = (int64_t)len_s[lo] + (r - start_s[lo]);
            pos = (int32_t)p;
            if (first_s[lo] >= 0) {
                const int32_t blk = (int32_t)(p >> 4), held = (len_s[lo] + 15) >> 4;
                int32_t id = (int32_t)((int64_t)lo * a.max_blocks + blk);
                if (table) {
                    int32_t *entry = a.block_table + (size_t)lo * a.max_blocks + blk;
                    if (blk < held) {
                        id = *entry;
                    } else {
                        id = a.free_blocks[first_s[lo] + blk - held];
                        if ((p & 15) == 0) *entry = id;
                    }
                }
                if (id >= 0 && (uint32_t)id < a.num_pool_blocks) slot = (int64_t)id * 16 + (p & 15);
            }
        }
        a.slots[r] = slot;
        a.positions[r] = pos;
        a.requests[r] = req;
    }
}

hipError_t launch_cache_slots(const psv_slots_args &a, hipStream_t s)
{
    uint32_t blocks = (a.rows + kSlotsThreads * 4 - 1) / (kSlotsThreads * 4);
    if (blocks < 1) blocks = 1;
    if (blocks > 256) blocks = 256;
    PSV_LAUNCH(k_cache_slots, dim3(blocks), dim3(kSlotsThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace psv
