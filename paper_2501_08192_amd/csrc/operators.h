// Internal interface between the entry points of include/preserve_ops.h (operators.cpp) and their kernels (rotary.hip,
// cache_rows.hip, slots.hip, logprobs.hip).  Launch wrappers validate nothing and return the hipError_t of the launch.
#pragma once

#include "internal.h"
#include "../../include/preserve_ops.h"

namespace psv {

// A grid has fewer than 2^32 threads in a direction: workgroups of 256 in one launch.
constexpr uint32_t kMostGroups = (1u << 24) - 1;

hipError_t launch_rotate(const psv_rotate_args &a, const psv_rope &rope, bool vectors, hipStream_t s);
hipError_t launch_cache_slots(const psv_slots_args &a, hipStream_t s);
hipError_t launch_cache_append(const psv_append_args &a, const psv_cache &cache, const psv_rope *rope, hipStream_t s);
hipError_t launch_cache_gather(const psv_gather_args &a, const psv_cache &cache, hipStream_t s);

// Columns that one workgroup of the log probabilities holds in registers: kLogprobThreads times 8, 16, 32, 64 or 128.
constexpr uint32_t kLogprobThreads = 256, kLogprobMostColumns = kLogprobThreads * 128;
// Columns of a record; a record may be empty.
inline uint32_t logprob_chunk(uint32_t columns, uint32_t records) { return ((columns + records - 1) / records + 7) / 8 * 8; }
hipError_t launch_logprobs_part(const psv_logprobs_args &a, float *records, hipStream_t s);
hipError_t launch_logprobs_join(const psv_logprobs_args &a, const float *records, uint32_t shards, const psv_logprobs_out &out, hipStream_t s);

}  // namespace psv
