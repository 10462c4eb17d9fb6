// C entry points of include/preserve_ops.h: frequencies, argument checks and launches.
#include <math.h>
#include <string.h>

#include "context.h"
#include "operators.h"

using namespace psv;

namespace {

constexpr double kPi = 3.14159265358979323846;
constexpr uint32_t kMostRows = 1u << 24, kMostHeads = 1u << 28;      // rows, and kv heads of all rows, of a call: what the launches divide into one grid

size_t elem_size(uint32_t dtype) { return dtype == PSV_F32 ? 4 : 2; }
bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// A launch goes to the current device: a stream of another one is refused.
psv_status check_stream(void *stream)
{
    if (reinterpret_cast<uintptr_t>(stream) <= 2) return PSV_OK;      // the default streams are the current device's
    int now = 0;
    hipDevice_t dev = 0;
    if (hipGetDevice(&now) != hipSuccess || hipStreamGetDevice(static_cast<hipStream_t>(stream), &dev) != hipSuccess) return PSV_ERR_HIP;
    return now == dev ? PSV_OK : PSV_ERR_INVALID_ARG;
}

psv_status launched(hipError_t e) { return e == hipSuccess ? PSV_OK : PSV_ERR_HIP; }

bool rope_ok(const psv_rope &r)
{
    if (r.dims < 2 || r.dims > PSV_ROPE_MAX_DIMS || r.dims % 2 || r.pairing > PSV_ROPE_INTERLEAVED || !isfinite(r.magnitude)) return false;
    for (uint32_t i = 0; i < r.dims / 2; ++i)
        if (!isfinite(r.freq[i])) return false;
    return true;
}

bool cache_ok(const psv_cache &c)
{
    if (!c.k_pool || !c.v_pool || !aligned(c.k_pool, 16) || !aligned(c.v_pool, 16)) return false;
    if (c.n_kv_heads == 0 || c.n_kv_heads > 128 || c.num_pool_blocks == 0 || c.num_pool_blocks > 0x7fffffffu) return false;
    return c.kv_format <= PSV_FMT_INT8 && c.kv_layout <= PSV_KV_TOKEN_MAJOR && !(c.kv_layout == PSV_KV_TOKEN_MAJOR && c.kv_format != PSV_FMT_BF16);
}

// Rows of `heads` heads of 128, every one of them on 16 bytes; written rows may not overlap.
bool rows_ok(const void *p, int64_t row, uint32_t heads, uint32_t dtype, uint32_t rows, bool written)
{
    if (!p || !aligned(p, 16) || row < 0 || (uint64_t)row * elem_size(dtype) % 16 || row > (1ll << 40)) return false;
    return !written || rows <= 1 || row >= (int64_t)heads * PSV_HEAD_DIM;
}

bool logprobs_ok(const psv_logprobs_args *a)
{
    if (!a || a->rows > (1u << 20) || a->given > PSV_LOGPROBS_MAX_GIVEN || a->top > PSV_LOGPROBS_MAX_TOP) return false;
    if (!(a->scale > 0.f) || a->scale < 0x1p-32f || a->scale > 0x1p32f || a->vocab == 0 || a->vocab > (1u << 21)) return false;
    return a->given == 0 || a->rows == 0 || (a->tokens && aligned(a->tokens, 4));
}

// psv_logprobs_part's arguments, with the number of records filled in.
psv_status part_args(const psv_logprobs_args *a, const void *records, psv_logprobs_args *out)
{
    if (!logprobs_ok(a) || a->dtype > PSV_F16 || a->columns == 0 || a->columns > (1u << 21)) return PSV_ERR_INVALID_ARG;
    if (a->first_token > a->vocab || a->columns > a->vocab - a->first_token) return PSV_ERR_INVALID_ARG;
    *out = *a;
    if (a->records == 0) out->records = psv_logprobs_records(a->rows, a->columns);
    if (out->records > PSV_LOGPROBS_MAX_RECORDS || logprob_chunk(a->columns, out->records) > kLogprobMostColumns) return PSV_ERR_INVALID_ARG;
    if ((uint64_t)a->rows * out->records > (1u << 23)) return PSV_ERR_UNSUPPORTED;
    if (a->rows == 0) return PSV_OK;
    if (!a->logits || !aligned(a->logits, elem_size(a->dtype)) || a->row < 0 || a->row > (1ll << 32) || !records || !aligned(records, 4)) return PSV_ERR_INVALID_ARG;
    return PSV_OK;
}

bool join_ok(const psv_logprobs_args *a, const void *records, uint32_t shards, const psv_logprobs_out *out)
{
    if (!logprobs_ok(a) || !out || a->records == 0 || shards == 0 || (uint64_t)shards * a->records > PSV_LOGPROBS_MAX_RECORDS) return false;
    if ((out->top_ids == nullptr) != (out->top_logprobs == nullptr)) return false;
    const void *words[] = {out->logprobs, out->entropy, out->top_logprobs, out->top_ids};
    for (const void *p : words)
        if (!aligned(p, 4)) return false;
    return a->rows == 0 || (records && aligned(records, 4));
}

}  // namespace

extern "C" {

psv_status psv_rope_plan(const psv_rope_desc *d, psv_rope *out)
{
    if (!d || !out) return PSV_ERR_INVALID_ARG;
    if (d->dims < 2 || d->dims > PSV_ROPE_MAX_DIMS || d->dims % 2 || d->pairing > PSV_ROPE_INTERLEAVED || d->scaling > PSV_ROPE_BY_CHANNEL) return PSV_ERR_INVALID_ARG;
    if (!(d->theta > 1.0) || !isfinite(d->theta) || !isfinite(d->magnitude)) return PSV_ERR_INVALID_ARG;
    const bool scaled = d->scaling != PSV_ROPE_PLAIN, ramp = d->scaling >= PSV_ROPE_BY_TURNS;
    if (scaled && (!(d->factor >= 1.0) || !isfinite(d->factor))) return PSV_ERR_INVALID_ARG;
    if (ramp && (!(d->low_turns > 0.0) || !(d->high_turns > d->low_turns) || !isfinite(d->high_turns) || !(d->trained_context >= 1.0) || !isfinite(d->trained_context)))
        return PSV_ERR_INVALID_ARG;
    memset(out, 0, sizeof *out);
    out->dims = d->dims;
    out->pairing = d->pairing;
    out->magnitude = d->magnitude == 0.0 ? 1.0 : d->magnitude;
    // the pair that makes n turns in the trained context: trained_context * theta^(-2i / dims) = 2 pi n
    auto pair_of = [&](double n) { return d->dims * log(d->trained_context / (2.0 * kPi * n)) / (2.0 * log(d->theta)); };
    double from = 0.0, to = 0.0;
    if (d->scaling == PSV_ROPE_BY_CHANNEL) {
        from = fmax(floor(pair_of(d->high_turns)), 0.0);
        to = fmin(ceil(pair_of(d->low_turns)), d->dims - 1.0);
    }
    for (uint32_t i = 0; i < d->dims / 2; ++i) {
        const double f = pow(d->theta, -2.0 * (double)i / d->dims);
        double w = 1.0;
        if (d->scaling == PSV_ROPE_LINEAR) w = 0.0;
        else if (d->scaling == PSV_ROPE_BY_TURNS) w = (d->trained_context * f / (2.0 * kPi) - d->low_turns) / (d->high_turns - d->low_turns);
        else if (d->scaling == PSV_ROPE_BY_CHANNEL) w = 1.0 - ((double)i - from) / fmax(to - from, 0.001);
        w = fmin(fmax(w, 0.0), 1.0);
        out->freq[i] = scaled ? w * f + (1.0 - w) * f / d->factor : f;
    }
    return PSV_OK;
}

psv_status psv_set_rope(psv_ctx *c, const psv_rope *rope)
{
    if (!c) return PSV_ERR_INVALID_ARG;
    if (rope) {
        if (!rope_ok(*rope)) return PSV_ERR_INVALID_ARG;
        if (rope->dims != PSV_HEAD_DIM || rope->pairing != PSV_ROPE_HALF) return PSV_ERR_UNSUPPORTED;
    }
    StepRope r = step_rope(c->d.rope_theta);
    if (rope) {
        memcpy(r.freq, rope->freq, sizeof r.freq);
        r.magnitude = rope->magnitude;
    }
    ST_TRY(check_stream(c->main));
    return launched(launch_store_rope(r, c->at<StepRope>(c->ws.rope_freq), c->main));
}

psv_status psv_rotate(const psv_rotate_args *a, const psv_rope *rope, void *stream)
{
    if (!a || !rope || !rope_ok(*rope)) return PSV_ERR_INVALID_ARG;
    if (a->rows > kMostRows || a->heads == 0 || a->heads > 65535 || a->head_dim < rope->dims || a->head_dim > 1024) return PSV_ERR_INVALID_ARG;
    if (a->dtype > PSV_F16 || a->transpose > 1) return PSV_ERR_INVALID_ARG;
    if (a->rows == 0) return PSV_OK;
    const size_t size = elem_size(a->dtype);
    if (!a->x || !a->y || !a->positions || !aligned(a->x, size) || !aligned(a->y, size) || !aligned(a->positions, 4)) return PSV_ERR_INVALID_ARG;
    const int64_t strides[4] = {a->x_row, a->x_head, a->y_row, a->y_head};
    for (int64_t v : strides)
        if (v < 0 || v > (1ll << 32)) return PSV_ERR_INVALID_ARG;
    // every element of y has a place of its own: heads within rows, or rows within heads
    const int64_t rows = a->rows, heads = a->heads, dim = a->head_dim;
    const bool by_row = (heads == 1 || a->y_head >= dim) && (rows == 1 || a->y_row >= (heads - 1) * a->y_head + dim);
    const bool by_head = (rows == 1 || a->y_row >= dim) && (heads == 1 || a->y_head >= (rows - 1) * a->y_row + dim);
    if (!by_row && !by_head) return PSV_ERR_INVALID_ARG;
    if (a->x == a->y && ((rows > 1 && a->x_row != a->y_row) || (heads > 1 && a->x_head != a->y_head))) return PSV_ERR_INVALID_ARG;
    // 16 bytes a lane, where every piece of a head starts on 16 bytes and every pair lies in one piece or in two alike
    const int64_t n = 16 / size;
    bool vectors = aligned(a->x, 16) && aligned(a->y, 16) && dim % n == 0 && rope->dims % (rope->pairing == PSV_ROPE_HALF ? 2 * n : n) == 0;
    for (int64_t v : strides) vectors = vectors && v % n == 0;
    ST_TRY(check_stream(stream));
    return launched(launch_rotate(*a, *rope, vectors, static_cast<hipStream_t>(stream)));
}

psv_status psv_cache_slots(const psv_slots_args *a, void *stream)
{
    if (!a || a->batch == 0 || a->batch > PSV_SLOTS_MAX_BATCH || a->max_blocks == 0 || (uint64_t)a->batch * a->max_blocks > 0x7fffffffull) return PSV_ERR_INVALID_ARG;
    if (a->max_blocks > 0x7ffffffu || a->num_pool_blocks == 0 || a->num_pool_blocks > 0x7fffffffu || a->rows > 0x7fffffffu) return PSV_ERR_INVALID_ARG;
    if (!a->lens || !a->new_lens || !a->seq_lens || !a->row_starts || !a->refused) return PSV_ERR_INVALID_ARG;
    if (a->rows && (!a->slots || !a->positions || !a->requests)) return PSV_ERR_INVALID_ARG;
    if (a->block_table && ((!a->free_blocks && a->free_capacity) || !a->free_range || !a->free_range_out || a->free_capacity > 0x7fffffffu)) return PSV_ERR_INVALID_ARG;
    const void *words[] = {a->lens, a->new_lens, a->seq_lens, a->row_starts, a->refused, a->positions, a->requests, a->block_table, a->free_blocks, a->free_range, a->free_range_out};
    for (const void *p : words)
        if (!aligned(p, 4)) return PSV_ERR_INVALID_ARG;
    if (!aligned(a->slots, 8)) return PSV_ERR_INVALID_ARG;
    // the workgroups of a call read the lengths and the free range while one of them writes the new ones
    if (a->seq_lens == a->lens || a->seq_lens == a->new_lens || (a->block_table && a->free_range_out == a->free_range)) return PSV_ERR_INVALID_ARG;
    ST_TRY(check_stream(stream));
    return launched(launch_cache_slots(*a, static_cast<hipStream_t>(stream)));
}

psv_status psv_cache_append(const psv_append_args *a, const psv_cache *cache, const psv_rope *rope, void *stream)
{
    if (!a || !cache || !cache_ok(*cache) || (rope && !rope_ok(*rope))) return PSV_ERR_INVALID_ARG;
    if (a->rows > kMostRows || a->n_q_heads > 128 || a->dtype > PSV_F16) return PSV_ERR_INVALID_ARG;
    if (rope && (rope->dims > PSV_HEAD_DIM || rope->dims % 16)) return PSV_ERR_UNSUPPORTED;
    if ((uint64_t)a->rows * cache->n_kv_heads > kMostHeads) return PSV_ERR_UNSUPPORTED;
    if (a->rows == 0) return PSV_OK;
    if (!a->slots || !aligned(a->slots, 8) || (rope && !a->positions) || !aligned(a->positions, 4)) return PSV_ERR_INVALID_ARG;
    if (!rows_ok(a->k, a->k_row, cache->n_kv_heads, a->dtype, a->rows, false) || !rows_ok(a->v, a->v_row, cache->n_kv_heads, a->dtype, a->rows, false)) return PSV_ERR_INVALID_ARG;
    if (a->n_q_heads && (!rows_ok(a->q, a->q_row, a->n_q_heads, a->dtype, a->rows, false) || !rows_ok(a->q_out, a->q_out_row, a->n_q_heads, a->dtype, a->rows, true) ||
                         (a->q == a->q_out && a->q_row != a->q_out_row && a->rows > 1)))
        return PSV_ERR_INVALID_ARG;
    ST_TRY(check_stream(stream));
    return launched(launch_cache_append(*a, *cache, rope, static_cast<hipStream_t>(stream)));
}

psv_status psv_cache_gather(const psv_gather_args *a, const psv_cache *cache, void *stream)
{
    if (!a || !cache || !cache_ok(*cache) || a->rows > kMostRows || a->dtype > PSV_F16) return PSV_ERR_INVALID_ARG;
    if ((uint64_t)a->rows * cache->n_kv_heads > kMostHeads) return PSV_ERR_UNSUPPORTED;
    if (a->rows == 0) return PSV_OK;
    if (!a->slots || !aligned(a->slots, 8)) return PSV_ERR_INVALID_ARG;
    if (!rows_ok(a->k, a->k_row, cache->n_kv_heads, a->dtype, a->rows, true) || !rows_ok(a->v, a->v_row, cache->n_kv_heads, a->dtype, a->rows, true)) return PSV_ERR_INVALID_ARG;
    ST_TRY(check_stream(stream));
    return launched(launch_cache_gather(*a, *cache, static_cast<hipStream_t>(stream)));
}

uint32_t psv_logprobs_records(uint32_t rows, uint32_t columns)
{
    if (rows > (1u << 20) || columns == 0 || columns > (1u << 21)) return 0;
    // The largest pieces, which cost least a column, that still give every compute unit one; below 4096 columns the records cost
    // more than the pieces gain.  (Both kernels of calls in a stream for 8 alternatives, pieces of 16384 / 8192 / 4096 / 2048: of 128256 columns in bf16
    // 256 rows 26.4 / 28.8 / 37.5 / 58.8 us, 64 rows 14.6 / 15.0 / 17.5 / 23.2, 8 rows 10.6 / 10.2 / 10.5 / 11.2; 61 rows of 32003 in f16 11.6 / 11.0 / 11.2 /
    // 12.3.)
    uint32_t most = kLogprobThreads * 64;
    while (most > 4096 && (uint64_t)rows * ((columns + most - 1) / most) < 256 && (columns + most / 2 - 1) / (most / 2) <= PSV_LOGPROBS_MAX_RECORDS) most /= 2;
    return (columns + most - 1) / most;
}

size_t psv_logprobs_bytes(uint32_t rows, uint32_t records, uint32_t given, uint32_t top)
{
    return (size_t)4 * rows * records * (4 + given + 2 * top);
}

psv_status psv_logprobs_part(const psv_logprobs_args *a, void *records, void *stream)
{
    psv_logprobs_args b;
    ST_TRY(part_args(a, records, &b));
    if (b.rows == 0) return PSV_OK;
    ST_TRY(check_stream(stream));
    return launched(launch_logprobs_part(b, static_cast<float *>(records), static_cast<hipStream_t>(stream)));
}

psv_status psv_logprobs_join(const psv_logprobs_args *a, const void *records, uint32_t shards, const psv_logprobs_out *out, void *stream)
{
    if (!join_ok(a, records, shards, out)) return PSV_ERR_INVALID_ARG;
    if (a->rows == 0) return PSV_OK;
    ST_TRY(check_stream(stream));
    return launched(launch_logprobs_join(*a, static_cast<const float *>(records), shards, *out, static_cast<hipStream_t>(stream)));
}

psv_status psv_logprobs(const psv_logprobs_args *a, const psv_logprobs_out *out, void *workspace, size_t workspace_bytes, void *stream)
{
    psv_logprobs_args b;
    ST_TRY(part_args(a, workspace, &b));
    // Pieces of twice the size, where there are thousands, two columns fit a register and alternatives are wanted: half as many records to join and to
    // choose from, against half as many waves at once.  (Both kernels of calls in a stream.  Rows in which a dozen logits stand out, 8 alternatives: 2048
    // rows of 128256 in bf16 109 us against 113, 512 rows 39.1 against 38.0, 2048 rows of 32000 40.1 against 40.6, 4096 in f16 62.3 against 65.1; more
    // padding costs: 2048 rows of 200000 177 against 172.  Rows without, 4 / 8 / 20 / 32 alternatives: 2048 rows of 128256 108.9 / 110.4 / 114.9 / 125.8
    // against 109.0 / 109.4 / 117.4 / 134.4, 512 rows 40.8 / 41.2 / 42.1 / 48.7 against 38.4 / 38.4 / 41.9 / 53.3.)  These are fewer records than the
    // workspace has room for.
    const uint32_t fewer = (b.columns + kLogprobMostColumns - 1) / kLogprobMostColumns;
    if (a->records == 0 && b.dtype != PSV_F32 && b.top >= 8 && fewer < b.records && (uint64_t)b.rows * fewer >= 2048) b.records = fewer;
    if (b.first_token != 0 || b.columns != b.vocab || workspace_bytes < psv_logprobs_bytes(b.rows, b.records, b.given, b.top)) return PSV_ERR_INVALID_ARG;
    if (!join_ok(&b, workspace, 1, out)) return PSV_ERR_INVALID_ARG;
    if (b.rows == 0) return PSV_OK;
    ST_TRY(check_stream(stream));
    ST_TRY(launched(launch_logprobs_part(b, static_cast<float *>(workspace), static_cast<hipStream_t>(stream))));
    return launched(launch_logprobs_join(b, static_cast<const float *>(workspace), 1, *out, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
