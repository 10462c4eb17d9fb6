// Rotary positions of rows (psv_rotate): every channel pair (a, b) of the first n channels of a head becomes
// (a c - b s, b c + a s), c and s the cosine and sine of position times frequency.
//
// Bound by memory: a row is read and written once, 16 bytes a lane (16384 rows of 16 heads in 32 bits, 268 MB: 50.4 us, 5.3 TB/s).  The angles
// are formed and reduced in 64 bits, once for each row and pair, by the workgroup that has the row, and lie in LDS for all of its heads; rows of
// one head pay for them (65536 rows of one head in 16 bits, 34 MB: 18.3 us).
#include "rows.h"

namespace psv {

struct RotateArgs {
    psv_rotate_args a;
    psv_rope rope;
    uint32_t tile;          // rows of a workgroup
    uint32_t items, pairs;  // pieces of a head, one a lane and step: `pairs` of rotated channels, then the others
    uint32_t slots;         // heads that the workgroup has in hand at once
};

constexpr int kRotateThreads = 256, kRotateAngles = 1024, kRotateAhead = 2;

__device__ __forceinline__ void make_angles(const RotateArgs &g, uint32_t row0, uint32_t n_rows, float2 *cs)
{
    const uint32_t n = g.rope.dims / 2;
    const double m = g.rope.magnitude;
    for (uint32_t i = threadIdx.x; i < n_rows * n; i += kRotateThreads) {
        const uint32_t r = i / n, p = i % n;
        float2 v = turn((double)g.a.positions[row0 + r] * g.rope.freq[p], m);
        if (g.a.transpose) v.y = -v.y;
        cs[i] = v;
    }
}

// Heads in pieces of 16 bytes.  A lane requests its pieces of kRotateAhead heads at once, the first ones before the angles are made
// (two ahead against four: 28.0 / 32.3 us for 16384 rows of 16 heads in 16 bits; the registers of four halve the waves).
template <uint32_t DT, bool HALF>
__global__ __launch_bounds__(kRotateThreads) void k_rotate(RotateArgs g)
{
    using T = typename Elem<DT>::T;
    constexpr int N = Elem<DT>::N, U = kRotateAhead;
    __shared__ float2 cs[kRotateAngles];
    const psv_rotate_args &a = g.a;
    const uint32_t row0 = blockIdx.x * g.tile, n_rows = min(g.tile, a.rows - row0), n = g.rope.dims / 2;
    const uint32_t slot = threadIdx.x / g.items, j = threadIdx.x % g.items;
    const bool turned = j < g.pairs;
    // channels of the lane's piece, and of its partner
    const uint32_t lo = turned ? j * N : 2 * n + (j - g.pairs) * N, hi = n + j * N;
    const T *x = static_cast<const T *>(a.x) + (int64_t)row0 * a.x_row;
    T *y = static_cast<T *>(a.y) + (int64_t)row0 * a.y_row;
    uint32_t r = slot / a.heads, h = slot % a.heads;
    if (slot >= g.slots) r = n_rows;                    // no piece of its own
    const uint32_t step_r = g.slots / a.heads, step_h = g.slots % a.heads;
    for (bool first = true;; first = false) {
        Pack<DT, N> pu[U], pv[U];
        uint32_t at_r[U], at_h[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            at_r[k] = r;
            at_h[k] = h;
            if (r < n_rows) {
                const T *p = x + (int64_t)r * a.x_row + (int64_t)h * a.x_head;
                pu[k] = fetch_row<DT, N>(p + lo);
                if (HALF && turned) pv[k] = fetch_row<DT, N>(p + hi);
                r += step_r;
                h += step_h;
                if (h >= a.heads) {
                    h -= a.heads;
                    ++r;
                }
            }
        }
        if (first) {
            make_angles(g, row0, n_rows, cs);
            __syncthreads();
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (at_r[k] >= n_rows) break;
            T *p = y + (int64_t)at_r[k] * a.y_row + (int64_t)at_h[k] * a.y_head;
            const float2 *c = cs + at_r[k] * n;
            float u[N], v[N];
            unpack_row<DT, N>(pu[k], u);
            if (HALF && turned) {
                unpack_row<DT, N>(pv[k], v);
#pragma unroll
                for (int e = 0; e < N; ++e) turn_pair(u[e], v[e], c[lo + e]);
                store_row<DT, N>(p + hi, v);
            } else if (turned) {
#pragma unroll
                for (int e = 0; e < N; e += 2) turn_pair(u[e], u[e + 1], c[(lo + e) / 2]);
            }
            store_row<DT, N>(p + lo, u);
        }
        if (r >= n_rows) return;
    }
}

// Rows of any alignment and heads of any size: one pair, or one channel, a lane and step.  Bound by its instructions and small accesses: 16384 rows of
// 16 heads one element off 16 bytes 64.4 us in 32 bits and 46.8 in 16 (2.9 TB/s); in 16 bits 40 of 80 channels rotated in halves 41.5 (2.0 TB/s; in neighbours,
// by the kernel above, 16.3), 24 of 96 60.5 (1.7).
template <uint32_t DT, bool HALF>
__global__ __launch_bounds__(kRotateThreads) void k_rotate_any(RotateArgs g)
{
    using T = typename Elem<DT>::T;
    __shared__ float2 cs[kRotateAngles];
    const psv_rotate_args &a = g.a;
    const uint32_t row0 = blockIdx.x * g.tile, n_rows = min(g.tile, a.rows - row0), n = g.rope.dims / 2;
    make_angles(g, row0, n_rows, cs);
    __syncthreads();
    const uint32_t slot = threadIdx.x / g.items;
    if (slot >= g.slots) return;
    for (uint32_t s = slot; s < n_rows * a.heads; s += g.slots) {
        const uint32_t r = s / a.heads, h = s % a.heads;
        const T *px = static_cast<const T *>(a.x) + (int64_t)(row0 + r) * a.x_row + (int64_t)h * a.x_head;
        T *py = static_cast<T *>(a.y) + (int64_t)(row0 + r) * a.y_row + (int64_t)h * a.y_head;
        for (uint32_t j = threadIdx.x % g.items; j < g.items; j += kRotateThreads) {      // more than one step only where a head has more pieces than the workgroup lanes
            if (j >= g.pairs) {
                py[2 * n + j - g.pairs] = px[2 * n + j - g.pairs];
            } else {
                const uint32_t lo = HALF ? j : 2 * j, hi = HALF ? n + j : 2 * j + 1;
                float u = Elem<DT>::get(px[lo]), v = Elem<DT>::get(px[hi]);
                turn_pair(u, v, cs[r * n + j]);
                py[lo] = Elem<DT>::put(u);
                py[hi] = Elem<DT>::put(v);
            }
        }
    }
}

template <uint32_t DT>
static void launch_rotate_as(RotateArgs &g, bool vectors, hipStream_t s)
{
    constexpr int N = Elem<DT>::N;
    const uint32_t dims = g.rope.dims, rest = g.a.head_dim - dims;
    const bool half = g.rope.pairing == PSV_ROPE_HALF;
    g.pairs = vectors ? (half ? dims / 2 / N : dims / N) : dims / 2;
    g.items = g.pairs + (vectors ? rest / N : rest);
    g.slots = g.items < (uint32_t)kRotateThreads ? kRotateThreads / g.items : 1;
    // Four heads a lane, and fewer rows until there are two workgroups a compute unit: more heads share angles but leave a longer last round
    // (2 / 4 / 8 heads a lane: 16384 rows of 16 heads in 32 bits 48.6 / 49.9 / 54.8 us, in 16 bits 29.1 / 28.3 / 30.2; 6001 rows of 16 heads
    // of which half is rotated 11.4 / 10.6 / 10.1; 4096 rows of 64 heads 29.9 / 27.7 / 30.1).
    const uint32_t most = kRotateAngles / (dims / 2), want = 4 * g.slots / g.a.heads;
    g.tile = want < 1 ? 1 : want < most ? want : most;
    while (g.tile > 1 && g.a.rows / g.tile < 512) g.tile /= 2;
    while ((g.a.rows + g.tile - 1) / g.tile > kMostGroups) g.tile *= 2;      // 2^24 rows, one a workgroup: two (at least eight have room for their angles)
    const dim3 grid((g.a.rows + g.tile - 1) / g.tile), block(kRotateThreads);
    if (half && vectors) PSV_LAUNCH((k_rotate<DT, true>), grid, block, 0, s, g);
    else if (half) PSV_LAUNCH((k_rotate_any<DT, true>), grid, block, 0, s, g);
    else if (vectors) PSV_LAUNCH((k_rotate<DT, false>), grid, block, 0, s, g);
    else PSV_LAUNCH((k_rotate_any<DT, false>), grid, block, 0, s, g);
}

hipError_t launch_rotate(const psv_rotate_args &a, const psv_rope &rope, bool vectors, hipStream_t s)
{
    RotateArgs g{};
    g.a = a;
    g.rope = rope;
    if (a.dtype == PSV_F32) launch_rotate_as<PSV_F32>(g, vectors, s);
    else if (a.dtype == PSV_BF16) launch_rotate_as<PSV_BF16>(g, vectors, s);
    else launch_rotate_as<PSV_F16>(g, vectors, s);
    return hipGetLastError();
}

}  // namespace psv
