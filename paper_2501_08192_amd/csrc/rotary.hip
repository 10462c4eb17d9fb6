// Rotary positions of rows (psv_rotate): every channel pair (a, b) of the first n channels of a head becomes
// (a c - b s, b c + a s), c and s the cosine and sine of position times frequency.
//
// Bound by memory: a row is read and written once, 16 bytes a lane.  The angles are formed and reduced in 64 bits, once for each row and
// pair, by the workgroup that has the row, and lie in LDS for all of its heads.
#include "rows.h"

namespace psv {

struct RotateArgs {
    psv_rotate_args a;
    psv_rope rope;
    uint32_t tile;          // rows of a workgroup
    uint32_t items, pairs;  // pieces of a head, one a lane and step: `pairs` of rotated channels, then the others
    uint32_t slots;         // heads that the workgroup has in hand at once
};

constexpr int kRotateThreads = 256, kRotateTileRows = 8;

// N: channels in a load (1: rows of any alignment and heads of any size).
template <uint32_t DT, bool HALF, int N>
__global__ __launch_bounds__(kRotateThreads) void k_rotate(RotateArgs g)
{
    using T = typename Elem<DT>::T;
    __shared__ float2 cs[kRotateTileRows * PSV_ROPE_MAX_DIMS / 2];
    const psv_rotate_args &a = g.a;
    const uint32_t row0 = blockIdx.x * g.tile, n_rows = min(g.tile, a.rows - row0), n = g.rope.dims / 2;
    const double m = g.rope.magnitude;
    for (uint32_t i = threadIdx.x; i < n_rows * n; i += kRotateThreads) {
        const uint32_t r = i / n, p = i % n;
        float2 v = turn((double)a.positions[row0 + r] * g.rope.freq[p], m);
        if (a.transpose) v.y = -v.y;
        cs[i] = v;
    }
    __syncthreads();
    const uint32_t slot = threadIdx.x / g.items;
    if (slot >= g.slots) return;
    const T *x = static_cast<const T *>(a.x);
    T *y = static_cast<T *>(a.y);
    for (uint32_t s = slot; s < n_rows * a.heads; s += g.slots) {
        const uint32_t r = s / a.heads, h = s % a.heads;
        const T *px = x + (int64_t)(row0 + r) * a.x_row + (int64_t)h * a.x_head;
        T *py = y + (int64_t)(row0 + r) * a.y_row + (int64_t)h * a.y_head;
        const float2 *c = cs + r * n;
        for (uint32_t j = threadIdx.x % g.items; j < g.items; j += kRotateThreads) {      // more than one step only where a head has more pieces than the workgroup lanes
            if (j >= g.pairs) {
                const uint32_t ch = 2 * n + (j - g.pairs) * N;
                float v[N];
                load_row<DT, N>(px + ch, v);
                store_row<DT, N>(py + ch, v);
            } else if (HALF) {
                float u[N], v[N];
                load_row<DT, N>(px + j * N, u);
                load_row<DT, N>(px + n + j * N, v);
#pragma unroll
                for (int e = 0; e < N; ++e) turn_pair(u[e], v[e], c[j * N + e]);
                store_row<DT, N>(py + j * N, u);
                store_row<DT, N>(py + n + j * N, v);
            } else if constexpr (N > 1) {
                float v[N];
                load_row<DT, N>(px + j * N, v);
#pragma unroll
                for (int e = 0; e < N; e += 2) turn_pair(v[e], v[e + 1], c[(j * N + e) / 2]);
                store_row<DT, N>(py + j * N, v);
            } else {
                float u = Elem<DT>::get(px[2 * j]), v = Elem<DT>::get(px[2 * j + 1]);
                turn_pair(u, v, c[j]);
                py[2 * j] = Elem<DT>::put(u);
                py[2 * j + 1] = Elem<DT>::put(v);
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
    g.tile = g.a.rows >= 8192 ? kRotateTileRows : g.a.rows >= 2048 ? 4 : 1;
    const dim3 grid((g.a.rows + g.tile - 1) / g.tile), block(kRotateThreads);
    if (half && vectors) PSV_LAUNCH((k_rotate<DT, true, N>), grid, block, 0, s, g);
    else if (half) PSV_LAUNCH((k_rotate<DT, true, 1>), grid, block, 0, s, g);
    else if (vectors) PSV_LAUNCH((k_rotate<DT, false, N>), grid, block, 0, s, g);
    else PSV_LAUNCH((k_rotate<DT, false, 1>), grid, block, 0, s, g);
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
