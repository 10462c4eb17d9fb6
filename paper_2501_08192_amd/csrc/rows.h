// Device-side pieces of the operators that work on rows of elements: conversions of the three element types, vectors of 16
// bytes, and the rotary angle.
#ifndef PSV_ROWS_H
#define PSV_ROWS_H

#include "device.h"
#include "operators.h"

namespace psv {

// N elements of a type as 32-bit floats, and back with one rounding to nearest even.
template <uint32_t DT> struct Elem;
template <> struct Elem<PSV_F32> {
    using T = float;
    static constexpr int N = 4;      // a vector of 16 bytes
    __device__ static float get(T v) { return v; }
    __device__ static T put(float v) { return v; }
};
template <> struct Elem<PSV_BF16> {
    using T = uint16_t;
    static constexpr int N = 8;
    __device__ static float get(T v) { return __uint_as_float((uint32_t)v << 16); }
    __device__ static T put(float v) { return (T)f32_to_bf16(v); }
};
template <> struct Elem<PSV_F16> {
    using T = _Float16;
    static constexpr int N = 8;
    __device__ static float get(T v) { return (float)v; }
    __device__ static T put(float v) { return (T)v; }
};

template <uint32_t DT, int N>
struct Pack { typename Elem<DT>::T e[N]; };

// N adjacent elements, in one load or store of 16 (or 8) bytes where N is that many.  A load and its conversion apart: kernels request the rows of
// their next step before they work on this one's.
template <uint32_t DT, int N>
__device__ __forceinline__ Pack<DT, N> fetch_row(const typename Elem<DT>::T *p)
{
    using P = Pack<DT, N>;
    struct alignas(sizeof(P) > 16 ? 16 : sizeof(P)) A { P p; };
    return reinterpret_cast<const A *>(p)->p;
}
template <uint32_t DT, int N>
__device__ __forceinline__ void unpack_row(const Pack<DT, N> &t, float (&v)[N])
{
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = Elem<DT>::get(t.e[e]);
}
template <uint32_t DT, int N>
__device__ __forceinline__ void load_row(const typename Elem<DT>::T *p, float (&v)[N])
{
    unpack_row<DT, N>(fetch_row<DT, N>(p), v);
}
template <uint32_t DT, int N>
__device__ __forceinline__ void store_row(typename Elem<DT>::T *p, const float (&v)[N])
{
    using P = Pack<DT, N>;
    struct alignas(sizeof(P) > 16 ? 16 : sizeof(P)) A { P p; };
    A t;
    if constexpr (DT == PSV_BF16 && N % 2 == 0) {
        uint32_t w[N / 2];
#pragma unroll
        for (int e = 0; e < N / 2; ++e) w[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
        __builtin_memcpy(&t, w, sizeof t);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) t.p.e[e] = Elem<DT>::put(v[e]);
    }
    *reinterpret_cast<A *>(p) = t;
}

// (cos, sin) of an angle in 64 bits, times a magnitude, rounded once.  The angle is reduced to a quarter turn either way (its multiple
// of pi/2 taken off in two pieces, exact for any position that an int32 holds); there the Taylor series to x^13 and x^14 are
// off by less than 2e-14.  About 30 instructions in 64 bits; the library's sincos, which also reduces angles beyond 2^40, takes several
// times that and registers that these kernels want for their rows.
__device__ __forceinline__ float2 turn(double angle, double magnitude)
{
    const double k = __builtin_rint(angle * 0.63661977236758134);          // 2 / pi
    double r = fma(-k, 1.5707963267948966, angle);                         // pi / 2, rounded
    r = fma(-k, 6.123233995736766e-17, r);                                 // ... and what the rounding left
    const double z = r * r;
    double s = 1.0 / 6227020800.0;                                         // 1 / 13!
    s = fma(s, z, -1.0 / 39916800.0);
    s = fma(s, z, 1.0 / 362880.0);
    s = fma(s, z, -1.0 / 5040.0);
    s = fma(s, z, 1.0 / 120.0);
    s = fma(s, z, -1.0 / 6.0);
    s = fma(s * z, r, r);
    double c = -1.0 / 87178291200.0;                                       // 1 / 14!
    c = fma(c, z, 1.0 / 479001600.0);
    c = fma(c, z, -1.0 / 3628800.0);
    c = fma(c, z, 1.0 / 40320.0);
    c = fma(c, z, -1.0 / 720.0);
    c = fma(c, z, 1.0 / 24.0);
    c = fma(c, z, -0.5);
    c = fma(c, z, 1.0);
    const long long q = (long long)k;
    const double cc = (q & 1) ? s : c, ss = (q & 1) ? c : s;
    return make_float2((float)(((q + 1) & 2) ? -cc * magnitude : cc * magnitude), (float)((q & 2) ? -ss * magnitude : ss * magnitude));
}

// Maximum over the 64 lanes of a wave, returned in every lane (all lanes must be active).
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, true));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, true));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, true));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xf, 0xf, true));
    const uint32_t a = max((uint32_t)__builtin_amdgcn_readlane((int)v, 0), (uint32_t)__builtin_amdgcn_readlane((int)v, 16));
    return max(a, max((uint32_t)__builtin_amdgcn_readlane((int)v, 32), (uint32_t)__builtin_amdgcn_readlane((int)v, 48)));
}

// Pairs (a, b) turned: a' = a c - b s, b' = b c + a s.
__device__ __forceinline__ void turn_pair(float &a, float &b, float2 cs)
{
    const float a0 = a, b0 = b;
    a = a0 * cs.x - b0 * cs.y;
    b = b0 * cs.x + a0 * cs.y;
}

}  // namespace psv

#endif
