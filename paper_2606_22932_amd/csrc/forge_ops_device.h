// Device-side helpers of forge_norm.hip and forge_multi.hip: eight consecutive elements of
// any type to and from fp32 registers, lane reductions, E4M3 codes.
#pragma once

#include "forge_device.h"
#include "forge_ops_arith.h"

namespace forge_impl {

// Device memory, told to the compiler for pointers that it cannot trace to a kernel argument (the
// table's): it would take flat accesses for them, which occupy the LDS counter too.
template <class T> using Global = T __attribute__((address_space(1))) *;
template <class T> __device__ __forceinline__ Global<const T> global_of(const void *p, size_t i = 0)
{
    return (Global<const T>)(static_cast<const T *>(p) + i);
}
template <class T> __device__ __forceinline__ Global<T> global_of(void *p, size_t i = 0)
{
    return (Global<T>)(static_cast<T *>(p) + i);
}
// Elements i .. of p as one vector V; T is what i counts.
template <class V, class T, bool NT> __device__ __forceinline__ V load_v(const void *p, size_t i)
{
    const auto q = (Global<const V>)global_of<T>(p, i);
    if constexpr (NT) return __builtin_nontemporal_load(q);
    else return *q;
}
template <class T, bool NT, class V> __device__ __forceinline__ void store_v(void *p, size_t i, V x)
{
    const auto q = (Global<V>)global_of<T>(p, i);
    if constexpr (NT) __builtin_nontemporal_store(x, q);
    else *q = x;
}

// N consecutive elements (4 or 8) from p[i ..] as they lie in memory, and as fp32 values.  bf16:
// 2 N bytes in one access; fp32: 16 bytes an access.  NT: non-temporal.
template <bool BF16, int N> struct Raw;
template <int N> struct Raw<true, N> {
    uint32_t u[N / 2];
    template <bool NT = false> __device__ __forceinline__ void load(const void *p, size_t i)
    {
        typedef uint32_t V __attribute__((ext_vector_type(N / 2)));
        const V x = load_v<V, uint16_t, NT>(p, i);
#pragma unroll
        for (int k = 0; k < N / 2; ++k) u[k] = x[k];
    }
    __device__ __forceinline__ float at(int k) const { return k & 1 ? bf_hi(u[k >> 1]) : bf_lo(u[k >> 1]); }
    __device__ __forceinline__ void set(const float (&f)[N])
    {
#pragma unroll
        for (int k = 0; k < N / 2; ++k) u[k] = pack_bf16(f[2 * k], f[2 * k + 1]);
    }
    template <bool NT = false> __device__ __forceinline__ void store(void *p, size_t i) const
    {
        typedef uint32_t V __attribute__((ext_vector_type(N / 2)));
        V x;
#pragma unroll
        for (int k = 0; k < N / 2; ++k) x[k] = u[k];
        store_v<uint16_t, NT>(p, i, x);
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int k = 0; k < N / 2; ++k) u[k] = 0;
    }
    // To the compiler another value: what it unpacked before is unpacked again, not kept.
    __device__ __forceinline__ void forget()
    {
#pragma unroll
        for (int k = 0; k < N / 2; ++k) asm volatile("" : "+v"(u[k]));
    }
};
template <int N> struct Raw<false, N> {
    f32x4_t v[N / 4];
    template <bool NT = false> __device__ __forceinline__ void load(const void *p, size_t i)
    {
#pragma unroll
        for (int k = 0; k < N / 4; ++k)
            v[k] = load_v<f32x4_t, float, NT>(p, i + 4 * k);
    }
    __device__ __forceinline__ float at(int k) const { return v[k >> 2][k & 3]; }
    __device__ __forceinline__ void set(const float (&f)[N])
    {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k >> 2][k & 3] = f[k];
    }
    template <bool NT = false> __device__ __forceinline__ void store(void *p, size_t i) const
    {
#pragma unroll
        for (int k = 0; k < N / 4; ++k) store_v<float, NT>(p, i + 4 * k, v[k]);
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int k = 0; k < N / 4; ++k) v[k] = f32x4_t{0, 0, 0, 0};
    }
    __device__ __forceinline__ void forget() {}
};
template <bool BF16, int N, bool NT = false> __device__ __forceinline__ void load_n(const void *p, size_t i, float (&f)[N])
{
    Raw<BF16, N> r;
    r.template load<NT>(p, i);
#pragma unroll
    for (int k = 0; k < N; ++k) f[k] = r.at(k);
}
template <bool BF16, bool NT = false, int N> __device__ __forceinline__ void store_n(void *p, size_t i, const float (&f)[N])
{
    Raw<BF16, N> r;
    r.set(f);
    r.template store<NT>(p, i);
}
// x rounded to the stored type and back.
template <bool BF16> __device__ __forceinline__ float as_stored(float x)
{
    return BF16 ? (float)(__bf16)x : x;
}

// Lane exchanges without LDS round trips, for reductions over aligned groups of lanes: each step
// gives a lane the value of one in the other half of a group twice as large, all lanes of a half
// holding the same.  0xB1 and 0x4E are the quad permutations [1,0,3,2] and [2,3,0,1], 0x141
// mirrors each half row of 8 lanes, 0x140 each row of 16.  Every lane must be active.
template <int CTRL> __device__ __forceinline__ uint32_t lane_dpp(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xF, 0xF, true);
}
template <class F> __device__ __forceinline__ uint32_t lanes_join(uint32_t x, int lanes, F f)
{
    x = f(x, lane_dpp<0xB1>(x));
    x = f(x, lane_dpp<0x4E>(x));
    x = f(x, lane_dpp<0x141>(x));
    if (lanes >= 16) x = f(x, lane_dpp<0x140>(x));
    if (lanes >= 32) {
        const auto h = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        x = f(h[0], h[1]);
    }
    if (lanes >= 64) {
        const auto h = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        x = f(h[0], h[1]);
    }
    return x;
}
// Sum or maximum over aligned groups of `lanes` (8, 16, 32 or 64) lanes, to all of them.
__device__ __forceinline__ float lanes_sum(float x, int lanes)
{
    return __uint_as_float(lanes_join(__float_as_uint(x), lanes, [](uint32_t a, uint32_t b) {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    }));
}
__device__ __forceinline__ uint32_t lanes_max(uint32_t x, int lanes)
{
    return lanes_join(x, lanes, [](uint32_t a, uint32_t b) { return max(a, b); });
}

// Magnitudes are compared as bit patterns, which order like the values with Inf and then NaN
// above them: a maximum over a block with a NaN is NaN.
__device__ __forceinline__ uint32_t mag(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }
template <int N> __device__ __forceinline__ uint32_t mag_n(const float (&f)[N])
{
    uint32_t b = 0;
#pragma unroll
    for (int k = 0; k < N; ++k) b = max(b, mag(f[k]));
    return b;
}

// Scale of a block of E4M3 codes: amax RN(1/448) in fp32, zero where that is no normal number.
// A NaN amax keeps its NaN and an Inf its Inf, so that such a block decodes to no finite number.
__device__ __forceinline__ float e4m3_scale(uint32_t amax)
{
    const float scale = __uint_as_float(amax) * (1.0f / 448.0f);
    return scale < 0x1p-126f ? 0.0f : scale;
}

// The values of a block divided by its scale, as IEEE division rounds them; all zero for a scale of
// zero, and by an Inf or NaN scale zero for every finite value.
template <int N> __device__ __forceinline__ void e4m3_quotients(float (&x)[N], float scale)
{
    if (!(scale >= E4M3_SMALL && scale < __builtin_inff())) {
        const bool some = scale > 0.0f && scale < __builtin_inff();
        scale = some ? scale * E4M3_LIFT : 1.0f;
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = some ? x[k] * E4M3_LIFT : x[k] * 0.0f + 0.0f;      // no -0
    }
    const float i = inverse_from(scale, __builtin_amdgcn_rcpf(scale));
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = quotient_from(x[k], scale, i);
}

// Codes of four values already divided by their scale, rounded to nearest even, as a word.  A
// quotient by the scale lies at most a few steps above 448, far below 464, past which the hardware
// conversion gives NaN.
__device__ __forceinline__ uint32_t e4m3_codes4(const float *x)
{
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false), true);
}
template <int N> __device__ __forceinline__ void e4m3_decode(const uint32_t (&c)[N / 4], float (&x)[N])
{
#pragma unroll
    for (int k = 0; k < N / 4; ++k) {
        const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[k], false);
        const f32x2_t hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[k], true);
        x[4 * k] = lo[0];
        x[4 * k + 1] = lo[1];
        x[4 * k + 2] = hi[0];
        x[4 * k + 3] = hi[1];
    }
}

}  // namespace forge_impl
