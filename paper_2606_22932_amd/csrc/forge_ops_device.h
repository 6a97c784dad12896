// Device-side helpers of forge_norm.hip and forge_multi.hip: eight consecutive elements of
// any type to and from fp32 registers, lane reductions, E4M3 codes.
#pragma once

#include "forge_device.h"

namespace forge_impl {

// Eight elements from p[i ..] in registers.  bf16: 16 bytes; fp32: 32 bytes.
template <bool BF16> __device__ __forceinline__ void load8(const void *p, size_t i, float (&f)[8])
{
    if constexpr (BF16) {
        const u32x4_t u = *reinterpret_cast<const u32x4_t *>(static_cast<const uint16_t *>(p) + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            f[2 * k] = bf_lo(u[k]);
            f[2 * k + 1] = bf_hi(u[k]);
        }
    } else {
        const f32x4_t a = *reinterpret_cast<const f32x4_t *>(static_cast<const float *>(p) + i);
        const f32x4_t b = *reinterpret_cast<const f32x4_t *>(static_cast<const float *>(p) + i + 4);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            f[k] = a[k];
            f[4 + k] = b[k];
        }
    }
}
template <bool BF16> __device__ __forceinline__ void store8(void *p, size_t i, const float (&f)[8])
{
    if constexpr (BF16) {
        u32x4_t u;
#pragma unroll
        for (int k = 0; k < 4; ++k) u[k] = pack_bf16(f[2 * k], f[2 * k + 1]);
        *reinterpret_cast<u32x4_t *>(static_cast<uint16_t *>(p) + i) = u;
    } else {
        f32x4_t a, b;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            a[k] = f[k];
            b[k] = f[4 + k];
        }
        *reinterpret_cast<f32x4_t *>(static_cast<float *>(p) + i) = a;
        *reinterpret_cast<f32x4_t *>(static_cast<float *>(p) + i + 4) = b;
    }
}
// x rounded to the stored type and back.
template <bool BF16> __device__ __forceinline__ float as_stored(float x)
{
    return BF16 ? (float)(__bf16)x : x;
}

// Sum over a workgroup of NT threads in a fixed order, to every thread.  `red` holds
// NT / 64 floats and is free again after the caller's next barrier.
template <int NT> __device__ __forceinline__ float group_sum(float x, float *red)
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) x += __shfl_xor(x, o);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.0f;
#pragma unroll
    for (int k = 0; k < NT / 64; ++k) x += red[k];
    return x;
}

// Magnitudes are compared as bit patterns, which order like the values with Inf and then NaN
// above them: a maximum over a block with a NaN is NaN.
__device__ __forceinline__ uint32_t mag(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t mag8(const float (&f)[8])
{
    uint32_t b = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) b = max(b, mag(f[k]));
    return b;
}
// Maximum over aligned groups of `lanes` (a power of two) lanes, to all of them; every lane active.
template <int LANES> __device__ __forceinline__ uint32_t lanes_max(uint32_t b)
{
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) b = max(b, (uint32_t)__shfl_xor((int)b, o));
    return b;
}
template <int NT> __device__ __forceinline__ uint32_t group_max(uint32_t b, uint32_t *red)
{
    b = lanes_max<64>(b);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = b;
    __syncthreads();
    b = 0;
#pragma unroll
    for (int k = 0; k < NT / 64; ++k) b = max(b, red[k]);
    return b;
}

// Scale of a block of E4M3 codes: amax RN(1/448) in fp32, zero where that is no normal number.
// A NaN amax keeps its NaN and an Inf its Inf, so that such a block decodes to no finite number.
__device__ __forceinline__ float e4m3_scale(uint32_t amax)
{
    const float scale = __uint_as_float(amax) * (1.0f / 448.0f);
    return scale < 0x1p-126f ? 0.0f : scale;
}
// Its reciprocal to one step, zero for a scale of zero.
__device__ __forceinline__ float e4m3_inverse(float scale)
{
    return scale > 0.0f ? __builtin_amdgcn_rcpf(scale) : 0.0f;
}

// Codes of eight values already divided by their scale, clamped to [lo, 448] first (the
// hardware conversion gives NaN past 464), rounded to nearest even.
__device__ __forceinline__ u32x2_t e4m3_encode8(const float (&x)[8], const float (&lo)[8])
{
    u32x2_t c;
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = __builtin_amdgcn_fmed3f(x[e], lo[e], 448.0f);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int h = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * k], y[4 * k + 1], 0, false);
        c[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * k + 2], y[4 * k + 3], h, true);
    }
    return c;
}
__device__ __forceinline__ u32x2_t e4m3_encode8(const float (&x)[8])
{
    const float lo[8] = {-448.0f, -448.0f, -448.0f, -448.0f, -448.0f, -448.0f, -448.0f, -448.0f};
    return e4m3_encode8(x, lo);
}
__device__ __forceinline__ void e4m3_decode8(const u32x2_t &c, float (&x)[8])
{
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[k], false);
        const f32x2_t hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[k], true);
        x[4 * k] = lo[0];
        x[4 * k + 1] = lo[1];
        x[4 * k + 2] = hi[0];
        x[4 * k + 3] = hi[1];
    }
}

}  // namespace forge_impl
