// The fp32 arithmetic behind the E4M3 codes, from products and fused multiply-adds alone, so that
// the host can run the same functions over every mantissa (there with __host__ and __device__
// defined as nothing).
#pragma once

namespace forge_impl {

// RN(sqrt(z)) from an approximation h of 1 / sqrt(z) good to two steps: root and half reciprocal
// refined together (Goldschmidt), then the root corrected by its exact remainder (Markstein).  Right
// for every mantissa; correcting z h alone left up to three of 2^24 a step off.  z from 2^-96 on,
// so that no remainder underflows.
__host__ __device__ inline float root_from(float z, float h)
{
    float y = z * h, k = 0.5f * h;
    const float r = __builtin_fmaf(-k, y, 0.5f);
    y = __builtin_fmaf(y, r, y);
    k = __builtin_fmaf(k, r, k);
    return __builtin_fmaf(__builtin_fmaf(-y, y, z), k, y);
}

// RN(1 / s) of a normal s from an approximation i good to two steps: two Newton steps, each from
// the exact remainder, end at the rounded value for every mantissa but 2 - 2^-23, which is none of
// a scale's (of no fp32 number times RN(1/448)).
__host__ __device__ inline float inverse_from(float s, float i)
{
    i = __builtin_fmaf(__builtin_fmaf(-s, i, 1.0f), i, i);
    return __builtin_fmaf(__builtin_fmaf(-s, i, 1.0f), i, i);
}

// RN(x / s) with i = RN(1 / s): the product, corrected once by its remainder (Markstein's theorem:
// right wherever the remainder is exact).  The remainder is a multiple of the last bits' product,
// 2^-46 of x at least, and exact while that is no less than 2^-149: x from 2^-103 on.
__host__ __device__ inline float quotient_from(float x, float s, float i)
{
    const float q = x * i;
    return __builtin_fmaf(__builtin_fmaf(q, s, -x), -i, q);      // by these signs -0 stays -0
}

// Roots of values below this are taken of the value times ROOT_LIFT.
constexpr float ROOT_SMALL = 0x1p-96f, ROOT_LIFT = 0x1p64f, ROOT_UNLIFT = 0x1p-32f;
// Scales below this are taken times E4M3_LIFT, and their values with them, so that the remainders
// of all that is not coded as zero are exact.
constexpr float E4M3_SMALL = 0x1p-64f, E4M3_LIFT = 0x1p64f;

}  // namespace forge_impl
