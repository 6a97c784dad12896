// The arithmetic of the E4M3 codes (forge_ops_arith.h, the kernels' own functions) against IEEE
// results, the hardware's approximation taken as the rounded value and its neighbours up to two
// steps off.  Prints how many results differ:
//   scale      amax RN(1/448) with the mantissa 2 - 2^-23, which the inverse does not cover;
//   inverse    1 / s, every other mantissa of s;
//   quotient   x / s, every mantissa of s, values of x at random, next to s and at both ends, and
//              zeros of either sign;
//   small      x / s of scales of every exponent from 2^-126 on, as a block is divided: x up to
//              448 s, down to what is coded as zero.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>

#define __host__
#define __device__
#include "forge_ops_arith.h"

using namespace forge_impl;

static float as_float(uint32_t b) { float f; std::memcpy(&f, &b, 4); return f; }
static uint32_t as_bits(float f) { uint32_t b; std::memcpy(&b, &f, 4); return b; }
static uint32_t next(uint32_t &z) { return (z = z * 1664525u + 1013904223u) >> 9; }

int main()
{
    const uint32_t last = 0x7FFFFFu;
    long long scales = 0, inverses = 0, smalls = 0;
    long long quotients = !std::signbit(quotient_from(-0.0f, 3.0f, 1.0f / 3.0f)) + std::signbit(quotient_from(0.0f, 3.0f, 1.0f / 3.0f));
#pragma omp parallel for reduction(+ : scales, inverses, quotients)
    for (uint32_t m = 0; m <= last; ++m) {
        scales += (as_bits(as_float(0x3F800000u | m) * (1.0f / 448.0f)) & last) == last;
        if (m == last) continue;
        const float s = as_float(0x3F800000u | m), want = (float)(1.0 / (double)s);
        for (int ulp = -2; ulp <= 2; ++ulp)
            inverses += inverse_from(s, as_float(as_bits(want) + (uint32_t)ulp)) != want;
        uint32_t z = m * 2654435761u;
        for (uint32_t j = 0; j < 16; ++j) {
            const uint32_t k = j < 2 ? j : j < 4 ? last + 2 - j : j < 8 ? (m + j - 6) & last : next(z);
            const float x = as_float(0x3F800000u | k);
            quotients += quotient_from(x, s, want) != x / s;
        }
    }
#pragma omp parallel for reduction(+ : smalls)
    for (int e = -126; e <= 100; ++e) {
        uint32_t z = (uint32_t)e * 2246822519u;
        for (int j = 0; j < 100000; ++j) {
            const uint32_t m = next(z);
            float s = std::ldexp(as_float(0x3F800000u | (m - (m == last))), e);
            float x = std::ldexp(as_float(0x3F800000u | next(z)), e - 11 + (int)(next(z) % 20u));
            const float want = x / s;
            if (s < E4M3_SMALL) {
                s *= E4M3_LIFT;
                x *= E4M3_LIFT;
            }
            smalls += quotient_from(x, s, inverse_from(s, (float)(1.0 / (double)s))) != want;
        }
    }
    std::printf("scale %lld inverse %lld quotient %lld small %lld\n", scales, inverses, quotients, smalls);
    return 0;
}
