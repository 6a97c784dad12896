// The square root behind the E4M3 codes of sqrt(v) (forge_ops_arith.h, the kernels' own function)
// against the fp64 root rounded to fp32 (exact: 53 >= 2 * 24 + 2 bits), the hardware's reciprocal
// root taken as the rounded value and its neighbours up to two steps off.  Prints how many differ:
//   root    every mantissa of two binades;
//   range   values of every exponent from 2^-149 on, small ones times 2^64 as the kernel takes them.
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
static float approx(float z, int ulp) { return as_float(as_bits((float)(1.0 / std::sqrt((double)z))) + (uint32_t)ulp); }

int main()
{
    long long roots = 0, range = 0;
#pragma omp parallel for reduction(+ : roots)
    for (uint32_t b = 0x3F800000u; b < 0x40800000u; ++b) {
        const float x = as_float(b), want = (float)std::sqrt((double)x);
        for (int ulp = -2; ulp <= 2; ++ulp) roots += root_from(x, approx(x, ulp)) != want;
    }
    for (uint32_t b = 1; b < 0x7F800000u; b += b < 0x800000u ? 37 : 1021) {
        const float x = as_float(b);
        const bool small = x < ROOT_SMALL;
        const float z = small ? x * ROOT_LIFT : x;
        for (int ulp = -2; ulp <= 2; ++ulp) {
            const float root = root_from(z, approx(z, ulp));
            range += (small ? root * ROOT_UNLIFT : root) != (float)std::sqrt((double)x);
        }
    }
    std::printf("root %lld range %lld\n", roots, range);
    return 0;
}
