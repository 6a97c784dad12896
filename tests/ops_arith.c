/* The two corrected fp32 operations of the 8-bit optimizer state against IEEE results.
 *   root:      x RN-or-neighbour(1/sqrt(x)), corrected once by fma from its remainder, for every
 *              mantissa of two binades (the scale of 4 is exact), against the fp64 root rounded to
 *              fp32 (exact: 53 >= 2 * 24 + 2 bits): a handful differ, by one step;
 *   quotient:  x / s from the reciprocal (RN or a neighbour) refined once, the product corrected
 *              once: none may differ from x / s.
 * Prints how many differ, and by how many steps at most. */
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

static float as_float(uint32_t b) { float f; memcpy(&f, &b, 4); return f; }
static uint32_t as_bits(float f) { uint32_t b; memcpy(&b, &f, 4); return b; }

int main(void)
{
    long long roots = 0, quotients = 0, worst = 0;
#pragma omp parallel for reduction(+ : roots) reduction(max : worst)
    for (uint32_t b = 0x3F800000u; b < 0x40800000u; ++b) {
        const float x = as_float(b), want = (float)sqrt((double)x), h0 = (float)(1.0 / sqrt((double)x));
        for (int ulp = -1; ulp <= 1; ++ulp) {
            const float h = as_float(as_bits(h0) + (uint32_t)ulp);
            const volatile float y = x * h;
            const float root = fmaf(fmaf(-y, y, x), 0.5f * h, y);
            const long long off = llabs((long long)as_bits(root) - (long long)as_bits(want));
            roots += off != 0;
            worst = off > worst ? off : worst;
        }
    }
#pragma omp parallel for reduction(+ : quotients)
    for (int k = 0; k < 2000; ++k) {
        const float s = as_float(0x3F800000u | (((uint32_t)k * 2654435761u) >> 9)), r0 = (float)(1.0 / (double)s);
        for (int ulp = -1; ulp <= 1; ++ulp) {
            const float i0 = as_float(as_bits(r0) + (uint32_t)ulp), i = fmaf(fmaf(-s, i0, 1.0f), i0, i0);
            for (uint32_t j = 0; j < 8000; ++j) {
                const uint32_t z = (j * 2246822519u) ^ ((uint32_t)k * 3266489917u);
                const float x = as_float(0x3F000000u + (z >> 8) % 0x01000000u);
                const volatile float q = x * i, want = x / s;
                quotients += fmaf(fmaf(-q, s, x), i, q) != want;
            }
        }
    }
    printf("root %lld by %lld quotient %lld\n", roots, worst, quotients);
    return 0;
}
