// forge_norm.hip -- residual add and RMS norm, forward and backward (include/forge_ops.h).
#include "forge_ops_device.h"
#include "forge_ops_internal.h"

namespace forge_impl {

namespace {

constexpr int NTH = 256;
constexpr int MAX_GROUPS = 1 << 20;

// One workgroup per row, the row read once for the sum of squares and once more (from cache)
// for the outputs.
template <bool HB, bool WB>
__global__ void __launch_bounds__(NTH) norm_kernel(NormArgs a)
{
    __shared__ float red[NTH / 64];
    __shared__ uint32_t redm[NTH / 64];
    const int nv = a.d >> 3;
    const void *src = a.r ? a.h : a.x;
    for (int t = blockIdx.x; t < a.T; t += gridDim.x) {
    const size_t row = (size_t)t * a.d;
    __syncthreads();                                      // red and redm are free
    float sum = 0.0f;
    for (int v = threadIdx.x; v < nv; v += NTH) {
        const size_t i = row + 8 * v;
        float f[8];
        if (a.r) {
            float x[8];
            load8<true>(a.x, i, x);
            load8<HB>(a.r, i, f);
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] = as_stored<HB>(f[k] + x[k]);
            store8<HB>(a.h, i, f);
        } else {
            load8<HB>(a.x, i, f);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) sum = __builtin_fmaf(f[k], f[k], sum);
    }
    sum = group_sum<NTH>(sum, red);
    const float s = __builtin_amdgcn_rsqf(sum / a.d + a.eps);
    auto out8 = [&](int v, float (&f)[8]) {
        float w[8];
        load8<HB>(src, row + 8 * v, f);
        load8<WB>(a.w, 8 * v, w);
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = f[k] * s * w[k];
    };
    float rs = 0.0f, rinv = 0.0f;
    if (a.q && a.q_group == 0) {
        uint32_t b = 0;
        for (int v = threadIdx.x; v < nv; v += NTH) {
            float f[8];
            out8(v, f);
            b = max(b, mag8(f));
        }
        rs = e4m3_scale(group_max<NTH>(b, redm));
        rinv = e4m3_inverse(rs);
        if (threadIdx.x == 0) a.qs[t] = rs;
    }
    const int groups = (nv + 15) >> 4;
    for (int v = threadIdx.x; v < (nv + 63) / 64 * 64; v += NTH) {     // whole waves
        float f[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (v < nv) out8(v, f);
        if (a.q && a.q_group) {
            rs = e4m3_scale(lanes_max<16>(mag8(f)));
            rinv = e4m3_inverse(rs);
            if (v < nv && (v & 15) == 0) a.qs[(size_t)t * groups + (v >> 4)] = rs;
        }
        if (v >= nv) continue;
        if (a.y) store8<true>(a.y, row + 8 * v, f);
        if (a.q) {
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] *= rinv;
            *reinterpret_cast<u32x2_t *>(a.q + row + 8 * v) = e4m3_encode8(f);
        }
    }
    }
}

// Workgroup b takes rows b, b + parts, ...: dh and dx of each, and its share of dw, which it
// sums in its row of the workspace.
template <bool HB, bool WB>
__global__ void __launch_bounds__(NTH) norm_grad_kernel(NormGradArgs a)
{
    __shared__ float red[2][NTH / 64];
    const int nv = a.d >> 3;
    float *part = a.part + (size_t)blockIdx.x * a.d;
    for (int t = blockIdx.x, first = 1; t < a.T; t += gridDim.x, first = 0) {
        const size_t row = (size_t)t * a.d;
        float s1 = 0.0f, s2 = 0.0f;
        auto in8 = [&](int v, float (&h)[8], float (&g)[8], float (&w)[8]) {
            load8<HB>(a.h, row + 8 * v, h);
            load8<true>(a.dy, row + 8 * v, g);
            load8<WB>(a.w, 8 * v, w);
        };
        for (int v = threadIdx.x; v < nv; v += NTH) {
            float h[8], g[8], w[8];
            in8(v, h, g, w);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                s1 = __builtin_fmaf(h[k], h[k], s1);
                s2 = __builtin_fmaf(g[k] * w[k], h[k], s2);
            }
        }
        __syncthreads();                                  // red is free
        s1 = group_sum<NTH>(s1, red[0]);
        s2 = group_sum<NTH>(s2, red[1]);
        const float s = __builtin_amdgcn_rsqf(s1 / a.d + a.eps);
        const float c = s * s * (s2 / a.d);
        for (int v = threadIdx.x; v < nv; v += NTH) {
            float h[8], g[8], w[8], o[8] = {0, 0, 0, 0, 0, 0, 0, 0}, p[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            in8(v, h, g, w);
            if (a.dres) load8<HB>(a.dres, row + 8 * v, o);
            if (!first) load8<false>(part, 8 * v, p);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                o[k] = __builtin_fmaf(s, __builtin_fmaf(-h[k], c, g[k] * w[k]), o[k]);
                p[k] = __builtin_fmaf(g[k], h[k] * s, p[k]);
            }
            if (a.dh) store8<HB>(a.dh, row + 8 * v, o);
            if (a.dx) store8<true>(a.dx, row + 8 * v, o);
            store8<false>(part, 8 * v, p);
        }
    }
}

// dw: the parts' sum, column by column.
__global__ void __launch_bounds__(64) norm_dw_kernel(const float *part, float *dw, int parts, int d)
{
    const int j = blockIdx.x * 64 + threadIdx.x;
    if (j >= d) return;
    float x = 0.0f;
    for (int p = 0; p < parts; ++p) x += part[(size_t)p * d + j];
    dw[j] = x;
}

}  // namespace

hipError_t launch_rmsnorm(const NormArgs &a, hipStream_t stream)
{
    auto k = a.h_bf16 ? (a.w_bf16 ? norm_kernel<true, true> : norm_kernel<true, false>)
                      : (a.w_bf16 ? norm_kernel<false, true> : norm_kernel<false, false>);
    k<<<a.T < MAX_GROUPS ? a.T : MAX_GROUPS, NTH, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_rmsnorm_backward(const NormGradArgs &a, hipStream_t stream)
{
    const int parts = norm_grad_parts(a.T, a.d);
    if (parts > 0) {
        auto k = a.h_bf16 ? (a.w_bf16 ? norm_grad_kernel<true, true> : norm_grad_kernel<true, false>)
                          : (a.w_bf16 ? norm_grad_kernel<false, true> : norm_grad_kernel<false, false>);
        k<<<parts, NTH, 0, stream>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    norm_dw_kernel<<<(a.d + 63) / 64, 64, 0, stream>>>(a.part, a.dw, parts, a.d);
    return hipGetLastError();
}

}  // namespace forge_impl
