// forge_multi.hip -- one pass over the tensors of a list: the norm of their gradients, and
// their AdamW step (include/forge_ops.h).
#include "forge_ops_device.h"
#include "forge_ops_internal.h"

namespace forge_impl {

namespace {

constexpr int NTH = 256;
static_assert(MT_CHUNK == NTH * 8, "a thread's share of a chunk is eight elements");

// Eight elements from i on, of which the first n exist (n >= 8: all of them); zeros after them.
template <int TY> __device__ __forceinline__ void load_some(const void *p, size_t i, int n, float (&f)[8])
{
    if (n >= 8) {
        load_n<TY == MT_BF16>(p, i, f);
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        f[k] = 0.0f;
        if (k < n) {
            if constexpr (TY == MT_BF16) f[k] = bf_lo(static_cast<const uint16_t *>(p)[i + k]);
            else f[k] = static_cast<const float *>(p)[i + k];
        }
    }
}
template <int TY> __device__ __forceinline__ void store_some(void *p, size_t i, int n, const float (&f)[8])
{
    if (n >= 8) {
        store_n<TY == MT_BF16>(p, i, f);
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < n) {
            if constexpr (TY == MT_BF16) static_cast<uint16_t *>(p)[i + k] = (uint16_t)pack_bf16(f[k], 0.0f);
            else static_cast<float *>(p)[i + k] = f[k];
        }
}
__device__ __forceinline__ void load_codes(const void *p, size_t i, int n, float (&f)[8])
{
    const uint8_t *b = static_cast<const uint8_t *>(p) + i;
    u32x2_t c = {0, 0};
    if (n >= 8) {
        c = *reinterpret_cast<const u32x2_t *>(b);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < n) c[k >> 2] |= (uint32_t)b[k] << (8 * (k & 3));
    }
    e4m3_decode8(c, f);
}
__device__ __forceinline__ void store_codes(void *p, size_t i, int n, const u32x2_t &c)
{
    uint8_t *b = static_cast<uint8_t *>(p) + i;
    if (n >= 8) {
        *reinterpret_cast<u32x2_t *>(b) = c;
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < n) b[k] = (uint8_t)(c[k >> 2] >> (8 * (k & 3)));
    }
}

// sqrt(x) rounded to nearest: the product with the reciprocal root, corrected by the exact
// remainder once.  Against the fp64 root over every fp32 mantissa, with the hardware's result and
// its two neighbours: another value in 5 of 50331648 cases, one step off.  Small x are taken
// times 2^64, so that no remainder underflows.
__device__ __forceinline__ float rounded_root(float x)
{
    const bool small = x < 0x1p-96f;
    const float z = small ? x * 0x1p64f : x;
    const float h = __builtin_amdgcn_rsqf(fmaxf(z, 0x1p-126f));
    const float y = z * h, root = __builtin_fmaf(__builtin_fmaf(-y, y, z), 0.5f * h, y);
    return z < __builtin_inff() ? (small ? root * 0x1p-32f : root) : z;      // Inf and NaN as they are
}
// x / s rounded to nearest from i = RN(1 / s): again one correction by the exact remainder (no
// difference from IEEE division in 2.4e8 cases, i off by a step or not before its refinement).
__device__ __forceinline__ float refined_inverse(float s)
{
    const float i = e4m3_inverse(s);
    return __builtin_fmaf(__builtin_fmaf(-s, i, 1.0f), i, i);
}
__device__ __forceinline__ float rounded_quotient(float x, float s, float i)
{
    const float q = x * i;
    return __builtin_fmaf(__builtin_fmaf(-q, s, x), i, q);
}

// One AdamW element (Algorithm 1).  fp32 and bf16 state: the arithmetic of forge_adamw's kernels
// to the bit.  fp8 state: every operation up to the codes is one IEEE fp32 operation, none of
// them fused, the root and the quotient by the scale correctly rounded.  Next to the border of
// two codes the last bit of m' or sqrt(v') decides, and a step later that code decides a block's
// scale; so the state of a run is what these formulas give in plain fp32 anywhere.
template <bool EXACT>
__device__ __forceinline__ void adamw1(float g, float &w, float &m, float &v, float &root, const MtHyper &h,
                                       float lr_bc1, float wdf)
{
    if constexpr (EXACT) {
        m = h.b1 * m + h.c1 * g;
        v = h.b2 * v + h.c2 * (g * g);
        root = rounded_root(v);
    } else {
        m = __builtin_fmaf(h.b1, m, h.c1 * g);
        v = __builtin_fmaf(h.b2, v, (h.c2 * g) * g);
        root = __builtin_amdgcn_sqrtf(v);
    }
    const float den = __builtin_fmaf(root, h.inv_sqrt_bc2, h.eps);
    w = __builtin_fmaf(wdf, w, -((m * lr_bc1) * __builtin_amdgcn_rcpf(den)));
}

// A workgroup's chunk of one tensor, eight elements a thread.
template <int WT, int GT, int ST>
__device__ __forceinline__ void adamw_chunk(const MtTensor &t, size_t i, int n, const MtHyper &h, float scale)
{
    const float lr_bc1 = (float)((double)t.lr_scale * h.lr_bc1);
    const float wdf = (float)(1.0 - h.lr * (double)t.lr_scale * (double)t.wd);
    float w[8], g[8], m[8], v[8], root[8];
    load_some<WT>(t.W, i, n, w);
    load_some<GT>(t.G, i, n, g);
    if constexpr (ST == MT_FP8) {
        load_codes(t.m, i, n, m);
        load_codes(t.v, i, n, v);
        float ms = 0.0f, vs = 0.0f;
        if (n > 0) {
            ms = t.ms[i / MT_BLOCK];
            vs = t.vs[i / MT_BLOCK];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            m[k] *= ms;
            v[k] *= vs;
            v[k] *= v[k];
        }
    } else {
        load_some<ST>(t.m, i, n, m);
        load_some<ST>(t.v, i, n, v);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) adamw1<ST == MT_FP8>(g[k] * scale, w[k], m[k], v[k], root[k], h, lr_bc1, wdf);
    store_some<WT>(t.W, i, n, w);
    if constexpr (ST == MT_FP8) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k >= n) m[k] = root[k] = 0.0f;
        const float ms = e4m3_scale(lanes_max(mag_n(m), 8));
        const float vs = e4m3_scale(lanes_max(mag_n(root), 8));
        const float mi = refined_inverse(ms), vi = refined_inverse(vs);
        float lo[8];
        if (n > 0 && i % MT_BLOCK == 0) {
            t.ms[i / MT_BLOCK] = ms;
            t.vs[i / MT_BLOCK] = vs;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            m[k] = rounded_quotient(m[k], ms, mi);
            lo[k] = root[k] > 0.0f ? 0x1p-9f : 0.0f;      // a sqrt(v) > 0 is not stored as zero
            root[k] = rounded_quotient(root[k], vs, vi);
        }
        store_codes(t.m, i, n, u32x2_t{e4m3_encode4(m[0], m[1], m[2], m[3]), e4m3_encode4(m[4], m[5], m[6], m[7])});
        store_codes(t.v, i, n, u32x2_t{e4m3_encode4(root[0], root[1], root[2], root[3], lo[0], lo[1], lo[2], lo[3]),
                                e4m3_encode4(root[4], root[5], root[6], root[7], lo[4], lo[5], lo[6], lo[7])});
    } else {
        store_some<ST>(t.m, i, n, m);
        store_some<ST>(t.v, i, n, v);
    }
}

template <int WT, int GT>
__device__ __forceinline__ void adamw_state(const MtTensor &t, size_t i, int n, const MtHyper &h, float scale)
{
    if (t.st == MT_F32) adamw_chunk<WT, GT, MT_F32>(t, i, n, h, scale);
    else if (t.st == MT_BF16) adamw_chunk<WT, GT, MT_BF16>(t, i, n, h, scale);
    else adamw_chunk<WT, GT, MT_FP8>(t, i, n, h, scale);
}

__global__ void __launch_bounds__(NTH) adamw_multi_kernel(MtTable tab, MtHyper h, const float *grad_scale)
{
    const int c = blockIdx.x;
    const MtTensor t = tab.t[tab.owner[c]];
    const float scale = grad_scale ? *grad_scale : 1.0f;
    const size_t i = (size_t)(c - t.first) * MT_CHUNK + 8 * threadIdx.x;
    const int n = (int)min((int64_t)8, max((int64_t)0, (int64_t)t.numel - (int64_t)i));
    if (t.wt == MT_F32) {
        if (t.gt == MT_F32) adamw_state<MT_F32, MT_F32>(t, i, n, h, scale);
        else adamw_state<MT_F32, MT_BF16>(t, i, n, h, scale);
    } else {
        if (t.gt == MT_F32) adamw_state<MT_BF16, MT_F32>(t, i, n, h, scale);
        else adamw_state<MT_BF16, MT_BF16>(t, i, n, h, scale);
    }
}

__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) x += __shfl_xor(x, o);
    return x;
}
__device__ __forceinline__ double group_sum(double x, double *red)
{
    x = wave_sum(x);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.0;
    for (int k = 0; k < NTH / 64; ++k) x += red[k];
    return x;
}

// The squares of the chunks from `blockIdx.x` on, gridDim.x apart, in fp64.
__global__ void __launch_bounds__(NTH) grad_norm_kernel(MtTable tab, double *part)
{
    __shared__ double red[NTH / 64];
    double sum = 0.0;
    for (int64_t c = blockIdx.x; c < tab.chunks; c += gridDim.x) {
        const MtTensor &t = tab.t[tab.owner[c]];
        const size_t i = (size_t)(c - t.first) * MT_CHUNK + 8 * threadIdx.x;
        const int n = (int)min((int64_t)8, max((int64_t)0, (int64_t)t.numel - (int64_t)i));
        float g[8];
        if (t.gt == MT_F32) load_some<MT_F32>(t.G, i, n, g);
        else load_some<MT_BF16>(t.G, i, n, g);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum = __builtin_fma((double)g[k], (double)g[k], sum);
    }
    sum = group_sum(sum, red);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

__global__ void __launch_bounds__(NTH) grad_norm_finish_kernel(const double *part, int parts, float max_norm, float *out)
{
    __shared__ double red[NTH / 64];
    double sum = 0.0;
    for (int p = threadIdx.x; p < parts; p += NTH) sum += part[p];
    sum = group_sum(sum, red);
    if (threadIdx.x == 0) {
        const double norm = sqrt(sum), c = (double)max_norm / (norm + 1e-6);
        out[0] = (float)norm;
        out[1] = c > 1.0 ? 1.0f : (float)c;      // a NaN stays one
    }
}

}  // namespace

hipError_t launch_grad_norm(const MtTable &t, float max_norm, float *out, double *part, hipStream_t stream)
{
    const int parts = (int)(t.chunks < MT_NORM_PARTS ? t.chunks : MT_NORM_PARTS);
    if (parts > 0) {
        grad_norm_kernel<<<parts, NTH, 0, stream>>>(t, part);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    grad_norm_finish_kernel<<<1, NTH, 0, stream>>>(part, parts, max_norm, out);
    return hipGetLastError();
}

hipError_t launch_adamw_multi(const MtTable &t, const MtHyper &h, const float *grad_scale, hipStream_t stream)
{
    adamw_multi_kernel<<<(unsigned)t.chunks, NTH, 0, stream>>>(t, h, grad_scale);
    return hipGetLastError();
}

}  // namespace forge_impl
