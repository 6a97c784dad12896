// forge_multi.hip -- one pass over the tensors of a list: the norm of their gradients, and
// their AdamW step (include/forge_ops.h).
//
// Both are bound by HBM.  The tensors are cut into chunks of MT_CHUNK elements; a table in device
// memory says which tensor a chunk belongs to and what that is of, so that tensors of any sizes
// and types take one launch, whose parallelism does not depend on how the elements are spread
// over them.  A workgroup finds its tensor by two scalar loads one after the other.
#include "forge_ops_device.h"
#include "forge_ops_internal.h"

#include <type_traits>

namespace forge_impl {

namespace {

constexpr int NTH = 256;
static_assert(MT_CHUNK == NTH * 8, "a thread's share of a chunk is eight elements");

// A thread's share of a chunk is 8 / V vectors of V elements, the vectors of the chunk dealt out
// in turn, so that each access of a wave is one dense run: V is 8 where nothing is wider than
// bf16, else 4.  (With fp32 in runs of eight elements a lane, every access touches half of twice the
// lines: 1185 against 1084 us with fp32 throughout on 218 M elements.)

// Elements i .. i + V - 1 as they lie in memory, of which the first n exist (n >= V: all of them);
// zeros after them.
template <int TY, int V> struct Share {
    static constexpr int PER = TY == MT_F32 ? 1 : TY == MT_BF16 ? 2 : 4, WORDS = V / PER;      // elements of a word
    uint32_t u[WORDS];

    __device__ __forceinline__ void load(const void *p, size_t i, int n)
    {
        using T = std::conditional_t<TY == MT_F32, uint32_t, std::conditional_t<TY == MT_BF16, uint16_t, uint8_t>>;
        if (n >= V) {
            typedef uint32_t W __attribute__((ext_vector_type(WORDS)));
            const W x = load_v<W, T, true>(p, i);
#pragma unroll
            for (int k = 0; k < WORDS; ++k) u[k] = x[k];
            return;
        }
#pragma unroll
        for (int k = 0; k < WORDS; ++k) u[k] = 0;
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (k < n) u[k / PER] |= (uint32_t)*global_of<T>(p, i + k) << (32 / PER * (k % PER));
    }
    // The compiler takes the value as first used here.
    __device__ __forceinline__ void arrive()
    {
#pragma unroll
        for (int k = 0; k < WORDS; ++k) asm volatile("" : "+v"(u[k]));
    }
    __device__ __forceinline__ void get(float (&f)[V]) const
    {
        if constexpr (TY == MT_FP8) {
            e4m3_decode<V>(u, f);
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k) {
                if constexpr (TY == MT_F32) f[k] = __uint_as_float(u[k]);
                else f[k] = k & 1 ? bf_hi(u[k >> 1]) : bf_lo(u[k >> 1]);
            }
        }
    }
};
template <int TY, int V> __device__ __forceinline__ void store_some(void *p, size_t i, int n, const float (&f)[V])
{
    if (n >= V) {
        store_n<TY == MT_BF16, true>(p, i, f);
        return;
    }
#pragma unroll
    for (int k = 0; k < V; ++k)
        if (k < n) {
            if constexpr (TY == MT_BF16) *global_of<uint16_t>(p, i + k) = (uint16_t)pack_bf16(f[k], 0.0f);
            else *global_of<float>(p, i + k) = f[k];
        }
}
template <int V> __device__ __forceinline__ void store_codes(void *p, size_t i, int n, const uint32_t (&c)[V / 4])
{
    if (n >= V) {
        typedef uint32_t W __attribute__((ext_vector_type(V / 4)));
        W x;
#pragma unroll
        for (int k = 0; k < V / 4; ++k) x[k] = c[k];
        store_v<uint8_t, true>(p, i, x);
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (k < n) *global_of<uint8_t>(p, i + k) = (uint8_t)(c[k >> 2] >> (8 * (k & 3)));
    }
}

// sqrt(x) of a thread's share, rounded to nearest.  Where all lie between 2^-96 and Inf no remainder
// needs care; else x below it is taken times 2^64, whose root is exact, and 0, Inf and NaN are their own.
template <int V> __device__ __forceinline__ void rounded_roots(const float (&x)[V], float (&root)[V])
{
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int k = 1; k < V; ++k) {
        lo = fminf(lo, x[k]);
        hi = fmaxf(hi, x[k]);
    }
    if (lo >= ROOT_SMALL && hi < __builtin_inff()) {
#pragma unroll
        for (int k = 0; k < V; ++k) root[k] = root_from(x[k], __builtin_amdgcn_rsqf(x[k]));
        return;
    }
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const bool small = x[k] < ROOT_SMALL;
        const float z = small ? x[k] * ROOT_LIFT : x[k];
        const float y = root_from(z, __builtin_amdgcn_rsqf(z)) * (small ? ROOT_UNLIFT : 1.0f);
        root[k] = x[k] > 0.0f && x[k] < __builtin_inff() ? y : x[k];
    }
}

__device__ __forceinline__ float adamw_weight(float w, float m, float root, const MtHyper &h, float lr_bc1, float wdf)
{
    const float den = __builtin_fmaf(root, h.inv_sqrt_bc2, h.eps);
    return __builtin_fmaf(wdf, w, -((m * lr_bc1) * __builtin_amdgcn_rcpf(den)));
}

// One AdamW step of a thread's share (Algorithm 1).  fp32 and bf16 state: the arithmetic of
// forge_adamw's kernels to the bit.  fp8 state: every operation up to the codes is one IEEE fp32
// operation, none of them fused, the root and the quotient by the scale correctly rounded.  Next to
// the border of two codes the last bit of m' or sqrt(v') decides, and a step later that code decides
// a block's scale; so the state of a run is what these formulas give in plain fp32 anywhere.
template <bool EXACT, int V>
__device__ __forceinline__ void adamw(const float (&grad)[V], float scale, float (&w)[V], float (&m)[V], float (&v)[V],
                                      float (&root)[V], const MtHyper &h, float lr_bc1, float wdf)
{
    if constexpr (EXACT) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const float g = grad[k] * scale;
            m[k] = h.b1 * m[k] + h.c1 * g;
            v[k] = h.b2 * v[k] + h.c2 * (g * g);
        }
        rounded_roots(v, root);
#pragma unroll
        for (int k = 0; k < V; ++k) w[k] = adamw_weight(w[k], m[k], root[k], h, lr_bc1, wdf);
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const float g = grad[k] * scale;
            m[k] = __builtin_fmaf(h.b1, m[k], h.c1 * g);
            v[k] = __builtin_fmaf(h.b2, v[k], (h.c2 * g) * g);
            w[k] = adamw_weight(w[k], m[k], __builtin_amdgcn_sqrtf(v[k]), h, lr_bc1, wdf);
        }
    }
}

// A workgroup's chunk of one tensor, from element `base` on.
template <int WT, int GT, int ST>
__device__ __forceinline__ void adamw_chunk(const MtTensor &t, size_t base, const MtHyper &h, float scale)
{
    constexpr int V = WT == MT_F32 || GT == MT_F32 || ST == MT_F32 ? 4 : 8, NV = 8 / V;
    const float lr_bc1 = (float)((double)t.lr_scale * h.lr_bc1);
    const float wdf = (float)(1.0 - h.lr * (double)t.lr_scale * (double)t.wd);
    // Whether each load is waited for before the next.  Left alone, the compiler moves the first operations
    // on a value up into the branches of its load, each behind a wait of its own, for whichever types it
    // likes: 65 tensors of 4096 in fp32 take 4.7 us like that and 3.2 with all loads under way.  With bf16
    // throughout one at a time is the better for long lists, whose four streams then reach the memory in
    // longer runs (526 M elements 1236 against 1257 us, 134 M 324 against 328, 65 of 4096 3.7 against 3.0).
    constexpr bool ONE_BY_ONE = WT == MT_BF16 && GT == MT_BF16 && ST == MT_BF16;
    Share<WT, V> W[NV];
    Share<GT, V> G[NV];
    Share<ST, V> M[NV], R[NV];
    float ms[NV], vs[NV];
    size_t at[NV];
    int n[NV];                                  // elements that exist from at[j] on
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        at[j] = base + V * (j * NTH + threadIdx.x);
        n[j] = (int)max((int64_t)0, min((int64_t)V, (int64_t)t.numel - (int64_t)at[j]));
        W[j].load(t.W, at[j], n[j]);
        if (ONE_BY_ONE) W[j].arrive();
        G[j].load(t.G, at[j], n[j]);
        if (ONE_BY_ONE) G[j].arrive();
        M[j].load(t.m, at[j], n[j]);
        if (ONE_BY_ONE) M[j].arrive();
        R[j].load(t.v, at[j], n[j]);
        if constexpr (ST == MT_FP8) {
            ms[j] = n[j] ? *global_of<float>((const void *)t.ms, at[j] / MT_BLOCK) : 0.0f;
            vs[j] = n[j] ? *global_of<float>((const void *)t.vs, at[j] / MT_BLOCK) : 0.0f;
        }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        W[j].arrive();
        G[j].arrive();
        M[j].arrive();
        R[j].arrive();
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        float w[V], g[V], m[V], v[V], root[V];
        W[j].get(w);
        G[j].get(g);
        M[j].get(m);
        R[j].get(v);
        if constexpr (ST == MT_FP8) {
#pragma unroll
            for (int k = 0; k < V; ++k) {
                m[k] *= ms[j];
                v[k] *= vs[j];
                v[k] *= v[k];
            }
        }
        adamw<ST == MT_FP8>(g, scale, w, m, v, root, h, lr_bc1, wdf);
        store_some<WT>(t.W, at[j], n[j], w);
        if constexpr (ST == MT_FP8) {
            if (n[j] < V) {
#pragma unroll
                for (int k = 0; k < V; ++k)
                    if (k >= n[j]) m[k] = root[k] = 0.0f;
            }
            const float ms1 = e4m3_scale(lanes_max(mag_n(m), MT_BLOCK / V));
            const float vs1 = e4m3_scale(lanes_max(mag_n(root), MT_BLOCK / V));
            if (n[j] && at[j] % MT_BLOCK == 0) {
                *global_of<float>((void *)t.ms, at[j] / MT_BLOCK) = ms1;
                *global_of<float>((void *)t.vs, at[j] / MT_BLOCK) = vs1;
            }
            float above[V];
#pragma unroll
            for (int k = 0; k < V; ++k) above[k] = root[k] * 0x1p84f;
            e4m3_quotients(m, ms1);
            e4m3_quotients(root, vs1);
            // a sqrt(v) > 0 is not stored as zero: the middle of its quotient, the smallest code and
            // 2^84 sqrt(v), which lies above both (a scale of roots is no less than 2^-84) or is zero
#pragma unroll
            for (int k = 0; k < V; ++k) root[k] = __builtin_amdgcn_fmed3f(root[k], 0x1p-9f, above[k]);
            uint32_t cm[V / 4], cv[V / 4];
#pragma unroll
            for (int k = 0; k < V / 4; ++k) {
                cm[k] = e4m3_codes4(m + 4 * k);
                cv[k] = e4m3_codes4(root + 4 * k);
            }
            store_codes<V>(t.m, at[j], n[j], cm);
            store_codes<V>(t.v, at[j], n[j], cv);
        } else {
            store_some<ST>(t.m, at[j], n[j], m);
            store_some<ST>(t.v, at[j], n[j], v);
        }
    }
}

template <int WT, int GT>
__device__ __forceinline__ void adamw_state(const MtTensor &t, size_t base, const MtHyper &h, float scale)
{
    if (t.st == MT_F32) adamw_chunk<WT, GT, MT_F32>(t, base, h, scale);
    else if (t.st == MT_BF16) adamw_chunk<WT, GT, MT_BF16>(t, base, h, scale);
    else adamw_chunk<WT, GT, MT_FP8>(t, base, h, scale);
}

// One workgroup a chunk; what its tensor is of is the same for all of its threads.  The streams
// are non-temporal: 1202 against 1302 us on 525 M elements with bf16 throughout.  Measured
// (replayed from a graph): that 1235 to 1270 us (5.8 to 5.95 TB/s; HBM counters 4.22 GB read and 3.15 written, the
// algorithm's own), 218 M bf16 with fp8 state 367 us (6.1 TB/s; 51 vector instructions a
// wave of elements, 280 us of the vector units' time), with fp32 throughout 1080 us (5.65 TB/s); 65
// tensors of 4096 in fp32 3.2 us, which is launch and latency.
__global__ void __launch_bounds__(NTH) adamw_multi_kernel(MtTable tab, MtHyper h, const float *grad_scale)
{
    const int c = blockIdx.x;
    const MtTensor t = tab.t[tab.owner[c]];
    const float scale = grad_scale ? *grad_scale : 1.0f;
    const size_t base = (size_t)(c - t.first) * MT_CHUNK;
    if (t.wt == MT_F32) {
        if (t.gt == MT_F32) adamw_state<MT_F32, MT_F32>(t, base, h, scale);
        else adamw_state<MT_F32, MT_BF16>(t, base, h, scale);
    } else {
        if (t.gt == MT_F32) adamw_state<MT_BF16, MT_F32>(t, base, h, scale);
        else adamw_state<MT_BF16, MT_BF16>(t, base, h, scale);
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

// A chunk of gradients: where it lies, how many elements it has, of which type.
struct GradChunk {
    const void *p;
    int n;
    bool bf16;

    __device__ __forceinline__ void find(const MtTable &tab, int64_t c)
    {
        p = nullptr;
        n = 0;
        bf16 = false;
        if (c >= tab.chunks) return;
        const MtTensor &t = tab.t[tab.owner[c]];
        const int64_t base = (c - t.first) * MT_CHUNK;
        bf16 = t.gt == MT_BF16;
        p = static_cast<const char *>(t.G) + base * (bf16 ? 2 : 4);
        n = (int)min((int64_t)MT_CHUNK, t.numel - base);
    }
};
// A thread's share of it as it lies in memory: two vectors of four fp32, or one of eight bf16.
struct GradShare {
    u32x4_t r[2];

    __device__ __forceinline__ void load(const GradChunk &g)
    {
        r[0] = r[1] = u32x4_t{0, 0, 0, 0};
        if (g.bf16) {
            const int at = 8 * threadIdx.x;
            if (at + 8 <= g.n) r[0] = load_v<u32x4_t, uint16_t, false>(g.p, at);
            else
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (at + k < g.n) r[0][k >> 1] |= (uint32_t)*global_of<uint16_t>(g.p, at + k) << (16 * (k & 1));
        } else {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int at = 4 * (j * NTH + (int)threadIdx.x);
                if (at + 4 <= g.n) r[j] = load_v<u32x4_t, uint32_t, false>(g.p, at);
                else
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (at + k < g.n) r[j][k] = *global_of<uint32_t>(g.p, at + k);
            }
        }
    }
    // Its squares, in fp64.
    __device__ __forceinline__ double add_to(double sum, bool bf16) const
    {
        if (bf16) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const double a = (double)bf_lo(r[0][k]), b = (double)bf_hi(r[0][k]);
                sum = __builtin_fma(b, b, __builtin_fma(a, a, sum));
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const double a = (double)__uint_as_float(r[k >> 2][k & 3]);
                sum = __builtin_fma(a, a, sum);
            }
        }
        return sum;
    }
};

// The squares of N neighbouring chunks at a time, from N blockIdx.x on, N gridDim.x apart:
// neighbouring workgroups read neighbouring chunks (a run of 52 chunks for each: 97 against 84 us
// on 218 M bf16).  The next chunks are looked up in the table while the loads of these are in
// flight (80 us).  The loads are plain, although non-temporal ones take 5 % less alone: the step
// that follows reads the gradients again, and what the caches keep of them counts for more (norm
// and step on 100 M bf16 252 against 275 us).  N = 4 from 2^18 chunks on, where it leaves the
// memory longer runs and measured faster (2 G bf16 680 against 750 us, 1 G 342 against 356, 500 M
// 175.6 against 176.6, 1 G fp32 712 against 730); below, the fewer waves with something to read
// cost more (100 M bf16 42.4 against 39.8, 218 M 81.3 against 79.2).  Measured (replayed from a
// graph, with the finish): 218 M bf16 77 us (5.7 TB/s), fp32 148 us (5.9 TB/s), 65 tensors of 4096
// in fp32 4.3 us.
template <int N> __device__ __forceinline__ double grad_squares(const MtTable &tab)
{
    const int64_t stride = (int64_t)N * gridDim.x;
    double sum = 0.0;
    GradChunk now[N];
#pragma unroll
    for (int k = 0; k < N; ++k) now[k].find(tab, (int64_t)N * blockIdx.x + k);
    for (int64_t c = (int64_t)N * blockIdx.x; c < tab.chunks; c += stride) {
        GradShare g[N];
        bool bf16[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            g[k].load(now[k]);
            bf16[k] = now[k].bf16;
        }
#pragma unroll
        for (int k = 0; k < N; ++k) now[k].find(tab, c + stride + k);
#pragma unroll
        for (int k = 0; k < N; ++k) sum = g[k].add_to(sum, bf16[k]);
    }
    return sum;
}
constexpr int64_t NORM_LONG = int64_t(1) << 18;

template <int N> __global__ void __launch_bounds__(NTH) grad_norm_kernel(MtTable tab, double *part)
{
    __shared__ double red[NTH / 64];
    const double sum = group_sum(grad_squares<N>(tab), red);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

__device__ __forceinline__ void put_norm(double sum, float max_norm, float *out)
{
    if (threadIdx.x == 0) {
        const double norm = sqrt(sum), c = (double)max_norm / (norm + 1e-6);
        out[0] = (float)norm;
        out[1] = c > 1.0 ? 1.0f : (float)c;      // a NaN stays one
    }
}

// The parts' sum, eight of a thread's in flight.
__global__ void __launch_bounds__(NTH) grad_norm_finish_kernel(const double *part, int parts, float max_norm, float *out)
{
    __shared__ double red[NTH / 64];
    static_assert(MT_NORM_PARTS == 8 * NTH, "a thread sums eight parts");
    double x[8], sum = 0.0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int p = k * NTH + threadIdx.x;
        x[k] = p < parts ? part[p] : 0.0;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += x[k];
    put_norm(group_sum(sum, red), max_norm, out);
}

// A list of up to NORM_SHORT chunks in one workgroup and one launch: 5.6 against 9.2 us a call, and
// 4.5 against 4.6 replayed from a graph (16 chunks: 7.3 against 4.5 there).
constexpr int64_t NORM_SHORT = 8;
__global__ void __launch_bounds__(NTH) grad_norm_short_kernel(MtTable tab, float max_norm, float *out)
{
    __shared__ double red[NTH / 64];
    put_norm(group_sum(grad_squares<4>(tab), red), max_norm, out);
}

}  // namespace

hipError_t launch_grad_norm(const MtTable &t, float max_norm, float *out, double *part, hipStream_t stream)
{
    if (t.chunks <= NORM_SHORT) {
        grad_norm_short_kernel<<<1, NTH, 0, stream>>>(t, max_norm, out);
        return hipGetLastError();
    }
    const int parts = (int)(t.chunks < MT_NORM_PARTS ? t.chunks : MT_NORM_PARTS);
    if (t.chunks >= NORM_LONG) grad_norm_kernel<4><<<parts, NTH, 0, stream>>>(t, part);
    else grad_norm_kernel<1><<<parts, NTH, 0, stream>>>(t, part);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    grad_norm_finish_kernel<<<1, NTH, 0, stream>>>(part, parts, max_norm, out);
    return hipGetLastError();
}

hipError_t launch_adamw_multi(const MtTable &t, const MtHyper &h, const float *grad_scale, hipStream_t stream)
{
    adamw_multi_kernel<<<(unsigned)t.chunks, NTH, 0, stream>>>(t, h, grad_scale);
    return hipGetLastError();
}

}  // namespace forge_impl
