// forge_norm.hip -- residual add and RMS norm, forward and backward (include/forge_ops.h).
//
// Both directions are bound by HBM (a few operations per element): a row stays in registers
// between its sums and its outputs, so that every input is read once and every output written
// once; rows of more than 32768 columns (the gradient: 16384) are read again instead.  (The
// gradient of an fp32 stream between 8192 and 16384 columns keeps 10 to 12 registers of 128 in
// scratch: 4096 x 16384 184 us, 5.1 TB/s, and 107 us, 5.0 TB/s, in bf16, which spills none.)
// A row belongs to WR waves, which join their sums through LDS; rows of up to 512 columns
// to one wave or a part of one, 8, 16 or 32 lanes, and join by lane exchanges alone.  A thread
// holds few elements of a row (E) rather than a wave the whole of it: more waves are in flight
// for the same registers, and a single row is spread over more loads.  One wave for up to 4096
// columns (E = 64) measured 7.7 us at 512 x 4096 and 4.3 us at 1 x 4096, four waves of E = 16
// 4.7 and 2.4 us; at 16384 x 4096 107 against 97 us.
#include "forge_ops_device.h"
#include "forge_ops_internal.h"

#include <algorithm>
#include <type_traits>

namespace forge_impl {

namespace {

// A thread's part of a row: E elements in vectors of V, the vectors of a row dealt out to its
// lanes in turn, so that each access of a wave is one dense run.  V is what makes every type's
// access dense at 16 bytes at most: 8 with a bf16 stream, 4 with an fp32 one.
template <bool HB, int E, int WR> struct Row {
    static constexpr int V = HB ? 8 : 4, NV = E / V;
    int lane, lanes;       // of this row: the thread's place and how many there are
    int slot, slots;       // the row's place among those that the workgroup holds at once
    int nv;                // vectors of a row

    __device__ __forceinline__ Row(int d)
    {
        nv = d / V;
        lanes = 64 * WR;
        if (WR == 1)
            while (lanes > 8 && lanes * E >= 2 * d) lanes >>= 1;
        lane = threadIdx.x & (lanes - 1);
        slot = threadIdx.x / lanes;
        slots = blockDim.x / lanes;
    }
    __device__ __forceinline__ int vec(int j) const { return j * lanes + lane; }
    __device__ __forceinline__ bool has(int j) const { return vec(j) < nv; }
};

// Sums over a row: lane exchanges, and for rows of several waves one trip through LDS.  `red`
// holds 2 * 2 * 16 values, used in turn by rows of even and odd `turn`, so that one barrier a
// row is enough.
template <int WR, int N, class R>
__device__ __forceinline__ void row_sum(float (&x)[N], const R &row, float (*red)[2][16], int turn)
{
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = lanes_sum(x[k], WR == 1 ? row.lanes : 64);
    if constexpr (WR > 1) {
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int k = 0; k < N; ++k) red[turn & 1][k][threadIdx.x >> 6] = x[k];
        }
        lds_barrier();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            x[k] = 0.0f;
#pragma unroll
            for (int i = 0; i < WR; ++i) x[k] += red[turn & 1][k][row.slot * WR + i];
        }
    }
}

// h = round(r + x), y = h / sqrt(mean(h^2) + eps) w, and the codes of the fp32 y.
//
// Of the outputs only h is stored non-temporally: y and q are read by the product that follows,
// h not before the layer's end.  A norm and a 4096 x 4096 product of its output at 2048 tokens
// take 78 us like this, 80 with all outputs non-temporal (which alone is faster, 12.8 against
// 15.7 us), at 8192 tokens 226 and 229.5.
//
// Measured (replayed from a graph): 1 x 4096 bf16 2.4 us, 512 x 4096 4.7 us, 16384 x 4096 97 us
// (5.55 TB/s), 16384 x 8192 fp32 with fp8 output 266 us (5.6 TB/s; a large copy 4.9 to 5.4).
// HBM counters at the latter: 808 MB read, 675 written, the algorithm's own 805 and 675.
template <bool HB, bool WB, int E, int WR>
__global__ void __launch_bounds__(WR == 16 ? 1024 : 256) norm_kernel(NormArgs a)
{
    using R = Row<HB, E, WR>;
    constexpr int V = R::V, NV = R::NV;
    __shared__ float red[2][2][16];
    __shared__ uint32_t redm[2][16];
    const R row(a.d);
    const float inv_d = 1.0f / a.d;
    const int stride = gridDim.x * row.slots, groups = (a.d + 127) >> 7;
    // every wave runs as many turns as the first, rows past the end empty: lane exchanges and
    // barriers need all of them
    int turn = 0;
    for (int t0 = blockIdx.x * row.slots; t0 < a.T; t0 += stride, ++turn) {
        const int t = t0 + row.slot;
        const bool live = t < a.T;
        const size_t at = (size_t)t * a.d;
        float f[NV][V], sum[1] = {0.0f};
        {
            Raw<HB, V> r[NV];
            if (a.r) {
                Raw<true, V> x[NV];
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    x[j].zero();
                    r[j].zero();
                    if (live && row.has(j)) {
                        x[j].load(a.x, at + V * row.vec(j));
                        r[j].load(a.r, at + V * row.vec(j));
                    }
                }
#pragma unroll
                for (int j = 0; j < NV; ++j) {
#pragma unroll
                    for (int k = 0; k < V; ++k) f[j][k] = r[j].at(k) + x[j].at(k);
                    r[j].set(f[j]);
                    if (live && row.has(j)) r[j].template store<true>(a.h, at + V * row.vec(j));
                }
            } else {
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    r[j].zero();
                    if (live && row.has(j)) r[j].load(a.x, at + V * row.vec(j));
                }
            }
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    f[j][k] = r[j].at(k);                      // the sum as it is stored
                    sum[0] = __builtin_fmaf(f[j][k], f[j][k], sum[0]);
                }
        }
        row_sum<WR, 1>(sum, row, red, turn);
        const float s = __builtin_amdgcn_rsqf(__builtin_fmaf(sum[0], inv_d, a.eps));
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (!row.has(j)) continue;
            float w[V];
            load_n<WB>(a.w, V * row.vec(j), w);
#pragma unroll
            for (int k = 0; k < V; ++k) f[j][k] = f[j][k] * s * w[k];
            if (live && a.y) store_n<true>(a.y, at + V * row.vec(j), f[j]);
            top = max(top, mag_n(f[j]));
        }
        if (!a.q) continue;
        float qs = 0.0f;
        if (a.q_group == 0) {
            top = lanes_max(top, WR == 1 ? row.lanes : 64);
            if constexpr (WR > 1) {
                if ((threadIdx.x & 63) == 0) redm[turn & 1][threadIdx.x >> 6] = top;
                lds_barrier();
#pragma unroll
                for (int i = 0; i < WR; ++i) top = max(top, redm[turn & 1][row.slot * WR + i]);
            }
            qs = e4m3_scale(top);
            if (live && row.lane == 0) a.qs[t] = qs;
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (a.q_group) {
                // 128 columns are 128 / V lanes (the launcher gives a row of up to 128 one scale)
                qs = e4m3_scale(lanes_max(row.has(j) ? mag_n(f[j]) : 0u, 128 / V));
                if (live && row.has(j) && row.vec(j) % (128 / V) == 0)
                    a.qs[(size_t)t * groups + row.vec(j) / (128 / V)] = qs;
            }
            if (!live || !row.has(j)) continue;
            e4m3_quotients(f[j], qs);
            uint32_t *q = reinterpret_cast<uint32_t *>(a.q + at + V * row.vec(j));
            if constexpr (V == 8) {
                const u32x2_t c = {e4m3_codes4(f[j]), e4m3_codes4(f[j] + 4)};
                *reinterpret_cast<u32x2_t *>(q) = c;
            } else {
                *q = e4m3_codes4(f[j]);
            }
        }
    }
}

// With s = 1 / sqrt(mean(h^2) + eps): dh = dres + s (dy w - h s^2 mean(dy w h)), dw = sum of
// dy h s over the rows.  s is formed again from h, which is read anyway.
//
// Each workgroup takes its rows in turn: dh and dx of each, and their share of dw in registers,
// which it leaves in its row of the workspace, summed by norm_dw_kernel in an order that the
// sizes fix.  The next rows' h and dy are loaded ahead of the sums of these, so that loads are in
// flight across the barrier (which waits for LDS only).  dres is not: those registers would take
// a quarter of the waves.  E = 8 with up to 16 waves a row takes 75 VGPRs (fp32: 90),
// E = 16 with half the waves 107 (128, and 8 to 10 spilled).  At 8192 columns E = 8 is the faster
// (bf16, 4096 rows 54 against 55 us, 16384 rows 195 against 199), at 4096 it is not (2048 rows 20.1
// against 18.4, 16384 rows 103 against 97).
//
// Inputs beyond what the L2s hold (norm_grad_streams) are read non-temporally: 103 against 108 us
// at 16384 x 4096 and 20.2 against 21.1 us at 2048 x 4096.  dh and dx
// are stored plainly for the product that follows: 4096 x 4096 products before and after this
// kernel and it at 2048 tokens take 135 us, 142 with non-temporal stores.
//
// Measured (replayed from a graph, both kernels, on inputs that no cache holds): 512 x 4096 bf16
// 9.7 us, of which 3.3 are norm_dw_kernel; 16384 x 4096 bf16 103 us (5.2 TB/s), fp32 with dh and dx
// 203 us (5.3 TB/s).
// HBM counters at 16384 x 4096 bf16: 403 MB read and 143 written, the algorithm's own 403 and 134
// and the parts' 8.
template <bool HB, bool NT, int E, int WR> struct GradRow {
    static constexpr int V = Row<HB, E, WR>::V, NV = Row<HB, E, WR>::NV;
    Raw<HB, V> h[NV];
    Raw<true, V> g[NV];
    __device__ __forceinline__ void load(const NormGradArgs &a, const Row<HB, E, WR> &row, int t)
    {
        const size_t at = (size_t)t * a.d;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            h[j].zero();
            g[j].zero();
            if (t >= a.T || !row.has(j)) continue;
            h[j].template load<NT>(a.h, at + V * row.vec(j));
            g[j].template load<NT>(a.dy, at + V * row.vec(j));
        }
    }
};

template <bool HB, bool WB, bool NT, int E, int WR>
__global__ void __launch_bounds__(WR == 16 ? 1024 : 512, 4) norm_grad_kernel(NormGradArgs a)
{
    using R = Row<HB, E, WR>;
    constexpr int V = R::V, NV = R::NV;
    __shared__ float red[2][2][16];
    __shared__ f32x4_t share[WR == 16 ? 1 : 16 * WR * E];
    const R row(a.d);
    const float inv_d = 1.0f / a.d;
    const int stride = gridDim.x * row.slots;
    float acc[NV][V];
    Raw<WB, V> w[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        w[j].zero();
        if (row.has(j)) w[j].load(a.w, V * row.vec(j));
#pragma unroll
        for (int k = 0; k < V; ++k) acc[j][k] = 0.0f;
    }
    GradRow<HB, NT, E, WR> now, next;
    now.load(a, row, blockIdx.x * row.slots + row.slot);
    int turn = 0;
    for (int t0 = blockIdx.x * row.slots; t0 < a.T; t0 += stride, ++turn) {
        const int t = t0 + row.slot;
        const size_t at = (size_t)t * a.d;
        Raw<HB, V> o[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            o[j].zero();
            if (a.dres && t < a.T && row.has(j)) o[j].template load<NT>(a.dres, at + V * row.vec(j));
        }
        next.load(a, row, t < a.T - stride ? t + stride : a.T);
        float sum[2] = {0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int k = 0; k < V; ++k) {
                sum[0] = __builtin_fmaf(now.h[j].at(k), now.h[j].at(k), sum[0]);
                sum[1] = __builtin_fmaf(now.g[j].at(k) * w[j].at(k), now.h[j].at(k), sum[1]);
            }
        row_sum<WR, 2>(sum, row, red, turn);
        const float s = __builtin_amdgcn_rsqf(__builtin_fmaf(sum[0], inv_d, a.eps));
        const float c = s * s * (sum[1] * inv_d);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            now.h[j].forget();
            now.g[j].forget();
            float x[V];
#pragma unroll
            for (int k = 0; k < V; ++k) {
                x[k] = __builtin_fmaf(s, __builtin_fmaf(-now.h[j].at(k), c, now.g[j].at(k) * w[j].at(k)), o[j].at(k));
                acc[j][k] = __builtin_fmaf(now.g[j].at(k), now.h[j].at(k) * s, acc[j][k]);
            }
            if (t >= a.T || !row.has(j)) continue;
            if (a.dh) store_n<HB>(a.dh, at + V * row.vec(j), x);
            if (a.dx) store_n<true>(a.dx, at + V * row.vec(j), x);
        }
        now = next;
    }
    float *part = a.part + (size_t)blockIdx.x * a.d;
    if constexpr (WR == 1) {
        // the rows that share a wave
        for (int o = row.lanes; o < 64; o <<= 1)
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int k = 0; k < V; ++k) acc[j][k] += __shfl_xor(acc[j][k], o);
    }
    if constexpr (WR < 16) {
        // the waves that held the same columns, one after the other
        const int mine = (threadIdx.x >> 6) / WR, all = (blockDim.x >> 6) / WR;
        const bool writes = WR > 1 || (int)(threadIdx.x & 63) < row.lanes;
        for (int i = 0; i < all; ++i) {
            if (mine == i && writes) {
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    if (!row.has(j)) continue;
                    f32x4_t *x = share + V / 4 * row.vec(j), y[V / 4];
                    if (i) {
#pragma unroll
                        for (int k = 0; k < V / 4; ++k) y[k] = x[k];
#pragma unroll
                        for (int k = 0; k < V; ++k) acc[j][k] += y[k >> 2][k & 3];
                    }
                    if (i + 1 < all) {
#pragma unroll
                        for (int k = 0; k < V; ++k) y[k >> 2][k & 3] = acc[j][k];
#pragma unroll
                        for (int k = 0; k < V / 4; ++k) x[k] = y[k];
                    } else {
                        store_n<false>(part, V * row.vec(j), acc[j]);
                    }
                }
            }
            lds_barrier();
        }
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (row.has(j)) store_n<false>(part, V * row.vec(j), acc[j]);
    }
}

// dw: the parts' sum.  A workgroup takes 32 columns (a line of each part), eight threads of four
// columns by 32 runs of parts, eight parts of a run in flight, joined through LDS in the runs'
// order.  Bound by latency: 512 parts of 4096 columns 4.9 us, 256 of them 3.3; with 64 columns
// and 16 runs to a workgroup, one part in flight each, 13.7 us.
constexpr int DW_COLS = 32, DW_RUNS = 32;
// Columns of one launch, which must have fewer than 2^32 threads: two rows can be 2^30 columns wide,
// and dw of no tokens any width.
constexpr int DW_LAUNCH = 1 << 28;
static_assert(int64_t(DW_LAUNCH) / DW_COLS * (DW_RUNS * 8) < (int64_t(1) << 32), "threads of a launch");

// Columns 0 .. cols - 1 of dw and of the parts, whose rows are d apart.
__global__ void __launch_bounds__(DW_RUNS * 8) norm_dw_kernel(const float *part, float *dw, int parts, int d, int cols)
{
    __shared__ f32x4_t red[DW_RUNS][8];
    const int c = threadIdx.x & 7, r = threadIdx.x >> 3, j = blockIdx.x * DW_COLS + 4 * c;
    f32x4_t x = {0, 0, 0, 0};
    if (j < cols)
        for (int p0 = r; p0 < parts; p0 += 8 * DW_RUNS) {
            f32x4_t y[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int p = p0 + k * DW_RUNS;
                y[k] = f32x4_t{0, 0, 0, 0};
                if (p < parts) y[k] = *reinterpret_cast<const f32x4_t *>(part + (size_t)p * d + j);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) x += y[k];
        }
    red[r][c] = x;
    __syncthreads();
    if (r || j >= cols) return;
#pragma unroll
    for (int k = 1; k < DW_RUNS; ++k) x += red[k][c];
    *reinterpret_cast<f32x4_t *>(dw + j) = x;
}

// Rows wider than registers hold: the row is read again for the outputs, and once more before them
// for the maximum of a scale per row; the gradient's dw is summed in the workspace, whose row is read
// and written for every row but a workgroup's first.  Measured: 1024 x 65536 bf16 136 us (4.0 TB/s
// of the bytes that it cannot do without), with fp8 output and a scale per row 130 us (3.6); the
// gradient of 1024 x 32768 123 us (2.2), of 4096 x 32768 452 us (2.4).
constexpr int NTH = 256;

__device__ __forceinline__ float wide_sum(float x, float *red)
{
    x = lanes_sum(x, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.0f;
#pragma unroll
    for (int k = 0; k < NTH / 64; ++k) x += red[k];
    return x;
}

// A workgroup a row.
template <bool HB, bool WB>
__global__ void __launch_bounds__(NTH) norm_wide_kernel(NormArgs a)
{
    __shared__ float red[NTH / 64];
    __shared__ uint32_t redm[NTH / 64];
    const int nv = a.d >> 3, groups = ((a.d - 1) >> 7) + 1;
    const void *src = a.r ? a.h : a.x;
    const int t = blockIdx.x;
    const size_t row = (size_t)t * a.d;
    float sum = 0.0f;
    for (int v = threadIdx.x; v < nv; v += NTH) {
        const size_t i = row + 8 * v;
        float f[8];
        if (a.r) {
            float x[8];
            load_n<true>(a.x, i, x);
            load_n<HB>(a.r, i, f);
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] = as_stored<HB>(f[k] + x[k]);
            store_n<HB>(a.h, i, f);
        } else {
            load_n<HB>(a.x, i, f);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) sum = __builtin_fmaf(f[k], f[k], sum);
    }
    const float s = __builtin_amdgcn_rsqf(wide_sum(sum, red) / a.d + a.eps);
    auto out8 = [&](int v, float (&f)[8]) {
        float w[8];
        load_n<HB>(src, row + 8 * v, f);
        load_n<WB>(a.w, 8 * v, w);
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = f[k] * s * w[k];
    };
    float qs = 0.0f;
    if (a.q && a.q_group == 0) {
        uint32_t top = 0;
        for (int v = threadIdx.x; v < nv; v += NTH) {
            float f[8];
            out8(v, f);
            top = max(top, mag_n(f));
        }
        top = lanes_max(top, 64);
        if ((threadIdx.x & 63) == 0) redm[threadIdx.x >> 6] = top;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NTH / 64; ++k) top = max(top, redm[k]);
        qs = e4m3_scale(top);
        if (threadIdx.x == 0) a.qs[t] = qs;
    }
    for (int v = threadIdx.x; v < (nv + 63) / 64 * 64; v += NTH) {     // whole waves
        float f[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (v < nv) out8(v, f);
        if (a.q && a.q_group) {
            qs = e4m3_scale(lanes_max(mag_n(f), 16));
            if (v < nv && (v & 15) == 0) a.qs[(size_t)t * groups + (v >> 4)] = qs;
        }
        if (v >= nv) continue;
        if (a.y) store_n<true>(a.y, row + 8 * v, f);
        if (a.q) {
            e4m3_quotients(f, qs);
            const u32x2_t c = {e4m3_codes4(f), e4m3_codes4(f + 4)};
            *reinterpret_cast<u32x2_t *>(a.q + row + 8 * v) = c;
        }
    }
}

template <bool HB, bool WB>
__global__ void __launch_bounds__(NTH) norm_grad_wide_kernel(NormGradArgs a)
{
    __shared__ float red[2][NTH / 64];
    const int nv = a.d >> 3;
    float *part = a.part + (size_t)blockIdx.x * a.d;
    for (int t = blockIdx.x, first = 1; t < a.T; t += gridDim.x, first = 0) {
        const size_t row = (size_t)t * a.d;
        float s1 = 0.0f, s2 = 0.0f;
        auto in8 = [&](int v, float (&h)[8], float (&g)[8], float (&w)[8]) {
            load_n<HB>(a.h, row + 8 * v, h);
            load_n<true>(a.dy, row + 8 * v, g);
            load_n<WB>(a.w, 8 * v, w);
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
        s1 = wide_sum(s1, red[0]);
        s2 = wide_sum(s2, red[1]);
        const float s = __builtin_amdgcn_rsqf(s1 / a.d + a.eps);
        const float c = s * s * (s2 / a.d);
        for (int v = threadIdx.x; v < nv; v += NTH) {
            float h[8], g[8], w[8], o[8] = {0, 0, 0, 0, 0, 0, 0, 0}, p[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            in8(v, h, g, w);
            if (a.dres) load_n<HB>(a.dres, row + 8 * v, o);
            if (!first) load_n<false>(part, 8 * v, p);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                o[k] = __builtin_fmaf(s, __builtin_fmaf(-h[k], c, g[k] * w[k]), o[k]);
                p[k] = __builtin_fmaf(g[k], h[k] * s, p[k]);
            }
            if (a.dh) store_n<HB>(a.dh, row + 8 * v, o);
            if (a.dx) store_n<true>(a.dx, row + 8 * v, o);
            store_n<false>(part, 8 * v, p);
        }
    }
}

template <int N> using Int = std::integral_constant<int, N>;

// f(E, WR): the elements that a thread holds of a row of d columns and the waves of the row.
template <class F> void norm_width(int64_t d, F f)
{
    if (d <= 512) f(Int<8>(), Int<1>());
    else if (d <= 1024) f(Int<8>(), Int<2>());
    else if (d <= 2048) f(Int<8>(), Int<4>());
    else if (d <= 4096) f(Int<16>(), Int<4>());
    else if (d <= 8192) f(Int<32>(), Int<4>());
    else if (d <= 16384) f(Int<16>(), Int<16>());
    else f(Int<32>(), Int<16>());
}
template <class F> void grad_width(int64_t d, F f)
{
    if (d <= 512) f(Int<8>(), Int<1>());
    else if (d <= 1024) f(Int<8>(), Int<2>());
    else if (d <= 2048) f(Int<8>(), Int<4>());
    else if (d <= 4096) f(Int<8>(), Int<8>());
    else if (d <= 8192) f(Int<8>(), Int<16>());
    else f(Int<16>(), Int<16>());
}

template <bool HB, bool WB> void run_norm(const NormArgs &a, hipStream_t stream)
{
    if (a.d > NORM_WIDEST) {
        norm_wide_kernel<HB, WB><<<a.T, NTH, 0, stream>>>(a);      // fewer than 2^16 rows
        return;
    }
    norm_width(a.d, [&](auto e, auto wr) {
        constexpr int E = decltype(e)::value, WR = decltype(wr)::value;
        const NormPlan p = norm_plan(a.T, a.d);
        norm_kernel<HB, WB, E, WR><<<p.groups, p.threads, 0, stream>>>(a);
    });
}

template <bool HB, bool WB> void run_grad(const NormGradArgs &a, int parts, hipStream_t stream)
{
    if (a.d > GRAD_WIDEST) {
        norm_grad_wide_kernel<HB, WB><<<parts, NTH, 0, stream>>>(a);
        return;
    }
    grad_width(a.d, [&](auto e, auto wr) {
        constexpr int E = decltype(e)::value, WR = decltype(wr)::value;
        const int threads = norm_grad_plan(a.T, a.d).threads;
        if (norm_grad_streams(a.T, a.d, HB, a.dres != nullptr)) norm_grad_kernel<HB, WB, true, E, WR><<<parts, threads, 0, stream>>>(a);
        else norm_grad_kernel<HB, WB, false, E, WR><<<parts, threads, 0, stream>>>(a);
    });
}

}  // namespace

hipError_t launch_rmsnorm(const NormArgs &args, hipStream_t stream)
{
    NormArgs a = args;
    if (a.d <= 128) a.q_group = 0;                            // one group is the row
    if (a.h_bf16) a.w_bf16 ? run_norm<true, true>(a, stream) : run_norm<true, false>(a, stream);
    else a.w_bf16 ? run_norm<false, true>(a, stream) : run_norm<false, false>(a, stream);
    return hipGetLastError();
}

hipError_t launch_rmsnorm_backward(const NormGradArgs &args, hipStream_t stream)
{
    NormGradArgs a = args;
    const int parts = norm_grad_plan(a.T, a.d).groups;
    if (parts == 1) a.part = a.dw;
    if (parts > 0) {
        if (a.h_bf16) a.w_bf16 ? run_grad<true, true>(a, parts, stream) : run_grad<true, false>(a, parts, stream);
        else a.w_bf16 ? run_grad<false, true>(a, parts, stream) : run_grad<false, false>(a, parts, stream);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (parts == 1) return hipSuccess;                        // its part is dw
    for (int64_t j = 0; j < a.d; j += DW_LAUNCH) {
        const int cols = (int)std::min<int64_t>(a.d - j, DW_LAUNCH);
        norm_dw_kernel<<<(cols + DW_COLS - 1) / DW_COLS, DW_RUNS * 8, 0, stream>>>(a.part + j, a.dw + j, parts, a.d, cols);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace forge_impl
