// Internal interface between forge_ops_api.cpp and the kernels of forge_norm.hip and
// forge_multi.hip.  Not installed; callers use include/forge_ops.h.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace forge_impl {

// ------------------------------------------------------------------------ RMS norm

struct NormArgs {
    const void *x;         // bf16 [T, d] with a residual, else the stream
    const void *r;         // residual, or null
    const void *w;         // [d]
    void *h;               // the stored sum (with a residual)
    uint16_t *y;           // bf16 output, or null
    uint8_t *q;            // fp8 output, or null
    float *qs;
    int T, d;
    int h_bf16, w_bf16;    // element types: bf16 or fp32
    int q_group;           // columns per scale; 0: the row
    float eps;
};

struct NormGradArgs {
    const uint16_t *dy;
    const void *h, *w;
    const void *dres;      // or null
    void *dh;              // or null
    uint16_t *dx;          // or null
    float *dw;
    float *part;           // [norm_grad_plan(T, d).groups, d]
    int T, d;
    int h_bf16, w_bf16;
    float eps;
};

hipError_t launch_rmsnorm(const NormArgs &a, hipStream_t stream);
// T == 0 fills dw with zeros.
hipError_t launch_rmsnorm_backward(const NormGradArgs &a, hipStream_t stream);

// Columns of the widest row that the registers of a workgroup hold.
constexpr int64_t NORM_WIDEST = 32768, GRAD_WIDEST = 16384;
// Inputs of the gradient (dy, h, and dres where it is given) beyond this many bytes are read
// non-temporally: what the L2s of eight XCDs hold together.  Below, what the kernel before has just
// written is found there: over two sets of inputs in turn 512 x 4096 bf16 takes 9.2 us plainly and
// 9.7 non-temporally, 1300 x 4096 12.4 and 15.4, without dres 1400 x 4096 11.9 and 13.8.  Inputs
// that no cache holds (sixteen sets in turn) are the faster non-temporally: 9.8 and 9.2, 14.2 and
// 13.6.
constexpr int64_t GRAD_CACHED = int64_t(32) << 20;
inline bool norm_grad_streams(int64_t T, int64_t d, bool h_bf16, bool dres)
{
    return T * d * (2 + (h_bf16 ? 2 : 4) * (dres ? 2 : 1)) > GRAD_CACHED;
}

// A launch over T rows: workgroups, and threads of each.
struct NormPlan {
    int groups, threads;
};
// Rows that a wave holds at once: a lane has eight elements at least, a row eight lanes.
inline int rows_per_wave(int64_t d) { return d <= 64 ? 8 : d <= 128 ? 4 : d <= 256 ? 2 : 1; }
inline NormPlan norm_plan(int64_t T, int64_t d)
{
    // Workgroups take a second row once there are more than this: rows of a wave sooner, whose
    // start costs more beside them (30000 x 512: 25.7 against 27.2 us), than rows of several
    // (16384 x 4096: 96.8 us at 8192 workgroups, 101.6 at 2048, 95.6 without a limit, which in
    // turn loses 2 % at 16384 x 8192).
    const int64_t per = d > 1024 ? 1 : d > 512 ? 2 : 4 * rows_per_wave(d), n = (T + per - 1) / per;
    const int64_t most = d > 512 ? 8192 : 2048;
    return {(int)(n < most ? n : most), d > 8192 ? 1024 : 256};
}
// The gradient's workgroups each leave a row of partial sums of dw, written and read again beside
// the rows' own bytes: one for each CU, two where that is no more than a row for four of the
// input, and as many rows at once in each as there are for all.
inline NormPlan norm_grad_plan(int64_t T, int64_t d)
{
    if (d > GRAD_WIDEST) return {(int)(T < 512 ? T : 512), 256};
    const int64_t waves = d <= 512 ? 1 : d <= 1024 ? 2 : d <= 2048 ? 4 : d <= 4096 ? 8 : 16;   // of a row
    int64_t rows = 1;
    // Up to four turns of one workgroup, whose sum is dw itself, save the second kernel and its
    // launch: a call takes 8.1 against 11.5 us at 4 x 4096 bf16 and 8.1 against 11.6 at 64 x 256.
    // Replayed from a graph, where launches cost less, it is 4.2 against 4.8 us at 4 x 4096 and 4.6
    // against 4.7 at 48 x 256, but 5.2 against 4.7 at 64 x 256, four turns of rows that share a wave
    // (eight turns: 8 x 4096 7.8 against 5.2, 8 x 16384 19.9 against 7.5).
    const bool few = T <= 4 * (waves < 8 ? 8 / waves : 1) * rows_per_wave(d);
    while (waves * rows < 8 && T > (few ? 1 : 256) * rows * rows_per_wave(d)) rows *= 2;
    const int64_t per = rows * rows_per_wave(d), n = (T + per - 1) / per;
    const int64_t most = few ? 1 : waves < 16 && T >= 2048 ? 512 : 256;
    return {(int)(n < most ? n : most), (int)(64 * waves * rows)};
}

// ------------------------------------------------------------------------ many tensors

// Elements of a chunk, the work of one workgroup's pass; a multiple of the 64 elements that
// share an fp8 scale.
constexpr int MT_CHUNK = 2048;
constexpr int MT_BLOCK = 64;
// Chunks of a list: a launch has fewer than 2^32 threads.
constexpr int64_t MT_MAX_CHUNKS = (int64_t(1) << 24) - 1;
// Workgroups of the gradient norm, each leaving one partial sum.
constexpr int MT_NORM_PARTS = 2048;

enum MtType { MT_F32 = 0, MT_BF16 = 1, MT_FP8 = 2 };

// A tensor as the kernels read it from the table.
struct alignas(16) MtTensor {
    void *W;
    const void *G;
    void *m, *v;
    float *ms, *vs;
    int32_t numel, first;  // elements; number of its first chunk
    float lr_scale, wd;
    int32_t wt, gt, st;    // MtType of weight, gradient, state
    int32_t pad;
};

// The table: n tensors, then for each chunk the tensor that it belongs to.
struct MtTable {
    const MtTensor *t;
    const int32_t *owner;
    int64_t chunks;
};

struct MtHyper {
    float b1, c1, b2, c2;  // betas and 1 - betas
    float inv_sqrt_bc2, eps;
    double lr, lr_bc1;     // lr, lr / (1 - beta1^t): scaled per tensor, then rounded to fp32
};

hipError_t launch_grad_norm(const MtTable &t, float max_norm, float *out, double *part, hipStream_t stream);
hipError_t launch_adamw_multi(const MtTable &t, const MtHyper &h, const float *grad_scale, hipStream_t stream);

}  // namespace forge_impl
