// forge_ops_api.cpp -- the C ABI declared in include/forge_ops.h: argument validation (host
// only, before any HIP call), the per-call scalars in fp64, the layout of a tensor list, and
// the kernel launches.
#include <algorithm>
#include <limits>
#include <new>

#include "forge_checks.h"
#include "forge_ops.h"
#include "forge_ops_internal.h"

using namespace forge_impl;

static_assert(int(FORGE_DTYPE_F32) == int(MT_F32) && int(FORGE_DTYPE_BF16) == int(MT_BF16) &&
                  int(FORGE_DTYPE_FP8) == int(MT_FP8),
              "type codes of the ABI and the kernels");
static_assert(FORGE_STATE_BLOCK == MT_BLOCK, "fp8 state block of the ABI and the kernels");

namespace {

bool is_float(int32_t t) { return t == FORGE_DTYPE_F32 || t == FORGE_DTYPE_BF16; }

int64_t bytes_of(int32_t t) { return t == FORGE_DTYPE_F32 ? 4 : t == FORGE_DTYPE_BF16 ? 2 : 1; }

bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// The tensors of a norm: T >= 0 rows of d columns, d in steps of 8, below 2^31 elements.
forge_status check_rows(int64_t T, int64_t d)
{
    if (T < 0 || d < 0) return FORGE_ERR_INVALID_SHAPE;
    if (d % 8 != 0 || T > kMaxElems || d > kMaxElems || T * d > kMaxElems) return FORGE_ERR_UNSUPPORTED_SHAPE;
    return FORGE_OK;
}

// eps > 0, and no subnormal number: the hardware takes those for zero in reciprocals, and rows of
// zeros (weights without a gradient) would become NaN.
bool bad_eps(float eps) { return !finite(eps) || !(eps >= std::numeric_limits<float>::min()); }

// One tensor of a call: what it covers and whether the call writes it.
struct Use {
    const void *p;
    int64_t bytes;
    bool out;
};

// Pointers that are given must be aligned; outputs must not overlap anything, but for an
// output that is exactly the input `same`.
forge_status check_uses(const Use *u, int n, const void *same_in, const void *same_out)
{
    for (int i = 0; i < n; ++i)
        if (u[i].p && !aligned16(u[i].p)) return FORGE_ERR_MISALIGNED;
    for (int i = 0; i < n; ++i)
        for (int j = i + 1; j < n; ++j) {
            if (!u[i].p || !u[j].p || !(u[i].out || u[j].out)) continue;
            if (!overlap(range_of(u[i].p, u[i].bytes), range_of(u[j].p, u[j].bytes))) continue;
            const bool in_place = same_in && same_in == same_out && u[i].out != u[j].out && u[i].p == same_in &&
                                  u[j].p == same_in && u[i].bytes == u[j].bytes;
            if (!in_place) return FORGE_ERR_ALIASING;
        }
    return FORGE_OK;
}

int64_t chunks_of(int64_t numel) { return (numel + MT_CHUNK - 1) / MT_CHUNK; }

MtTable table_of(const forge_tensor_list &l, const void *table)
{
    MtTable t;
    t.t = static_cast<const MtTensor *>(table);
    t.owner = reinterpret_cast<const int32_t *>(t.t + l.n);
    t.chunks = l.chunks;
    return t;
}

// A tensor's own rules; `live`: it has elements.
forge_status check_tensor(const forge_tensor &x, bool &live)
{
    live = x.numel > 0;
    if (!is_float(x.g_dtype)) return FORGE_ERR_INVALID_DTYPE;
    if (x.W && (!is_float(x.w_dtype) || (!is_float(x.state_dtype) && x.state_dtype != FORGE_DTYPE_FP8)))
        return FORGE_ERR_INVALID_DTYPE;
    if (x.numel < 0) return FORGE_ERR_INVALID_SHAPE;
    if (x.numel > kMaxElems) return FORGE_ERR_UNSUPPORTED_SHAPE;
    if (!live) return FORGE_OK;
    const bool f8 = x.W && x.state_dtype == FORGE_DTYPE_FP8;
    if (!x.G || (x.W && (!x.m || !x.v)) || (f8 && (!x.m_scale || !x.v_scale))) return FORGE_ERR_NULL_POINTER;
    if (!finite(x.lr_scale) || !(x.lr_scale >= 0.0f) || !finite(x.weight_decay)) return FORGE_ERR_INVALID_HYPERPARAM;
    if (!aligned16(x.G) || (x.W && (!aligned16(x.W) || !aligned16(x.m) || !aligned16(x.v))) ||
        (f8 && (!aligned16(x.m_scale) || !aligned16(x.v_scale))))
        return FORGE_ERR_MISALIGNED;
    return FORGE_OK;
}

struct Span {
    Range r;
    bool out;
};

// No written range meets another range: in order of their starts, each range against the
// furthest end of the written ones before it, and a written one against that of all.
bool disjoint(Span *s, int64_t n)
{
    std::sort(s, s + n, [](const Span &a, const Span &b) { return a.r.lo < b.r.lo; });
    uintptr_t any = 0, out = 0;
    for (int64_t i = 0; i < n; ++i) {
        if (s[i].r.lo < (s[i].out ? any : out)) return false;
        any = std::max(any, s[i].r.hi);
        if (s[i].out) out = std::max(out, s[i].r.hi);
    }
    return true;
}

}  // namespace

extern "C" {

forge_status forge_rmsnorm(const void *x, const void *residual, const void *w, void *h, void *y, void *q, float *q_scale,
                           int64_t T, int64_t d, int32_t h_dtype, int32_t w_dtype, int32_t q_group, float eps,
                           void *stream)
{
    forge_status s;
    if (!is_float(h_dtype) || !is_float(w_dtype)) return FORGE_ERR_INVALID_DTYPE;
    if ((s = check_rows(T, d)) != FORGE_OK) return s;
    if (q && q_group != 0 && q_group != FORGE_Q_GROUP) return FORGE_ERR_UNSUPPORTED_SHAPE;
    if (T == 0 || d == 0) return FORGE_OK;
    if (!x || !w || (!y && !q) || (q && !q_scale) || (residual != nullptr) != (h != nullptr))
        return FORGE_ERR_NULL_POINTER;
    if (bad_eps(eps)) return FORGE_ERR_INVALID_HYPERPARAM;
    const int64_t N = T * d, hb = bytes_of(h_dtype);
    const int64_t scales = T * (q_group ? (d + FORGE_Q_GROUP - 1) / FORGE_Q_GROUP : 1);
    const Use u[] = {{x, N * (residual ? 2 : hb), false}, {residual, N * hb, false}, {w, d * bytes_of(w_dtype), false},
                     {h, N * hb, true}, {y, N * 2, true}, {q, N, true}, {q ? q_scale : nullptr, scales * 4, true}};
    if ((s = check_uses(u, 7, residual, h)) != FORGE_OK) return s;
    if ((s = check_device()) != FORGE_OK) return s;
    NormArgs a{x, residual, w, h, static_cast<uint16_t *>(y), static_cast<uint8_t *>(q), q_scale,
               static_cast<int>(T), static_cast<int>(d), h_dtype == FORGE_DTYPE_BF16, w_dtype == FORGE_DTYPE_BF16,
               q_group, eps};
    return from_hip(launch_rmsnorm(a, static_cast<hipStream_t>(stream)));
}

int64_t forge_rmsnorm_backward_workspace(int64_t T, int64_t d)
{
    return check_rows(T, d) == FORGE_OK ? 4 * d * norm_grad_plan(T, d).groups : 0;
}

forge_status forge_rmsnorm_backward(const void *dy, const void *h, const void *w, const void *dres, void *dh, void *dx,
                                    float *dw, int64_t T, int64_t d, int32_t h_dtype, int32_t w_dtype, float eps,
                                    void *ws, int64_t ws_bytes, void *stream)
{
    forge_status s;
    if (!is_float(h_dtype) || !is_float(w_dtype)) return FORGE_ERR_INVALID_DTYPE;
    if ((s = check_rows(T, d)) != FORGE_OK) return s;
    const int64_t need = forge_rmsnorm_backward_workspace(T, d);
    if (d == 0) return FORGE_OK;
    if (ws_bytes < need) return FORGE_ERR_INVALID_SHAPE;
    if (!dw || (T > 0 && (!dy || !h || !w || (!dh && !dx) || !ws))) return FORGE_ERR_NULL_POINTER;
    if (bad_eps(eps)) return FORGE_ERR_INVALID_HYPERPARAM;
    const int64_t N = T * d, hb = bytes_of(h_dtype);
    const Use u[] = {{dy, N * 2, false}, {h, N * hb, false}, {w, d * bytes_of(w_dtype), false}, {dres, N * hb, false},
                     {dh, N * hb, true}, {dx, N * 2, true}, {dw, d * 4, true}, {ws, need, true}};
    if (T == 0) s = aligned16(dw) ? FORGE_OK : FORGE_ERR_MISALIGNED;
    else s = check_uses(u, 8, dres, dh);
    if (s != FORGE_OK) return s;
    if ((s = check_device()) != FORGE_OK) return s;
    NormGradArgs a{static_cast<const uint16_t *>(dy), h, w, dres, dh, static_cast<uint16_t *>(dx), dw,
                   static_cast<float *>(ws), static_cast<int>(T), static_cast<int>(d), h_dtype == FORGE_DTYPE_BF16,
                   w_dtype == FORGE_DTYPE_BF16, eps};
    return from_hip(launch_rmsnorm_backward(a, static_cast<hipStream_t>(stream)));
}

int64_t forge_tensor_list_bytes(const forge_tensor *tensors, int32_t n)
{
    if (!tensors || n <= 0) return 0;
    int64_t chunks = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (tensors[i].numel < 0 || tensors[i].numel > kMaxElems) return 0;
        chunks += chunks_of(tensors[i].numel);
    }
    return static_cast<int64_t>(sizeof(MtTensor)) * n + 4 * chunks;
}

forge_status forge_tensor_list_build(const forge_tensor *tensors, int32_t n, void *table, int64_t bytes,
                                     forge_tensor_list *list)
{
    forge_status s;
    if (!list || (n > 0 && (!tensors || !table))) return FORGE_ERR_NULL_POINTER;
    if (n < 0) return FORGE_ERR_INVALID_SHAPE;
    int64_t chunks = 0;
    bool steppable = true, live;
    for (int32_t i = 0; i < n; ++i) {
        if ((s = check_tensor(tensors[i], live)) != FORGE_OK) return s;
        chunks += chunks_of(tensors[i].numel);
        if (live && !tensors[i].W) steppable = false;
    }
    if (chunks > MT_MAX_CHUNKS) return FORGE_ERR_UNSUPPORTED_SHAPE;
    const int64_t need = n > 0 ? forge_tensor_list_bytes(tensors, n) : 0;
    if (bytes < need) return FORGE_ERR_INVALID_SHAPE;
    if (n > 0) {
        Span *spans = new (std::nothrow) Span[6 * static_cast<size_t>(n)];
        if (!spans) return FORGE_ERR_LAUNCH;
        int64_t k = 0;
        for (int32_t i = 0; i < n; ++i) {
            const forge_tensor &x = tensors[i];
            if (x.numel == 0) continue;
            spans[k++] = {range_of(x.G, x.numel * bytes_of(x.g_dtype)), false};
            if (!x.W) continue;
            const int64_t state = x.numel * bytes_of(x.state_dtype);
            spans[k++] = {range_of(x.W, x.numel * bytes_of(x.w_dtype)), true};
            spans[k++] = {range_of(x.m, state), true};
            spans[k++] = {range_of(x.v, state), true};
            if (x.state_dtype == FORGE_DTYPE_FP8) {
                const int64_t sc = 4 * ((x.numel + MT_BLOCK - 1) / MT_BLOCK);
                spans[k++] = {range_of(x.m_scale, sc), true};
                spans[k++] = {range_of(x.v_scale, sc), true};
            }
        }
        const bool ok = disjoint(spans, k);
        delete[] spans;
        if (!ok) return FORGE_ERR_ALIASING;
    }
    MtTensor *t = static_cast<MtTensor *>(table);
    int32_t *owner = n > 0 ? reinterpret_cast<int32_t *>(t + n) : nullptr;
    int32_t c = 0;
    for (int32_t i = 0; i < n; ++i) {
        const forge_tensor &x = tensors[i];
        t[i] = MtTensor{x.W, x.G, x.m, x.v, x.m_scale, x.v_scale, static_cast<int32_t>(x.numel), c, x.lr_scale,
                        x.weight_decay, x.w_dtype, x.g_dtype, x.state_dtype, 0};
        const int32_t end = c + static_cast<int32_t>(chunks_of(x.numel));
        for (; c < end; ++c) owner[c] = i;
    }
    *list = forge_tensor_list{need, chunks, n, steppable};
    return FORGE_OK;
}

int64_t forge_grad_norm_workspace(const forge_tensor_list *list)
{
    return list ? 8 * std::min<int64_t>(std::max<int64_t>(list->chunks, 0), MT_NORM_PARTS) : 0;
}

forge_status forge_grad_norm(const forge_tensor_list *list, const void *table, float max_norm, float *out, void *ws,
                             int64_t ws_bytes, void *stream)
{
    forge_status s;
    if (!list) return FORGE_ERR_NULL_POINTER;
    const int64_t need = forge_grad_norm_workspace(list);
    if (list->chunks < 0 || list->n < 0 || ws_bytes < need) return FORGE_ERR_INVALID_SHAPE;
    if (!out || (list->chunks > 0 && (!table || !ws))) return FORGE_ERR_NULL_POINTER;
    if (!finite(max_norm) || !(max_norm > 0.0f)) return FORGE_ERR_INVALID_HYPERPARAM;
    if (!aligned4(out) || (list->chunks > 0 && (!aligned16(table) || !aligned16(ws)))) return FORGE_ERR_MISALIGNED;
    if (list->chunks > 0) {
        const Range ro = range_of(out, 8), rt = range_of(table, list->table_bytes), rw = range_of(ws, need);
        if (overlap(ro, rt) || overlap(ro, rw) || overlap(rt, rw)) return FORGE_ERR_ALIASING;
    }
    if ((s = check_device()) != FORGE_OK) return s;
    return from_hip(launch_grad_norm(table_of(*list, table), max_norm, out, static_cast<double *>(ws),
                                     static_cast<hipStream_t>(stream)));
}

forge_status forge_adamw_multi(const forge_tensor_list *list, const void *table, float lr, float beta1, float beta2,
                               float eps, const float *grad_scale, int64_t step, void *stream)
{
    forge_status s;
    if (!list) return FORGE_ERR_NULL_POINTER;
    if (list->chunks < 0 || list->n < 0) return FORGE_ERR_INVALID_SHAPE;
    if (list->chunks == 0) return FORGE_OK;
    if (!table || !list->steppable) return FORGE_ERR_NULL_POINTER;
    if ((s = check_hyper(lr, beta1, beta2, eps, 0.0f, step)) != FORGE_OK) return s;
    if (bad_eps(eps)) return FORGE_ERR_INVALID_HYPERPARAM;
    if (!aligned16(table) || !aligned4(grad_scale)) return FORGE_ERR_MISALIGNED;
    if ((s = check_device()) != FORGE_OK) return s;
    const double t = static_cast<double>(step), b1 = beta1, b2 = beta2;
    MtHyper h;
    h.b1 = beta1;
    h.c1 = static_cast<float>(1.0 - b1);
    h.b2 = beta2;
    h.c2 = static_cast<float>(1.0 - b2);
    h.inv_sqrt_bc2 = static_cast<float>(1.0 / std::sqrt(1.0 - std::pow(b2, t)));
    h.eps = eps;
    h.lr = lr;
    h.lr_bc1 = static_cast<double>(lr) / (1.0 - std::pow(b1, t));
    return from_hip(launch_adamw_multi(table_of(*list, table), h, grad_scale, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
