"""The operators of include/forge_ops.h in 64 bits, and how far an fp32 kernel may be from them.

Everything here is torch on the CPU in float64, written from the formulas in the header.  The
bounds count roundings: U is half a step of fp32, `half(t)` half a step of a stored type.
"""
import torch

D = torch.float64
U = 2.0 ** -24
TINY = 2.0 ** -126                  # values below may be flushed or lose bits: an absolute slack


def half(dtype):
    return torch.finfo(dtype).eps / 2


def f64(t):
    return t.detach().cpu().to(D)


def sums(d):
    """Relative error of an fp32 sum of d products: each thread adds at most d / 64 of them and the
    joins add at most 64 more, each addition off by U; the products and the functions after the
    sum (mean, eps, reciprocal root, which the hardware gives to one step) add under 32 U."""
    return (d / 64 + 96) * U


def stream_sum(x, r):
    return f64(r) + f64(x)


def rms(h, eps):
    return 1.0 / torch.sqrt(f64(h).square().mean(-1, keepdim=True) + eps)


def rmsnorm(h, w, eps):
    return f64(h) * rms(h, eps) * f64(w)


def scales(y, group):
    """amax / 448 of each group of columns (0: the row), and it spread over the columns."""
    d = y.shape[-1]
    size = group or max(d, 1)
    at = torch.arange(d) // size
    amax = torch.nn.functional.pad(y.abs(), (0, -d % size)).unflatten(-1, (-1, size)).amax(-1)
    s = torch.where(amax / 448 < TINY, torch.zeros_like(amax), amax / 448)
    return (s if group else s[:, 0]), s[:, at]


def rmsnorm_backward(dy, h, w, eps, dres=None):
    """dh, dw, and for each the sum of its terms' magnitudes."""
    g, x, s = f64(dy), f64(h), rms(h, eps)
    a = g * f64(w)
    c, ca = s * s * (a * x).mean(-1, keepdim=True), s * s * (a * x).abs().mean(-1, keepdim=True)
    dh, size = s * (a - x * c), s * (a.abs() + x.abs() * ca)
    if dres is not None:
        dh, size = dh + f64(dres), size + f64(dres).abs()
    t = g * x * s
    return dh, size, t.sum(0), t.abs().sum(0)


def grad_norm(grads, max_norm):
    n = float(sum(float(f64(g).square().sum()) for g in grads)) ** 0.5
    return n, min(1.0, max_norm / (n + 1e-6))


def adamw(w, g, m, v, *, lr, beta1, beta2, eps, step, lr_scale=1.0, weight_decay=0.0, grad_scale=1.0):
    """New w, m, v, root (all before any storage rounding; m and v are decoded values), and bounds
    on what fp32 arithmetic loses of each."""
    f = lambda x: float(torch.tensor(x, dtype=torch.float32))
    lr, beta1, beta2, eps, ls, wd = f(lr), f(beta1), f(beta2), f(eps), f(lr_scale), f(weight_decay)
    g = g * grad_scale
    bc1, bc2 = 1 - beta1 ** step, 1 - beta2 ** step
    m1 = beta1 * m + (1 - beta1) * g
    # roundings: of 1 - beta1, of the scaled gradient, of c1 g, of the fma; of the decoded m
    em = 5 * U * ((beta1 * m).abs() + ((1 - beta1) * g).abs()) + TINY
    v1 = beta2 * v + (1 - beta2) * g * g
    ev = 8 * U * v1 + TINY                    # as for m, the gradient's counted twice
    root = v1.sqrt()
    er = 4 * U * root + 2 * U * root + (ev + root * root).sqrt() - root
    den = root / bc2 ** 0.5 + eps
    u = lr * ls / bc1 * m1 / den
    eu = lr * ls / bc1 * em / den + u.abs() * ((er / bc2 ** 0.5) / den + 8 * U)
    w1 = (1 - lr * ls * wd) * w - u
    return dict(w=w1, m=m1, v=v1, root=root, ew=eu + 3 * U * (w.abs() + u.abs()), em=em, ev=ev, er=er)


def within(got, want, bound, what):
    """Every element finite where wanted and at most `bound` from `want`."""
    got = f64(got)
    off = (got - want).abs()
    bad = ~(off <= bound)
    if bool(bad.any()):
        k = int(torch.where(bad.flatten(), (off / (bound + 1e-300)).flatten(), torch.zeros_like(off).flatten()).argmax())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} outside, e.g. at {k}: got "
                             f"{float(got.flatten()[k])!r}, want {float(want.flatten()[k])!r}, "
                             f"bound {float(bound.flatten()[k])!r}")


def stored(got, want, err, what):
    """`got` is `want`, known up to err, rounded to got's type: half a step of the rounded value
    (|want| + err bounds it) and the smallest step of the type."""
    t = got.dtype
    within(got, want, half(t) * (want.abs() + err) + err + torch.finfo(t).tiny * 2 * half(t), what)


def coded(q, scale, each, want, err, what, floor=None):
    """E4M3 codes q of `want` (known up to err) with scales `each`: half a step, 2^-4 of the value,
    or half the smallest code, 2^-10 of the scale; a division by the scale off by 3 U.  Where the
    scale itself is off by a relative error, so are codes and their decoded values together."""
    got = f64(q.float()) * each
    bound = (2.0 ** -4 + 8 * U) * (want.abs() + err) + (1 + 2.0 ** -4) * err + 2.0 ** -10 * each + TINY
    if floor is not None:                       # raised to the smallest positive code
        bound = torch.where(floor, torch.maximum(bound, 2.0 ** -9 * each + err), bound)
    within(got, want, bound, what)
