"""The 64-bit references of the operators against differences and torch's own double arithmetic."""
import pytest
import torch

import ops_ref as R

D = torch.float64


def _rand(*shape, seed):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=D)


@pytest.mark.parametrize("T,d,eps", [(1, 8, 1e-5), (3, 24, 1e-2), (5, 7, 1e-6)])
def test_norm_gradient_against_differences(T, d, eps):
    h, w, dy, dres = _rand(T, d, seed=1), _rand(d, seed=2), _rand(T, d, seed=3), _rand(T, d, seed=4)
    dh, _, dw, _ = R.rmsnorm_backward(dy, h, w, eps, dres)
    # the loss whose gradient reaches the norm's output as dy and the stream as dres
    loss = lambda h, w: float((dy * R.rmsnorm(h, w, eps)).sum() + (dres * h).sum())
    step = 1e-6
    for x, grad, f in ((h, dh, lambda p: loss(p, w)), (w, dw, lambda p: loss(h, p))):
        for k in range(x.numel()):
            e = torch.zeros(x.numel(), dtype=D)
            e[k] = step
            e = e.view_as(x)
            diff = (f(x + e) - f(x - e)) / (2 * step)
            # central differences: step^2 of truncation, 1e-16 |loss| / step of rounding
            assert abs(diff - float(grad.flatten()[k])) < 1e-7 * (1 + abs(diff))


@pytest.mark.parametrize("step", [1, 7, 1000])
def test_adamw_against_torch(step):
    n, hp = 40, dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8)
    w, g, m, v = _rand(n, seed=1), _rand(n, seed=2), _rand(n, seed=3), _rand(n, seed=4).abs()
    p = torch.nn.Parameter(w.clone())
    f = lambda x: float(torch.tensor(x, dtype=torch.float32))       # hyper-parameters are fp32 numbers
    opt = torch.optim.AdamW([p], lr=f(1e-3) * 0.5, betas=(f(0.9), f(0.999)), eps=f(1e-8), weight_decay=f(0.1),
                            foreach=False)
    opt.state[p] = dict(step=torch.tensor(float(step - 1)), exp_avg=m.clone(), exp_avg_sq=v.clone())
    p.grad = g * 0.25
    opt.step()
    r = R.adamw(w, g, m, v, step=step, lr_scale=0.5, weight_decay=0.1, grad_scale=0.25, **hp)
    torch.testing.assert_close(r["w"], p.detach(), rtol=1e-13, atol=1e-15)
    torch.testing.assert_close(r["m"], opt.state[p]["exp_avg"], rtol=1e-13, atol=1e-15)
    torch.testing.assert_close(r["v"], opt.state[p]["exp_avg_sq"], rtol=1e-13, atol=1e-15)


def test_clip_coefficient_against_torch():
    g = [_rand(5, 3, seed=1), _rand(7, seed=2)]
    p = [torch.nn.Parameter(torch.zeros_like(x)) for x in g]
    for q, x in zip(p, g):
        q.grad = x.clone()
    n = torch.nn.utils.clip_grad_norm_(p, 0.5)
    norm, coef = R.grad_norm(g, 0.5)
    assert abs(float(n) - norm) < 1e-12 * norm
    for q, x in zip(p, g):
        torch.testing.assert_close(q.grad, x * coef, rtol=1e-12, atol=0)
    assert R.grad_norm(g, 1e9)[1] == 1.0


def test_bounds_notice_a_wrong_value():
    """A mistake planted in the oracle is seen."""
    h, w = _rand(4, 64, seed=1).float(), _rand(64, seed=2).float()
    y = R.rmsnorm(h, w, 1e-5)
    R.stored(y.to(torch.bfloat16), y, R.sums(64) * y.abs(), "y")
    with pytest.raises(AssertionError):
        R.stored(y.to(torch.bfloat16), y * (1 + 2 ** -6), R.sums(64) * y.abs(), "y")
    s, each = R.scales(y, 16)
    q = (y / each).to(torch.float32).to(torch.float8_e4m3fn)
    R.coded(q, s, each, y, R.sums(64) * y.abs(), "q")
    with pytest.raises(AssertionError):
        R.coded(q, s, each, y * 1.2, R.sums(64) * y.abs(), "q")
