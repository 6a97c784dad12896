"""The operators as a training step uses them: two residual blocks, each an RMS norm ahead of a
linear layer, the layers stepped by forge_linear_backward, or (clipped) by forge_wgrad and then
the norm of all gradients and one AdamW step over every tensor; against the same network in 64 bits.
"""
import pytest
import torch

import ops_ref as R
from paper_2606_22932_amd import forge

pytestmark = pytest.mark.gpu

HP = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8)
EPS, T, D_MODEL = 1e-5, 96, 264
BF, F32 = torch.bfloat16, torch.float32


def rand(shape, std, seed, dtype=F32, mean=0.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std + mean).to(dtype)


class Net:
    """x0 -> h1 = x0 + norm(x0; g0) W0^T -> h2 = h1 + norm(h1; g1) W1^T; the stream in fp32."""

    def __init__(self):
        self.gain = [rand((D_MODEL,), 0.1, k, mean=1.0).cuda() for k in (1, 2)]
        self.W = [rand((D_MODEL, D_MODEL), 0.05, k, BF).cuda() for k in (3, 4)]
        self.state = lambda t: (torch.zeros_like(t), torch.zeros_like(t))
        self.x0 = rand((T, D_MODEL), 1.0, 5).cuda()
        self.top = rand((T, D_MODEL), 1e-2, 6).cuda()         # the loss's gradient at h2

    def forward(self):
        y0, y1 = (torch.empty((T, D_MODEL), dtype=BF, device="cuda") for _ in range(2))
        forge.forge_rmsnorm(self.x0, self.gain[0], y=y0, eps=EPS)
        out0 = y0 @ self.W[0].t()                           # the layer's forward, bf16
        h1 = torch.empty_like(self.x0)
        forge.forge_rmsnorm(out0, self.gain[1], residual=self.x0, h=h1, y=y1, eps=EPS)
        return y0, h1, y1

    def backward(self, layer):
        """layer(k, X, dY, dX) steps W_k or stores its gradient, and writes dX = dY W_k."""
        y0, h1, y1 = self.forward()
        new = lambda dt, *s: torch.empty(s or (T, D_MODEL), dtype=dt, device="cuda")
        ws = new(torch.uint8, forge.forge_rmsnorm_backward_workspace(T, D_MODEL))
        dY, dX, dg = self.top.to(BF), new(BF), [new(F32, D_MODEL) for _ in range(2)]
        layer(1, y1, dY, dX)
        dh1, dY0 = new(F32), new(BF)
        forge.forge_rmsnorm_backward(dX, h1, self.gain[1], dres=self.top, dh=dh1, dx=dY0, dw=dg[1], eps=EPS, ws=ws)
        dX0 = new(BF)
        layer(0, y0, dY0, dX0)
        dx = new(F32)
        forge.forge_rmsnorm_backward(dX0, self.x0, self.gain[0], dres=dh1, dh=dx, dw=dg[0], eps=EPS, ws=ws)
        return dg, dx

    def reference(self):
        """Gradients of sum(top * h2) in 64 bits by autograd: of the gains, the weights and x0."""
        leaves = [R.f64(t).requires_grad_() for t in (*self.gain, *self.W, self.x0)]
        g0, g1, W0, W1, x = leaves
        norm = lambda h, g: h * (h.square().mean(-1, keepdim=True) + EPS).rsqrt() * g
        h1 = x + norm(x, g0) @ W0.t()
        h2 = h1 + norm(h1, g1) @ W1.t()
        (R.f64(self.top) * h2).sum().backward()
        return [t.grad for t in leaves]


def near(got, want, what):
    """Activations and gradients between the kernels are bf16: each value passes at most six such
    roundings of 2^-8 on its way, each at most adding that share of the result's size; of a sum over
    many the errors add by their squares, and twice their root is taken."""
    got, n = R.f64(got), want.numel() ** 0.5
    off = float((got - want).norm() / want.norm())
    assert off <= 2 * (6 ** 0.5) * 2 ** -8, (what, off)


def test_clipped_step():
    net = Net()
    grads = [torch.empty((D_MODEL, D_MODEL), dtype=BF, device="cuda") for _ in range(2)]

    def layer(k, X, dY, dX):
        forge.forge_input_grad(dY, net.W[k], dX)
        forge.forge_wgrad(X, dY, grads[k])

    dg, dx = net.backward(layer)
    want = net.reference()
    for what, got, ref in zip(("dg0", "dg1", "dW0", "dW1", "dx"), (*dg, *grads, dx), want):
        near(got, ref, what)
    params, gs = (*net.gain, *net.W), (*dg, *grads)
    before = [p.cpu().clone() for p in params]
    lst = forge.TensorList([(p, g, *net.state(p)) for p, g in zip(params, gs)], weight_decay=[0.0, 0.0, 0.1, 0.1])
    out = torch.zeros(2, device="cuda")
    ws = torch.empty(forge.forge_grad_norm_workspace(lst), dtype=torch.uint8, device="cuda")
    forge.forge_grad_norm(lst, out, max_norm=0.5, ws=ws)
    forge.forge_adamw_multi(lst, step=1, grad_scale=out[1:], **HP)
    norm, coef = R.grad_norm([g.cpu() for g in gs], 0.5)
    assert coef < 1 and abs(float(out[1]) - coef) <= 2 * R.U * coef
    for p, old, g, wd in zip(params, before, gs, (0.0, 0.0, 0.1, 0.1)):
        z = torch.zeros(old.shape, dtype=R.D)
        r = R.adamw(R.f64(old), R.f64(g), z, z, step=1, weight_decay=wd, grad_scale=float(out.cpu()[1]), **HP)
        R.stored(p.cpu(), r["w"], r["ew"], "parameter")


def test_fused_layers_and_the_gains_beside_them():
    """The layers' weights stepped by the fused backward, the gains by the multi-tensor step: the
    weights end as forge_linear_backward leaves them, the gains as the formula says."""
    net = Net()
    st = [net.state(w) for w in net.W]

    def layer(k, X, dY, dX):
        forge.forge_linear_backward(X, dY, net.W[k], *st[k], dX=dX, step=1, weight_decay=0.1, **HP)

    want = net.reference()
    old = [g.cpu().clone() for g in net.gain]
    dg, dx = net.backward(layer)
    for what, got, ref in zip(("dg0", "dg1", "dx"), (*dg, dx), (*want[:2], want[4])):
        near(got, ref, what)
    forge.forge_adamw_multi(forge.TensorList([(p, g, *net.state(p)) for p, g in zip(net.gain, dg)]), step=1, **HP)
    for p, o, g in zip(net.gain, old, dg):
        z = torch.zeros(o.shape, dtype=R.D)
        r = R.adamw(R.f64(o), R.f64(g), z, z, step=1, **HP)
        R.stored(p.cpu(), r["w"], r["ew"], "gain")
