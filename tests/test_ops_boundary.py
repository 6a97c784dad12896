"""The boundary of include/forge_ops.h on the host: every documented refusal is returned before
any HIP call, and a tensor list is laid out as the kernels read it.

Pointers are fake addresses that validation never dereferences.  Where arguments are valid the
call stops at the device check (FORGE_ERR_NO_DEVICE), so those calls are made only where no GPU
is visible.
"""
import ctypes
import struct

import pytest
import torch

from paper_2606_22932_amd import forge

OK, NULLP, SHAPE, UNSUP, HYPER, DTYPE, MISAL, ALIAS, NODEV = range(9)
F32, BF16, FP8 = 0, 1, 2
GiB = 1 << 30
no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="a valid call would launch")


def lib():
    return forge._ops()


NORM = dict(x=1 * GiB, residual=2 * GiB, w=3 * GiB, h=4 * GiB, y=5 * GiB, q=6 * GiB, q_scale=7 * GiB, T=4, d=256,
            h_dtype=BF16, w_dtype=BF16, q_group=128, eps=1e-5)


def norm(**over):
    a = {**NORM, **over}
    return lib().forge_rmsnorm(*a.values(), None)


GRAD = dict(dy=1 * GiB, h=2 * GiB, w=3 * GiB, dres=4 * GiB, dh=5 * GiB, dx=6 * GiB, dw=7 * GiB, T=4, d=256,
            h_dtype=BF16, w_dtype=BF16, eps=1e-5, ws=8 * GiB, ws_bytes=1 << 24)


def grad(**over):
    a = {**GRAD, **over}
    return lib().forge_rmsnorm_backward(*a.values(), None)


def test_library_exports_the_header():
    names = forge.header_functions(forge.OPS_HEADER)
    assert set(names) == set(forge._OPS_SIGS)
    for n in names:
        assert hasattr(lib(), n), n


@pytest.mark.parametrize("over,want", [
    (dict(h_dtype=2), DTYPE), (dict(w_dtype=-1), DTYPE), (dict(T=-1), SHAPE), (dict(d=-8), SHAPE),
    (dict(d=12), UNSUP), (dict(T=1 << 20, d=1 << 12), UNSUP), (dict(T=1 << 62, d=8), UNSUP),
    (dict(q_group=64), UNSUP),
    (dict(T=0, x=0, w=0), OK), (dict(d=0, x=0, w=0), OK),
    (dict(x=0), NULLP), (dict(w=0), NULLP), (dict(h=0), NULLP), (dict(residual=0), NULLP), (dict(y=0, q=0), NULLP),
    (dict(q_scale=0), NULLP),
    (dict(eps=0.0), HYPER), (dict(eps=-1.0), HYPER), (dict(eps=float("nan")), HYPER), (dict(eps=float("inf")), HYPER),
    *[({k: NORM[k] + 8}, MISAL) for k in ("x", "residual", "w", "h", "y", "q", "q_scale")],
    (dict(y=NORM["x"]), ALIAS), (dict(y=NORM["h"]), ALIAS), (dict(h=NORM["x"]), ALIAS), (dict(q=NORM["w"]), ALIAS),
    (dict(h=NORM["residual"] + 16), ALIAS), (dict(q_scale=NORM["q"] + 4 * 256 - 16), ALIAS),
    (dict(w=NORM["y"] + 2 * 4 * 256 - 16), ALIAS),
], ids=str)
def test_rmsnorm_refusals(over, want):
    assert norm(**over) == want


@no_gpu
@pytest.mark.parametrize("over", [
    {}, dict(h=NORM["residual"]), dict(residual=0, h=0), dict(y=0), dict(q=0, q_scale=0, q_group=7),
    dict(w=NORM["y"] + 2 * 4 * 256), dict(T=1, d=8), dict(h_dtype=F32, w_dtype=F32)], ids=str)
def test_rmsnorm_accepts(over):
    assert norm(**over) == NODEV


@pytest.mark.parametrize("over,want", [
    (dict(h_dtype=2), DTYPE), (dict(w_dtype=7), DTYPE), (dict(T=-1), SHAPE), (dict(d=9), UNSUP),
    (dict(ws_bytes=0), SHAPE), (dict(d=0, dw=0, ws_bytes=0), OK),
    (dict(dw=0), NULLP), (dict(dy=0), NULLP), (dict(h=0), NULLP), (dict(w=0), NULLP), (dict(dh=0, dx=0), NULLP),
    (dict(ws=0), NULLP), (dict(T=0, dw=0), NULLP), (dict(eps=0.0), HYPER), (dict(T=0, dw=GRAD["dw"] + 4), MISAL),
    *[({k: GRAD[k] + 8}, MISAL) for k in ("dy", "h", "w", "dres", "dh", "dx", "dw", "ws")],
    (dict(dh=GRAD["h"]), ALIAS), (dict(dh=GRAD["dres"] + 16), ALIAS), (dict(dx=GRAD["dy"]), ALIAS),
    (dict(dx=GRAD["dh"]), ALIAS), (dict(dw=GRAD["w"]), ALIAS), (dict(ws=GRAD["h"]), ALIAS),
], ids=str)
def test_rmsnorm_backward_refusals(over, want):
    assert grad(**over) == want


@no_gpu
@pytest.mark.parametrize("over", [
    {}, dict(dh=GRAD["dres"]), dict(dres=0), dict(dh=0), dict(dx=0),
    dict(T=0, dy=0, h=0, w=0, dh=0, dx=0, ws=0, ws_bytes=0)], ids=str)
def test_rmsnorm_backward_accepts(over):
    assert grad(**over) == NODEV


def test_workspace_sizes():
    L = lib()
    assert L.forge_rmsnorm_backward_workspace(0, 64) == 0
    assert L.forge_rmsnorm_backward_workspace(-1, 64) == L.forge_rmsnorm_backward_workspace(3, 12) == 0
    need = L.forge_rmsnorm_backward_workspace(GRAD["T"], GRAD["d"])
    assert grad(ws_bytes=need - 1) == SHAPE and grad(ws_bytes=need, w=0) == NULLP
    for T, d in ((1, 8), (7, 4096), (1 << 20, 64), (1 << 14, 1 << 14), ((1 << 31) // 8 - 1, 8)):
        n = L.forge_rmsnorm_backward_workspace(T, d)
        assert n > 0 and n % (4 * d) == 0 and n <= 4 * d * min(T, 4096)


# ----------------------------------------------------------------------------- tensor lists

def tensor(k, numel=1000, **over):
    """The k-th of well separated fake tensors."""
    b = (1 + 8 * k) * GiB
    t = dict(W=b, G=b + GiB, m=b + 2 * GiB, v=b + 3 * GiB, m_scale=b + 4 * GiB, v_scale=b + 5 * GiB, numel=numel,
             lr_scale=1.0, weight_decay=0.1, w_dtype=BF16, g_dtype=BF16, state_dtype=BF16)
    return forge.forge_tensor(**{**t, **over})


def build(ts, short=0):
    n = len(ts)
    arr = (forge.forge_tensor * max(n, 1))(*ts)
    size = lib().forge_tensor_list_bytes(arr, n)
    buf = (ctypes.c_uint8 * max(size - short, 1))()
    out = forge.forge_tensor_list()
    st = lib().forge_tensor_list_build(arr, n, ctypes.addressof(buf), size - short, ctypes.byref(out))
    return st, out, bytes(buf)


@pytest.mark.parametrize("over,want", [
    (dict(g_dtype=2), DTYPE), (dict(w_dtype=2), DTYPE), (dict(state_dtype=3), DTYPE), (dict(state_dtype=-1), DTYPE),
    (dict(numel=-1), SHAPE), (dict(numel=1 << 31), UNSUP),
    (dict(G=0), NULLP), (dict(m=0), NULLP), (dict(v=0), NULLP), (dict(state_dtype=FP8, m_scale=0), NULLP),
    (dict(state_dtype=FP8, v_scale=0), NULLP),
    (dict(lr_scale=-1.0), HYPER), (dict(lr_scale=float("nan")), HYPER), (dict(weight_decay=float("inf")), HYPER),
    *[({k: 100 * GiB + 8}, MISAL) for k in ("W", "G", "m", "v")],
    *[({k: 100 * GiB + 8, "state_dtype": FP8}, MISAL) for k in ("m_scale", "v_scale")],
    (dict(W=2 * GiB), ALIAS), (dict(m=4 * GiB), ALIAS), (dict(G=1 * GiB + 1984), ALIAS),
    (dict(state_dtype=FP8, v_scale=5 * GiB), ALIAS),
], ids=str)
def test_list_refusals(over, want):
    assert build([tensor(0, **over)])[0] == want
    assert build([tensor(2), tensor(0, **over), tensor(1)])[0] == want


def test_list_of_the_same_tensor_twice():
    assert build([tensor(0), tensor(1), tensor(0)])[0] == ALIAS
    shared = [tensor(0, W=0), tensor(0, W=0)]            # read only: gradients may be shared
    assert build(shared)[0] == OK


def test_list_arguments():
    L, out = lib(), forge.forge_tensor_list()
    arr = (forge.forge_tensor * 1)(tensor(0))
    assert build([tensor(0)], short=1)[0] == SHAPE
    assert L.forge_tensor_list_build(None, 1, None, 0, ctypes.byref(out)) == NULLP
    assert L.forge_tensor_list_build(arr, 1, None, 0, ctypes.byref(out)) == NULLP
    assert L.forge_tensor_list_build(arr, 1, ctypes.addressof(arr), 1 << 20, None) == NULLP
    assert L.forge_tensor_list_build(None, -1, None, 0, ctypes.byref(out)) == SHAPE
    assert L.forge_tensor_list_build(None, 0, None, 0, ctypes.byref(out)) == OK and out.chunks == 0
    assert L.forge_tensor_list_bytes(None, 3) == 0 and L.forge_tensor_list_bytes(arr, -1) == 0
    big = (forge.forge_tensor * 17)(*(tensor(k, numel=(1 << 31) - 1) for k in range(17)))
    mem = (ctypes.c_uint8 * 16)()                        # refused before the table is touched
    assert L.forge_tensor_list_build(big, 17, ctypes.addressof(mem), 1 << 40, ctypes.byref(out)) == UNSUP


@pytest.mark.parametrize("numels", [[1], [0], [0, 0, 5], [2048, 1, 2049, 0, 4096, 63], list(range(1, 40))], ids=str)
def test_list_layout(numels):
    """Descriptors of 80 bytes, then for each chunk of 2048 elements its tensor."""
    st, out, raw = build([tensor(k, numel=x) for k, x in enumerate(numels)])
    assert st == OK and out.n == len(numels) and out.steppable
    owner = []
    for k, x in enumerate(numels):
        f = struct.unpack_from("<6Q2i2f4i", raw, 80 * k)
        b = (1 + 8 * k) * GiB
        assert f[:6] == tuple(b + i * GiB for i in range(6)) and f[6:8] == (x, len(owner))
        assert f[8] == 1.0 and f[9] == pytest.approx(0.1) and f[10:13] == (BF16, BF16, BF16)
        owner += [k] * -(-x // 2048)
    assert out.chunks == len(owner) and out.table_bytes == 80 * len(numels) + 4 * len(owner)
    assert list(struct.unpack_from("<%di" % len(owner), raw, 80 * len(numels))) == owner


def some_list(n=2, **over):
    st, out, _ = build([tensor(k, **over) for k in range(n)])
    assert st == OK
    return out


NORMS = dict(table=1 * GiB, max_norm=1.0, out=2 * GiB, ws=3 * GiB, ws_bytes=1 << 20)


def total(lst, **over):
    a = {**NORMS, **over}
    return lib().forge_grad_norm(None if lst is None else ctypes.byref(lst), *a.values(), None)


STEP = dict(table=1 * GiB, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=2 * GiB, step=1)


def step(lst, **over):
    a = {**STEP, **over}
    return lib().forge_adamw_multi(None if lst is None else ctypes.byref(lst), *a.values(), None)


@pytest.mark.parametrize("over,want", [
    (dict(ws_bytes=0), SHAPE), (dict(table=0), NULLP), (dict(out=0), NULLP), (dict(ws=0), NULLP),
    (dict(max_norm=0.0), HYPER), (dict(max_norm=float("nan")), HYPER), (dict(max_norm=float("inf")), HYPER),
    (dict(out=2 * GiB + 2), MISAL), (dict(ws=3 * GiB + 8), MISAL), (dict(table=GiB + 4), MISAL),
    (dict(out=3 * GiB), ALIAS), (dict(ws=GiB), ALIAS)], ids=str)
def test_grad_norm_refusals(over, want):
    assert total(some_list(), **over) == want
    assert total(None) == NULLP


@pytest.mark.parametrize("over,want", [
    (dict(table=0), NULLP), (dict(step=0), HYPER), (dict(beta1=1.0), HYPER), (dict(beta2=-0.5), HYPER),
    (dict(eps=0.0), HYPER), (dict(lr=-1.0), HYPER), (dict(lr=float("nan")), HYPER),
    (dict(table=GiB + 8), MISAL), (dict(grad_scale=2 * GiB + 2), MISAL)], ids=str)
def test_adamw_multi_refusals(over, want):
    assert step(some_list(), **over) == want
    assert step(None) == NULLP
    assert step(some_list(W=0)) == NULLP                 # a list that is only normed
    assert step(some_list(n=0), table=0) == OK
    assert step(some_list(numel=0), table=0) == OK


@no_gpu
def test_list_calls_accept():
    assert total(some_list()) == total(some_list(W=0)) == NODEV
    assert total(some_list(n=0), table=0, ws=0, ws_bytes=0) == NODEV     # the norm of nothing is written
    assert step(some_list()) == step(some_list(), grad_scale=0) == NODEV


# ----------------------------------------------------------------------------- the binding

def test_binding_refuses_host_tensors():
    x, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.ones(8)
    with pytest.raises(ValueError, match="HIP device"):
        forge.forge_rmsnorm(x, w, y=x.clone(), eps=1e-5)
    with pytest.raises(ValueError, match="HIP device"):
        forge.forge_rmsnorm_backward(x, x, w, dh=x.clone(), dw=w.clone(), eps=1e-5, ws=w)
    with pytest.raises(ValueError, match="HIP device"):
        forge.TensorList([(x, x, x, x)])
    with pytest.raises(ValueError, match="one number, or one per tensor"):
        forge.TensorList([(x, x, x, x)], lr_scale=[1.0, 2.0])
    with pytest.raises(ValueError, match="gradient"):
        forge.TensorList([(x, None, x, x)])


def test_an_empty_list():
    t = forge.TensorList([])
    assert t.table is None and forge.forge_grad_norm_workspace(t) == 0
    forge.forge_adamw_multi(t, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
