"""forge_rmsnorm and forge_rmsnorm_backward against 64 bits (ops_ref.py: every bound is a count of
roundings).  Outputs lie inside larger buffers whose other elements must keep their bytes.
"""
import pytest
import torch

import ops_ref as R
from paper_2606_22932_amd import forge

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
F8 = torch.float8_e4m3fn
EPS = 1e-5


def _say(*a):
    print(*a, flush=True)


class Guarded:
    """Output tensors with 256 bytes of 0xA5 on both sides."""

    def __init__(self):
        self.all = []

    def __call__(self, shape, dtype):
        n = torch.Size(shape).numel() * torch.empty(0, dtype=dtype).element_size()
        raw = torch.full((n + 512 + (-n) % 16,), 0xA5, dtype=torch.uint8, device="cuda")
        self.all.append((raw, n))
        return raw[256:256 + n].view(dtype).view(shape)

    def check(self):
        torch.cuda.synchronize()
        for raw, n in self.all:
            assert bool((raw[:256] == 0xA5).all()) and bool((raw[256 + n:] == 0xA5).all()), "written outside"


def rand(shape, std, dtype, seed, mean=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std + mean).to(dtype)


def forward(x, w, r=None, *, y=True, group=None, eps=EPS, in_place=False, stream=None):
    """Host inputs in, host outputs out (h, y, q, qs as asked for)."""
    T, d = x.shape
    new = Guarded()
    st = DT["bf16"] if r is None else r.dtype
    xs, ws = x.cuda(), w.cuda()
    o = {}
    rs = None
    if r is not None:
        rs = new(r.shape, r.dtype).copy_(r.cuda())
        o["h"] = rs if in_place else new((T, d), st)
    if y:
        o["y"] = new((T, d), torch.bfloat16)
    if group is not None:
        o["q"] = new((T, d), F8)
        o["q_scale"] = new((T, -(-d // 128)) if group else (T,), torch.float32)
    keep = [t.clone() for t in (xs, ws)] + ([rs.clone()] if r is not None and not in_place else [])
    forge.forge_rmsnorm(xs, ws, residual=rs, eps=eps, **o)
    new.check()
    for t, k in zip((xs, ws, rs), keep):
        assert torch.equal(t.view(torch.uint8), k.view(torch.uint8)), "an input changed"
    return {k: t.cpu() for k, t in o.items()}


def check_forward(o, x, w, r=None, *, group=None, eps=EPS):
    h = x
    if r is not None:
        want = R.stream_sum(x, r)
        R.stored(o["h"], want, R.U * want.abs(), "h")        # the fp32 sum, then its rounding
        h = o["h"]
    y = R.rmsnorm(h, w, eps)
    err = R.sums(x.shape[1]) * y.abs() + R.TINY
    if "y" in o:
        R.stored(o["y"], y, err, "y")
    if "q" in o:
        s, _ = R.scales(y, group)
        R.within(o["q_scale"], s, (R.sums(x.shape[1]) + 4 * R.U) * s + 2 * R.TINY, "q_scale")
        got = R.f64(o["q_scale"])
        each = got.unsqueeze(-1) if not group else got.repeat_interleave(128, -1)[:, :y.shape[1]]
        R.coded(o["q"], got, each.expand_as(y), y, err, "q")


FORMS = [("bf16", "bf16", True, None), ("bf16", "f32", False, 0), ("f32", "f32", True, 128), ("f32", "bf16", False, 128),
         ("f32", "bf16", True, 0), ("bf16", "bf16", True, 128)]
SHAPES = [(1, 8), (3, 64), (17, 72), (5, 120), (2, 128), (9, 136), (4, 504), (3, 520), (33, 1032), (7, 2048), (2, 2056),
          (3, 4096), (2, 4104), (1, 8192), (2, 16384), (1, 16392), (2, 32768), (1, 32776), (1, 65544)]


@pytest.mark.parametrize("T,d", SHAPES, ids=str)
@pytest.mark.parametrize("h,w,res,group", FORMS, ids=str)
def test_forward(T, d, h, w, res, group):
    _say("rmsnorm", T, d, h, w, res, group)
    x = rand((T, d), 0.5, DT["bf16"] if res else DT[h], seed=d)
    g = rand((d,), 0.1, DT[w], seed=d + 1, mean=1.0)
    r = rand((T, d), 1.0, DT[h], seed=d + 2) if res else None
    o = forward(x, g, r, y=group is None or d % 16 == 8, group=group)
    check_forward(o, x, g, r, group=group)


@pytest.mark.parametrize("T,d", [(70000, 8), (5001, 256), (17001, 520), (8300, 1032), (515, 4096)], ids=str)
@pytest.mark.parametrize("h", ["bf16", "f32"])
def test_forward_many_rows(T, d, h):
    _say("rmsnorm rows", T, d, h)
    x, g, r = rand((T, d), 0.5, DT["bf16"], 1), rand((d,), 0.1, DT["f32"], 2, 1.0), rand((T, d), 1.0, DT[h], 3)
    check_forward(forward(x, g, r, group=128), x, g, r, group=128)


@pytest.mark.parametrize("h", ["bf16", "f32"])
def test_forward_in_place(h):
    x, g, r = rand((37, 520), 0.5, DT["bf16"], 1), rand((520,), 0.1, DT["bf16"], 2, 1.0), rand((37, 520), 1.0, DT[h], 3)
    a, b = forward(x, g, r, group=0), forward(x, g, r, group=0, in_place=True)
    for k in a:
        assert torch.equal(a[k].view(torch.uint8), b[k].view(torch.uint8)), k


@pytest.mark.parametrize("group", [0, 128])
def test_forward_rows_of_zeros_small_and_large(group):
    """Rows of zeros give zeros (and scales of zero); rows far below eps and far above it hold the
    bounds; a zero gain over a whole group gives that group a zero scale."""
    T, d = 6, 392
    x = rand((T, d), 1.0, DT["f32"], 5)
    x *= torch.tensor([0.0, 1e-12, 1e-4, 1.0, 1e6, 1e15]).unsqueeze(1)
    g = rand((d,), 0.3, DT["f32"], 6)
    g[128:256] = 0.0
    o = forward(x, g, group=group)
    check_forward(o, x, g, group=group)
    assert not o["y"][0].any() and not o["q_scale"][0].any() and not o["q"][0].float().any()
    if group:
        assert not o["q_scale"][:, 1].any()


@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_forward_not_finite(bad, group):
    """What is not finite stays in its row: y has NaN there (Inf gives 0 beside itself, as the
    formula says), the scales of a row with NaN decode to no finite number, other rows are as before."""
    T, d = 5, 264
    x, g = rand((T, d), 1.0, DT["f32"], 7), rand((d,), 0.1, DT["f32"], 8, 1.0)
    a = forward(x, g, group=group)
    x[2, 130] = bad
    b = forward(x, g, group=group)
    rows = [0, 1, 3, 4]
    for k in a:
        assert torch.equal(a[k][rows].view(torch.uint8), b[k][rows].view(torch.uint8)), k
    assert torch.isnan(b["y"][2, 130])
    at = b["q_scale"][2, 1] if group else b["q_scale"][2]
    assert torch.isnan(at)
    if bad == bad:
        assert not b["y"][2, :130].any() and not b["y"][2, 131:].any()
    else:
        assert torch.isnan(b["y"][2]).all() and torch.isnan(b["q_scale"][2]).all()


def test_forward_codes_of_a_large_gain():
    """An Inf of the gain alone: the group's scale is Inf, the others finite."""
    x, g = rand((2, 256), 1.0, DT["f32"], 7), rand((256,), 0.1, DT["f32"], 8, 1.0)
    g[200] = float("inf")
    o = forward(x, g, group=128)
    assert torch.isinf(o["q_scale"][:, 1]).all() and torch.isfinite(o["q_scale"][:, 0]).all()


# ----------------------------------------------------------------------------- gradient

def backward(dy, h, w, dres=None, *, out="dh", eps=EPS, in_place=False, ws=None):
    T, d = dy.shape
    new = Guarded()
    o = {"dw": new((d,), torch.float32)}
    gs, hs, wt = dy.cuda(), h.cuda(), w.cuda()
    ds = None if dres is None else new((T, d), h.dtype).copy_(dres.cuda())
    if "dh" in out:
        o["dh"] = ds if in_place else new((T, d), h.dtype)
    if "dx" in out:
        o["dx"] = new((T, d), torch.bfloat16)
    if ws is None:
        ws = new((forge.forge_rmsnorm_backward_workspace(T, d),), torch.uint8)
        ws.fill_(0xFF)                                    # NaN: nothing may be read before it is written
    keep = [t.clone() for t in (gs, hs, wt)]
    forge.forge_rmsnorm_backward(gs, hs, wt, dres=ds, eps=eps, ws=ws, **o)
    new.check()
    for t, k in zip((gs, hs, wt), keep):
        assert torch.equal(t.view(torch.uint8), k.view(torch.uint8)), "an input changed"
    return {k: t.cpu() for k, t in o.items()}


def check_backward(o, dy, h, w, dres=None, eps=EPS):
    T, d = dy.shape
    dh, size, dw, dwsize = R.rmsnorm_backward(dy, h, w, eps, dres)
    e = R.sums(d)
    for k in ("dh", "dx"):
        if k in o:
            R.stored(o[k], dh, 3 * e * size + R.TINY, k)    # two sums and the terms' own roundings
    R.within(o["dw"], dw, (e + (T + 8) * R.U) * dwsize + R.TINY, "dw")


@pytest.mark.parametrize("T,d", SHAPES, ids=str)
@pytest.mark.parametrize("h,w,res,out", [("bf16", "bf16", True, "dh"), ("bf16", "f32", False, "dhdx"),
                                         ("f32", "f32", True, "dhdx"), ("f32", "bf16", False, "dx"),
                                         ("f32", "bf16", True, "dh")], ids=str)
def test_backward(T, d, h, w, res, out):
    _say("rmsnorm_backward", T, d, h, w, res, out)
    dy, x = rand((T, d), 1e-2, DT["bf16"], d), rand((T, d), 1.2, DT[h], d + 1)
    g, dres = rand((d,), 0.1, DT[w], d + 2, 1.0), rand((T, d), 1e-2, DT[h], d + 3) if res else None
    check_backward(backward(dy, x, g, dres, out=out), dy, x, g, dres)


@pytest.mark.parametrize("T,d", [(70000, 8), (30011, 64), (5001, 256), (1031, 1032), (6001, 1032), (515, 4096), (300, 8200)], ids=str)
@pytest.mark.parametrize("h", ["bf16", "f32"])
def test_backward_many_rows(T, d, h):
    _say("rmsnorm_backward rows", T, d, h)
    dy, x, g = rand((T, d), 1e-2, DT["bf16"], 1), rand((T, d), 1.2, DT[h], 2), rand((d,), 0.1, DT["f32"], 3, 1.0)
    dres = rand((T, d), 1e-2, DT[h], 4)
    o = backward(dy, x, g, dres, out="dhdx")
    check_backward(o, dy, x, g, dres)
    again = backward(dy, x, g, dres, out="dhdx")
    for k in o:
        assert torch.equal(o[k].view(torch.uint8), again[k].view(torch.uint8)), f"{k} differs between two calls"


@pytest.mark.parametrize("h", ["bf16", "f32"])
def test_backward_in_place(h):
    dy, x, g = rand((37, 520), 1e-2, DT["bf16"], 1), rand((37, 520), 1.2, DT[h], 2), rand((520,), 0.1, DT["bf16"], 3, 1.0)
    dres = rand((37, 520), 1e-2, DT[h], 4)
    a, b = backward(dy, x, g, dres), backward(dy, x, g, dres, in_place=True)
    assert torch.equal(a["dh"].view(torch.uint8), b["dh"].view(torch.uint8)) and torch.equal(a["dw"], b["dw"])


def test_backward_without_tokens():
    e = lambda dt: torch.empty((0, 72), dtype=dt, device="cuda")
    dw = torch.full((72,), 7.0, device="cuda")
    assert forge.forge_rmsnorm_backward_workspace(0, 72) == 0
    forge.forge_rmsnorm_backward(e(torch.bfloat16), e(torch.float32), torch.ones(72, device="cuda"),
                                 dh=e(torch.float32), dw=dw, eps=EPS, ws=None)
    assert not dw.any()
    y = e(torch.bfloat16)
    forge.forge_rmsnorm(e(torch.float32), torch.ones(72, device="cuda"), y=y, eps=EPS)


def test_backward_rows_of_zeros_and_not_finite():
    """A row of zeros: dh = dres + dy w / sqrt(eps).  A NaN stays in its row of dh and its column of dw."""
    T, d = 7, 136
    dy, x, g = rand((T, d), 1e-2, DT["bf16"], 1), rand((T, d), 1.2, DT["f32"], 2), rand((d,), 0.1, DT["f32"], 3, 1.0)
    x[1] = 0.0
    a = backward(dy, x, g)
    check_backward(a, dy, x, g)
    x[4, 9] = float("nan")
    b = backward(dy, x, g)
    rows = [0, 1, 2, 3, 5, 6]
    assert torch.equal(a["dh"][rows], b["dh"][rows]) and torch.isnan(b["dh"][4]).all()
    assert torch.isnan(b["dw"]).all()                     # every column has the row's s in it
    dy[4] = 0.0
    assert torch.isnan(backward(dy, x, g)["dw"]).all()


def test_gradient_against_differences():
    """The kernel's gradients along random directions against differences of the 64-bit forward."""
    T, d = 6, 200
    dy, h, w = rand((T, d), 1.0, DT["bf16"], 1), rand((T, d), 1.2, DT["f32"], 2), rand((d,), 0.1, DT["f32"], 3, 1.0)
    o = backward(dy, h, w)
    loss = lambda h, w: float((R.f64(dy) * R.rmsnorm(h, w, EPS)).sum())
    for seed in range(5):
        u, v = rand((T, d), 1.0, R.D, 10 + seed), rand((d,), 1.0, R.D, 20 + seed)
        e = 1e-6
        dif_h = (loss(R.f64(h) + e * u, w) - loss(R.f64(h) - e * u, w)) / (2 * e)
        dif_w = (loss(h, R.f64(w) + e * v) - loss(h, R.f64(w) - e * v)) / (2 * e)
        # fp32 gradients against differences whose own error is below 1e-7 of the terms' size
        size = float((R.f64(o["dh"]) * u).abs().sum()), float((R.f64(o["dw"]) * v).abs().sum())
        assert abs(float((R.f64(o["dh"]) * u).sum()) - dif_h) < 1e-6 * size[0]
        assert abs(float((R.f64(o["dw"]) * v).sum()) - dif_w) < 1e-6 * size[1]


def test_offsets_past_32_bits():
    """Close to 2^31 elements of fp32: the first and the last rows of both passes."""
    d = 4096
    T = (1 << 31) // d - 1
    h, w = torch.zeros((T, d), device="cuda"), rand((d,), 0.1, DT["f32"], 3, 1.0)
    ends = [0, 1, T - 2, T - 1]
    rows = rand((4, d), 1.2, DT["f32"], 1)
    h[ends] = rows.cuda()
    y = torch.zeros((T, d), dtype=torch.bfloat16, device="cuda")
    forge.forge_rmsnorm(h, w.cuda(), y=y, eps=EPS)
    check_forward({"y": y[ends].cpu()}, rows, w)
    assert not y[2:T - 2].any()
    dy = y.zero_()
    g = rand((4, d), 1e-2, DT["bf16"], 2)
    dy[ends] = g.cuda()
    dw = torch.empty(d, device="cuda")
    ws = torch.empty(forge.forge_rmsnorm_backward_workspace(T, d), dtype=torch.uint8, device="cuda")
    dx = torch.ones((T, d), dtype=torch.bfloat16, device="cuda")
    forge.forge_rmsnorm_backward(dy, h, w.cuda(), dx=dx, dw=dw, eps=EPS, ws=ws)
    check_backward({"dx": dx[ends].cpu(), "dw": dw.cpu()}, g, rows, w)
    assert not dx[2:T - 2].any()


# ----------------------------------------------------------------------------- streams, graphs, refusals

@pytest.mark.parametrize("d", [72, 1032, 4096])
def test_on_another_stream_and_in_a_graph(d):
    """The same bits on a side stream and from every replay of a captured graph, with inputs
    changed and eager work between the replays."""
    T = 130
    x, w = rand((T, d), 0.5, DT["bf16"], 1).cuda(), rand((d,), 0.1, DT["bf16"], 2, 1.0).cuda()
    r, dy = rand((T, d), 1.0, DT["bf16"], 3).cuda(), rand((T, d), 1e-2, DT["bf16"], 4).cuda()
    e = lambda dt, *s: torch.zeros(s or (T, d), dtype=dt, device="cuda")
    h, y, q, qs, dh = e(r.dtype), e(r.dtype), e(F8), e(torch.float32, T, -(-d // 128)), e(r.dtype)
    dw, ws = e(torch.float32, d), e(torch.uint8, forge.forge_rmsnorm_backward_workspace(T, d))

    def both(h, y, q, qs, dh, dw, ws):
        forge.forge_rmsnorm(x, w, residual=r, h=h, y=y, q=q, q_scale=qs, eps=EPS)
        forge.forge_rmsnorm_backward(dy, h, w, dres=r, dh=dh, dw=dw, eps=EPS, ws=ws)

    outs = (h, y, q, qs, dh, dw)
    other = tuple(torch.zeros_like(t) for t in outs)
    both(*other, torch.zeros_like(ws))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        both(*outs, ws)
    side.synchronize()
    for a, b in zip(outs, other):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(*outs, ws)
    for k in range(3):
        x.copy_(rand((T, d), 0.5 + k, DT["bf16"], 30 + k))
        both(*other, torch.zeros_like(ws))                # eager, with a workspace of its own
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, other):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), f"replay {k}"


def test_refusals():
    x, w = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda"), torch.ones(64, device="cuda")
    y, f = torch.empty_like(x), torch.empty((4, 64), device="cuda")
    run = lambda **k: forge.forge_rmsnorm(**{**dict(x=x, w=w, y=y, eps=EPS), **k})
    for k in (dict(w=w[:32]), dict(y=f), dict(y=y[:2]), dict(residual=x, h=f), dict(x=f, residual=f, h=torch.empty_like(f)),
              dict(q=y), dict(q=torch.empty((4, 64), dtype=F8, device="cuda"), q_scale=torch.empty(5, device="cuda")),
              dict(x=x.t())):
        with pytest.raises(ValueError):
            run(**k)
    with pytest.raises(TypeError):
        run(x=x.half())
    for k, name in ((dict(y=None), "FORGE_ERR_NULL_POINTER"), (dict(residual=x.clone()), "FORGE_ERR_NULL_POINTER"),
                    (dict(eps=0.0), "FORGE_ERR_INVALID_HYPERPARAM"), (dict(y=x), "FORGE_ERR_ALIASING"),
                    (dict(x=x.view(8, 32)[1:, :].reshape(-1)[4:196].view(3, 64), y=y[:3]), "FORGE_ERR_MISALIGNED"),
                    (dict(x=torch.zeros((4, 60), dtype=x.dtype, device="cuda"), w=w[:60],
                          y=torch.empty((4, 60), dtype=x.dtype, device="cuda")), "FORGE_ERR_UNSUPPORTED_SHAPE")):
        with pytest.raises(forge.ForgeError) as e:
            run(**k)
        assert e.value.name == name, k
    dw = torch.empty(64, device="cuda")
    need = forge.forge_rmsnorm_backward_workspace(4, 64)
    back = lambda **k: forge.forge_rmsnorm_backward(**{**dict(dy=x, h=f, w=w, dh=torch.empty_like(f), dw=dw, eps=EPS,
                                                              ws=torch.empty(need, dtype=torch.uint8, device="cuda")), **k})
    back()
    for k in (dict(ws=torch.empty(need - 1, dtype=torch.uint8, device="cuda")), dict(ws=None), dict(dh=x.clone()),
              dict(dw=dw[:8]), dict(dres=x), dict(dx=f.clone())):
        with pytest.raises(ValueError):
            back(**k)
    torch.cuda.synchronize()
