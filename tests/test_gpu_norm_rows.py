"""forge_rmsnorm and its gradient where workgroups take several rows in turn, rows wider than registers
hold, and every row's share of dw.

For dw the rows are +-1/2 with eps = 3/4, whose norm is exactly 1 (the mean, 1/4, is off by less than
a quarter step of 1), and dy is of the row's sign and 1, 2 or 3 times 2^-7: each term of dw is a
multiple of 2^-8, at most 3 of them, and every partial sum of fewer than 2^22 rows is exact in fp32.
dw must be the sum to the bit: a row left out or taken twice anywhere shows.
"""
import pytest
import torch

import ops_ref as R
from paper_2606_22932_amd import forge
from test_gpu_norm import DT, EPS, F8, Guarded, check_forward, forward, rand

pytestmark = pytest.mark.gpu


def _say(*a):
    print(*a, flush=True)


# ----------------------------------------------------------------------------- forward

@pytest.mark.parametrize("T,d", [(3, 32776), (5, 65544)], ids=str)
@pytest.mark.parametrize("h,w,res,group", [("bf16", "f32", True, 0), ("f32", "bf16", True, 128), ("f32", "f32", False, 0),
                                           ("bf16", "bf16", False, 128), ("bf16", "bf16", True, None)], ids=str)
def test_forward_of_several_wide_rows(T, d, h, w, res, group):
    _say("rmsnorm", T, d, h, w, res, group)
    x = rand((T, d), 0.5, DT["bf16"] if res else DT[h], seed=d)
    g = rand((d,), 0.1, DT[w], seed=d + 1, mean=1.0)
    r = rand((T, d), 1.0, DT[h], seed=d + 2) if res else None
    check_forward(forward(x, g, r, group=group), x, g, r, group=group)


@pytest.mark.parametrize("T,d", [(70000, 8), (5001, 256), (17001, 520), (8300, 1032), (515, 4096)], ids=str)
@pytest.mark.parametrize("h", ["bf16", "f32"])
def test_forward_row_scales_of_many_rows(T, d, h):
    _say("rmsnorm row scales", T, d, h)
    x, g, r = rand((T, d), 0.5, DT["bf16"], 1), rand((d,), 0.1, DT["f32"], 2, 1.0), rand((T, d), 1.0, DT[h], 3)
    check_forward(forward(x, g, r, group=0), x, g, r, group=0)


@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("T,d,h", [(8209, 8200, "bf16"), (8200, 16384, "bf16"), (8209, 8200, "f32")], ids=str)
def test_forward_second_turn_of_wide_rows(T, d, h, group):
    """Every row as in calls of 1000 rows, which take one turn."""
    _say("rmsnorm second turn", T, d, h, group)
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((T, d), generator=gen, device="cuda").to(torch.bfloat16)
    r = torch.randn((T, d), generator=gen, device="cuda").to(DT[h])
    g = rand((d,), 0.1, DT["f32"], 2, 1.0).cuda()
    e = lambda n: dict(h=torch.zeros_like(r[:n]), y=torch.zeros_like(x[:n]), q=torch.zeros((n, d), dtype=F8, device="cuda"),
                       q_scale=torch.zeros((n, -(-d // 128)) if group else (n,), device="cuda"))
    o = e(T)
    forge.forge_rmsnorm(x, g, residual=r, eps=EPS, **o)
    for a in range(0, T, 1000):
        b = min(a + 1000, T)
        p = e(b - a)
        forge.forge_rmsnorm(x[a:b], g, residual=r[a:b], eps=EPS, **p)
        for k in o:
            assert torch.equal(o[k][a:b].view(torch.uint8), p[k].view(torch.uint8)), (k, a)
    last = slice(T - 9, T)
    check_forward({k: t[last].cpu() for k, t in o.items()}, x[last].cpu(), g.cpu(), r[last].cpu(), group=group)


# ----------------------------------------------------------------------------- gradient

ONE_GROUP = [(64, 256), (128, 72), (256, 64), (200, 8), (32, 504), (16, 520), (8, 1032), (4, 4096), (3, 16384)]
TURNS = [(70001, 8), (70001, 64), (20011, 256), (10007, 504), (10007, 520), (5003, 1032), (2600, 4096), (700, 8200),
         (520, 16384)]
WIDE = [(600, 16392), (1030, 16392), (515, 40960)]


@pytest.mark.parametrize("T,d", ONE_GROUP + TURNS + WIDE, ids=str)
@pytest.mark.parametrize("h,w,res,out", [("bf16", "bf16", True, "dh"), ("f32", "f32", True, "dhdx"), ("f32", "bf16", False, "dx")],
                         ids=str)
def test_every_row_of_dw(T, d, h, w, res, out):
    _say("rmsnorm_backward", T, d, h, w, res, out)
    gen = torch.Generator().manual_seed(T + d)
    sign = torch.randint(0, 2, (T, d), generator=gen) * 2 - 1
    count = torch.randint(1, 4, (T, d), generator=gen)
    x, dy, g = (0.5 * sign).to(DT[h]), (sign * count * 2.0 ** -7).to(torch.bfloat16), rand((d,), 0.1, DT[w], 3, 1.0)
    dres = rand((T, d), 1e-2, DT[h], 4) if res else None
    new = Guarded()
    o = {"dw": new((d,), torch.float32)}
    for k, dt in (("dh", DT[h]), ("dx", torch.bfloat16)):
        if k in out:
            o[k] = new((T, d), dt)
    ws = new((forge.forge_rmsnorm_backward_workspace(T, d),), torch.uint8).fill_(0xFF)
    given = [t.cuda() for t in (dy, x, g)] + ([dres.cuda()] if res else [])
    keep = [t.clone() for t in given]
    forge.forge_rmsnorm_backward(*given[:3], dres=given[3] if res else None, eps=0.75, ws=ws, **o)
    new.check()
    for t, k in zip(given, keep):
        assert torch.equal(t.view(torch.uint8), k.view(torch.uint8)), "an input changed"
    want = count.sum(0).to(torch.float64) * 2.0 ** -8
    assert torch.equal(R.f64(o["dw"]), want), (R.f64(o["dw"]) - want).abs().max()
    dh, size, _, _ = R.rmsnorm_backward(dy, x, g, 0.75, dres)
    for k in ("dh", "dx"):
        if k in o:
            R.stored(o[k].cpu(), dh, 3 * R.sums(d) * size + R.TINY, k)


@pytest.mark.parametrize("T,d", [(3, 64), (5, 520), (2, 4096), (1, 16392)], ids=str)
def test_rows_of_zeros_with_the_least_eps(T, d):
    """1 / sqrt(eps) is 2^63: zeros give zeros, dh = dres + dy w 2^63, and dw is zero."""
    x, g = torch.zeros((T, d), device="cuda"), rand((d,), 0.1, DT["f32"], 3, 1.0).cuda()
    dy, y, dh, dw = rand((T, d), 1.0, DT["bf16"], 1).cuda(), rand((T, d), 1.0, DT["bf16"], 2).cuda(), torch.ones_like(x), torch.ones_like(g)
    forge.forge_rmsnorm(x, g, y=y, eps=2.0 ** -126)
    ws = torch.full((forge.forge_rmsnorm_backward_workspace(T, d),), 0xFF, dtype=torch.uint8, device="cuda")
    forge.forge_rmsnorm_backward(dy, x, g, dh=dh, dw=dw, eps=2.0 ** -126, ws=ws)
    assert not y.any() and not dw.any()
    want = R.f64(dy) * R.f64(g) * 2.0 ** 63
    R.stored(dh.cpu(), want, 8 * R.U * want.abs(), "dh")
