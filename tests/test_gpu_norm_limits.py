"""The norm's widest rows: launches of more than 2^32 threads, counts next to 2^31.  Rows are zero but
for a few columns, so that every sum has a few terms and 64-bit results are found from those."""
import pytest
import torch

import ops_ref as R
from paper_2606_22932_amd import forge

pytestmark = pytest.mark.gpu

BF, F8 = torch.bfloat16, torch.float8_e4m3fn
EPS = 0.0625
E = 32 * R.U                              # of at most eight terms and the functions around them: ops_ref.sums


def _say(*a):
    print(*a, flush=True)


def rand(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(BF)


def only(t, cols):
    """No other column of the rows of t holds anything."""
    return int(torch.count_nonzero(t)) == int(torch.count_nonzero(t[..., cols]))


def test_a_row_of_nearly_2_31_columns():
    d = (1 << 31) - 8
    _say("rmsnorm", 1, d)
    cols = torch.tensor([0, 127, 128, 1 << 28, d - 121, d - 120, d - 1])
    x = torch.zeros((1, d), dtype=BF, device="cuda")
    x[0, cols.cuda()] = rand(len(cols), 1).cuda()
    w = torch.ones(d, dtype=BF, device="cuda")
    y, q = torch.full((1, d), 7.0, dtype=BF, device="cuda"), torch.full((1, d), 0x7F, dtype=torch.uint8, device="cuda")
    qs = torch.full((1, 1 << 24), 7.0, device="cuda")
    forge.forge_rmsnorm(x, w, y=y, q=q.view(F8), q_scale=qs, eps=EPS)
    h = R.f64(x[0, cols.cuda()])
    want = h / (h.square().sum() / d + EPS).sqrt()
    R.stored(y[0, cols.cuda()].cpu(), want, E * want.abs() + R.TINY, "y")
    assert only(y, cols.cuda()) and only(q, cols.cuda())
    # the groups that hold the columns: the last, of 120, begins at d - 120 = 2^31 - 128, and d - 121 is
    # of the one before
    at = (cols // 128).unique()
    assert at.tolist() == [0, 1, 1 << 21, (1 << 24) - 2, (1 << 24) - 1]
    top = torch.stack([want[(cols // 128 == k).nonzero()[:, 0]].abs().max() for k in at]) / 448
    R.within(qs[0, at.cuda()], top, (E + 4 * R.U) * top, "scales")
    assert only(qs, at.cuda())


@pytest.mark.parametrize("T,d", [(2, (1 << 30) - 8), (3, (1 << 29) + 8)], ids=str)
def test_gradient_of_rows_past_2_29_columns(T, d):
    _say("rmsnorm_backward", T, d)
    cols = torch.tensor([0, 7, (1 << 28) - 1, 1 << 28, (1 << 28) + 31, d - 9, d - 1])
    at = cols.cuda()
    new = lambda *s: torch.zeros(s, dtype=BF, device="cuda")
    h, dy, w = new(T, d), new(T, d), new(d).fill_(1.0)
    h[:, at], dy[:, at] = rand((T, len(cols)), 2).cuda(), rand((T, len(cols)), 3).cuda()
    dh, dw = new(T, d).fill_(7.0), torch.full((d,), float("nan"), device="cuda")
    ws = torch.full((forge.forge_rmsnorm_backward_workspace(T, d),), 0xFF, dtype=torch.uint8, device="cuda")
    forge.forge_rmsnorm_backward(dy, h, w, dh=dh, dw=dw, eps=EPS, ws=ws)
    x, g = R.f64(h[:, at]), R.f64(dy[:, at])
    s = 1 / (x.square().sum(1, keepdim=True) / d + EPS).sqrt()
    c = s * s * (g * x).sum(1, keepdim=True) / d
    want, size = s * (g - x * c), s * (g.abs() + (x * c).abs())
    R.stored(dh[:, at].cpu(), want, 3 * E * size + R.TINY, "dh")
    t = g * x * s
    R.within(dw[at], t.sum(0), E * t.abs().sum(0) + R.TINY, "dw")
    assert only(dh, at) and only(dw, at)


def test_gradient_of_no_tokens_of_the_widest_rows():
    d = (1 << 31) - 8
    _say("rmsnorm_backward", 0, d)
    e = torch.empty((0, d), dtype=BF, device="cuda")
    w = torch.empty(d, dtype=BF, device="cuda")
    dw = torch.full((d,), 7.0, device="cuda")
    forge.forge_rmsnorm_backward(e, e, w, dh=torch.empty_like(e), dw=dw, eps=EPS, ws=None)
    assert not dw.any()
