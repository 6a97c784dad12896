"""E4M3 codes next to the border of two: they and their scales are those of IEEE fp32 operations,
for scales of every size (values chosen so that the quotient's last bit decides)."""
import pytest
import torch

from paper_2606_22932_amd import forge

pytestmark = pytest.mark.gpu

F8, F32 = torch.float8_e4m3fn, torch.float32
RECIP = torch.tensor(1.0 / 448.0, dtype=F32)
LOW = 2.0 ** -126


def steps(x, n):
    """x n steps of fp32 further from zero."""
    return (x.view(torch.int32) + n).view(F32)


def scale_of(amax):
    s = amax * RECIP
    return torch.where(s < LOW, torch.zeros_like(s), s)


def borders(exponents, count, size, seed):
    """Rows of `size` values: the largest, 2^exponent times a random mantissa, then the middles of two
    neighbouring codes times the row's scale, up to a step off, of either sign."""
    g = torch.Generator().manual_seed(seed)
    codes = torch.arange(0x7F, dtype=torch.uint8).view(F8).float()
    mid = (codes[1:] + codes[:-1]) / 2
    rows = []
    for e in exponents:
        top = (torch.rand((count, 1), generator=g) + 1).clamp_max(2 - 2.0 ** -23) * 2.0 ** e
        x = scale_of(top) * mid[torch.randint(0, len(mid), (count, size - 1), generator=g)]
        x = torch.where(x > 0, steps(x, torch.randint(-1, 2, x.shape, generator=g, dtype=torch.int32)), x)
        x = torch.minimum(x, top) * (torch.randint(0, 2, x.shape, generator=g) * 2 - 1)
        rows.append(torch.cat([top, x], 1))
    return torch.cat(rows)


def codes_of(x):
    """IEEE fp32: scale = amax RN(1/448), code of x / scale."""
    s = scale_of(x.abs().amax(-1, keepdim=True))
    q = torch.where(s > 0, x / s, torch.zeros_like(x)).clamp(-448, 448).to(F8)
    return q, s[:, 0]


EXPONENTS = [-118, -117, -116, -114, -112, -110, -106, -100, -90, -60, -55, -20, 0, 30, 100, 126]


def same(got, want, x, what):
    got, want = got.cpu().view(torch.uint8).view(x.shape), want.view(torch.uint8).view(x.shape)
    off = (got != want).nonzero()
    assert not len(off), (what, len(off), x[tuple(off[0])].item(), x[off[0][0], 0].item())


def test_state_codes_at_borders():
    """beta1 = 0 and cold state: m' is the gradient itself."""
    x = borders(EXPONENTS, 500, 64, 1)
    n = x.numel()
    w, m, v = torch.zeros(n), torch.zeros(n).to(F8), torch.zeros(n).to(F8)
    t = [w.cuda(), x.flatten().cuda(), m.cuda(), v.cuda(), torch.zeros(n // 64).cuda(), torch.zeros(n // 64).cuda()]
    forge.forge_adamw_multi(forge.TensorList([t]), lr=0.0, beta1=0.0, beta2=0.999, eps=1e-8, step=1)
    q, s = codes_of(x)
    assert torch.equal(t[4].cpu(), s), "scales"
    same(t[2], q, x, "codes")


def test_state_of_a_block_with_an_infinite_value():
    """Its scale is Inf, the codes of its finite values zero: none decodes to a finite number."""
    x = torch.ones(3, 64)
    x[1, 5] = float("inf")
    t = [torch.zeros(192).cuda(), x.flatten().cuda(), torch.zeros(192).to(F8).cuda(), torch.zeros(192).to(F8).cuda(),
         torch.zeros(3).cuda(), torch.zeros(3).cuda()]
    forge.forge_adamw_multi(forge.TensorList([t]), lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
    s = t[4].cpu()
    assert torch.isinf(s[1]) and torch.isfinite(s[[0, 2]]).all() and torch.isinf(t[5].cpu()[1])
    m = t[2].float().cpu().view(3, 64)
    keep = torch.arange(64) != 5
    assert not m[1, keep].any() and bool((m[[0, 2]] == 448).all())
    assert not torch.isfinite(m[1] * s[1]).any() and not torch.isfinite(t[3].float().cpu().view(3, 64)[1] * t[5].cpu()[1]).any()


@pytest.mark.parametrize("w", [torch.bfloat16, F32], ids=["bf16", "f32"])
def test_state_of_bf16_gradients_to_the_bit(w):
    """bf16 gradients beside bf16 weights (eight elements a thread) and fp32 ones (four), over several
    steps from cold state, with blocks of zeros, of tiny numbers and of very large ones, and a short
    last block: codes and scales are those of plain fp32 arithmetic."""
    n = 200035
    gen = torch.Generator().manual_seed(17)
    f = lambda x: torch.tensor(x, dtype=F32)
    b1, b2 = f(0.9), f(0.999)
    c1, c2, coef = f(1 - float(b1)), f(1 - float(b2)), f(0.37)
    zero = lambda dt, k=n: torch.zeros(k, dtype=dt, device="cuda")
    t = [zero(w), zero(torch.bfloat16), zero(F8), zero(F8), zero(F32, -(-n // 64)), zero(F32, -(-n // 64))]
    lst = forge.TensorList([t])
    pad = -n % 64
    blocks = lambda x: torch.nn.functional.pad(x, (0, pad)).view(-1, 64)
    q = {k: torch.zeros(n + pad).to(F8).view(-1, 64) for k in "mv"}
    s = {k: torch.zeros(-(-n // 64)) for k in "mv"}
    for step in range(1, 5):
        g = (torch.randn(n, generator=gen) * 10.0 ** -step).to(torch.bfloat16)
        g[:640], g[640:1280], g[1280:1920] = 0.0, 1e-21, 1e15
        t[1].copy_(g)
        forge.forge_adamw_multi(lst, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=step, grad_scale=coef.view(1).cuda())
        x = blocks(g.float() * coef)
        m, r = q["m"].float() * s["m"][:, None], q["v"].float() * s["v"][:, None]
        m, v = b1 * m + c1 * x, b2 * (r * r) + c2 * (x * x)
        root = v.double().sqrt().float()                  # the fp64 root, rounded once more, is the fp32 root
        q["m"], s["m"] = codes_of(m)
        code, s["v"] = codes_of(root)
        q["v"] = torch.where(root > 0, code.float().clamp_min(2.0 ** -9), code.float()).to(F8)
        for k, c, e in (("m", t[2], t[4]), ("v", t[3], t[5])):
            assert torch.equal(e.cpu(), s[k]), (step, k, "scales")
            want = q[k].view(torch.uint8).view(-1)[:n]
            assert torch.equal(c.cpu().view(torch.uint8), want), (step, k, "codes")
