"""forge_rmsnorm's E4M3 codes next to the border of two: those of the fp32 y divided by its group's
scale in IEEE arithmetic.  Rows of +-1/2 with eps = 3/4 have a norm of exactly 1 (the mean, 1/4,
is off by less than a quarter step of 1), so that y is half the gain to the bit.
"""
import pytest
import torch

from paper_2606_22932_amd import forge
from test_gpu_codes import EXPONENTS, F8, borders, codes_of, same

pytestmark = pytest.mark.gpu


def norm(y, group, stream):
    """Codes and scales of rows of y, one row of gains a call."""
    d = y.shape[1]
    x = torch.full((1, d), 0.5, dtype=stream, device="cuda")
    out = []
    for gain in 2 * y:
        q, s = torch.empty((1, d), dtype=F8, device="cuda"), torch.empty((1, -(-d // 128)) if group else 1, device="cuda")
        forge.forge_rmsnorm(x, gain.cuda(), q=q, q_scale=s, eps=0.75)
        out.append((q.view(torch.uint8), s.flatten()))
    return tuple(torch.cat(t).cpu() for t in zip(*out))


@pytest.mark.parametrize("stream", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [128, 1024, 4096, 40960])
def test_codes_at_borders(d, stream):
    y = borders(EXPONENTS[:-1], 64, 128, 3 + d)
    y[:, 5] = -0.0
    y = y.view(-1, d)
    q, s = norm(y, 128, stream)
    want, scale = codes_of(y.view(-1, 128))
    assert torch.equal(s, scale), "scales"
    same(q, want, y.view(-1, 128), "codes")


@pytest.mark.parametrize("stream", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 520, 4096, 40960])
def test_codes_of_rows_at_borders(d, stream):
    y = borders(EXPONENTS[:-1], 3, d, 5 + d)
    q, s = norm(y, 0, stream)
    want, scale = codes_of(y)
    assert torch.equal(s, scale), "scales"
    same(q, want, y, "codes")
