"""Limits of include/forge_ops.h on the host, beside test_ops_boundary.py."""
import pytest

from test_ops_boundary import HYPER, NODEV, grad, no_gpu, norm, some_list, step

LEAST = 2.0 ** -126                        # the smallest normal fp32 number
CALLS = {"rmsnorm": norm, "rmsnorm_backward": grad, "adamw_multi": lambda **k: step(some_list(), **k)}


@pytest.mark.parametrize("call", CALLS)
def test_eps_is_a_normal_number(call):
    """The reciprocal (root) of a subnormal eps is no fp32 number to the hardware: rows of zeros and
    weights without a gradient would become NaN."""
    for eps in (LEAST * (1 - 2.0 ** -23), 1e-40, 2.0 ** -149):
        assert CALLS[call](eps=eps) == HYPER


@no_gpu
@pytest.mark.parametrize("call", CALLS)
def test_the_least_eps(call):
    assert CALLS[call](eps=LEAST) == NODEV
