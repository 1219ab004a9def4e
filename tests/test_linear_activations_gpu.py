"""Relative errors of the activations over all bf16 arguments of their range, through a layer of one input
with weight 1 (its sums are exact).

u = 2^-8 is the rounding of the result. GELU: the fitted polynomial leaves Phi(z) a relative error of 2.2e-3
down to z = -5, and 8e-7 for z >= 0; its arithmetic in float32 adds some units of 2^-24 of an exponent of
up to 22 and of the reciprocal, 1e-5 in all. Below -5 z Phi(z) is off by at most 1.8e-8. SiLU: an exponent of up
to 116 with two roundings of 2^-24, and approximations of 2^-21: 2e-5."""
import pytest
import torch

from paper_2608_11519_gb300 import flarepp
from test_linear_gpu import U, _device, act64  # noqa: F401

pytestmark = pytest.mark.gpu


def arguments(lo, hi):
    """All bf16 numbers from lo to hi of at least 2^-100."""
    z = torch.arange(-32768, 32768, device="cuda").to(torch.int16).view(torch.bfloat16)
    return z[(z >= lo) & (z <= hi) & (z.abs() >= 2.0 ** -100)].view(-1, 1)


def outputs(z, act, rows):
    one = torch.ones(1, 1, dtype=torch.bfloat16, device="cuda")
    parts = z.split(rows) if rows else (z,)
    return torch.cat([flarepp.linear_fwd(p.clone(), one, None, None, act) for p in parts]).double()


@pytest.mark.parametrize("rows", [100, 0])  # the form for few rows, and tiles
@pytest.mark.parametrize("act,lo,hi,off", [("gelu", 0, 40, 1e-5), ("gelu", -5, 0, 2.2e-3 + 1e-5),
                                           ("silu", -80, 40, 2e-5)])
def test_relative_error(act, lo, hi, off, rows):
    z = arguments(lo, hi)
    z = z[::37].contiguous() if rows else z
    y = act64(z.double(), act)
    assert bool(((outputs(z, act, rows) - y).abs() <= (U + off) * y.abs()).all())


def test_gelu_below_minus_five():
    z = arguments(-40, -5)
    y = act64(z.double(), "gelu")
    assert bool(((outputs(z, "gelu", 0) - y).abs() <= U * y.abs() + 1.9e-8).all())
