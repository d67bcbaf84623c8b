"""GELU and its slope where the gate is negative and the normal distribution
function small (run with -m gpu).  One input that is 1 and one up weight make
every gate an exact value of the tensors' type, so what is left is the
activation's own error, held relative to the value: the argument g / sqrt(2) and
g^2 / 2 are rounded to fp32, which the tail magnifies by at most g^2, and the
functions are good to a few ulp: (g^2 + 16) 2^-23, beside the result's rounding."""
import math

import pytest
import torch

import paper_2003_04296_amd as q

pytestmark = pytest.mark.gpu

E = 2.0 ** -23
# type, its rounding, lowest gate, the other factor (which keeps the results among the normal values)
TYPES = [(torch.float16, 2.0 ** -11, -4.5, 2.0 ** 11), (torch.bfloat16, 2.0 ** -8, -12.0, 1.0)]


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    q.lib()
    return torch.device("cuda:0")


def _gates(dtype, low, dev):
    return torch.cat((torch.linspace(low, 0, 301, device=dev), torch.linspace(0, 8, 100, device=dev))).to(dtype)


@pytest.mark.parametrize("dtype,unit,low,factor", TYPES)
@pytest.mark.parametrize("m", [1, 20, 200])
def test_value(dev, m, dtype, unit, low, factor):
    g = _gates(dtype, low, dev)
    x = torch.ones((m, 1), dtype=dtype, device=dev)
    h, _ = q.ffn_forward(x, g[:, None].contiguous(), torch.full((len(g), 1), factor, dtype=dtype, device=dev), q.ACT_GELU)
    g = g.double()
    want = g * 0.5 * torch.erfc(-g / math.sqrt(2)) * factor
    assert bool(((h.double() - want).abs() <= (1.01 * unit + (g * g + 16) * E) * want.abs()).all())


@pytest.mark.parametrize("dtype,unit,low,factor", TYPES)
def test_slope(dev, dtype, unit, low, factor):
    """The gate weights' gradient for one token that is 1 is the slope itself."""
    g = _gates(dtype, low, dev)
    x = torch.ones((1, 1), dtype=dtype, device=dev)
    wg, wu = g[:, None].contiguous(), torch.full((len(g), 1), factor, dtype=dtype, device=dev)
    _, pre = q.ffn_forward(x, wg, wu, q.ACT_GELU, keep_pre=True)
    got = q.ffn_backward(x, wg, wu, pre, torch.ones((1, len(g)), dtype=dtype, device=dev), q.ACT_GELU)[1][:, 0].double()
    g = g.double()
    cdf, rest = 0.5 * torch.erfc(-g / math.sqrt(2)), g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    want = (cdf + rest) * factor
    assert bool(((got - want).abs() <= 1.01 * unit * want.abs() + (g * g + 16) * E * (cdf + rest.abs()) * factor).all())
