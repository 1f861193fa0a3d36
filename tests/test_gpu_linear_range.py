"""Activations and their slopes over all values of either 16-bit type, and infinities and NaN in the products' inputs."""
import pytest
import torch

from paper_2505_07004_b200 import api as libgq
from test_gpu_linear import ACTS, DT, act64, layer, rounded, slope64, within

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available()
    return torch.device("cuda:0")


def all_values(dev, dtype):
    """Every finite number of a 16-bit type, once."""
    v = torch.arange(-32768, 32768, device=dev, dtype=torch.int32).to(torch.int16).view(dtype)
    return v[v.isfinite()]


def slope_tolerance(z, act):
    """Of the slope in fp32, derived.  ReLU: none.  SiLU, s (1 + z (1 - s)): the exponential is good to two units in the last place
    (4 u relative), a quotient to two more on top of the sum below it, so s and 1 - s are good to 11 u and the slope to 24 u of
    s (1 + |z| (1 - s)); where the exponential is subnormal its steps are 2^-149, times |z|.  GELU: an error function good to two units
    (2 u times 1/2), its argument's rounding and the sum's (2 u), and z phi(z) <= 0.25 with an exponential (4 u) of a rounded argument, all
    together less than 6 u; where it is saturated nothing of that grows."""
    if act == libgq.GQ_ACT_RELU:
        return torch.zeros_like(z)
    if act == libgq.GQ_ACT_SILU:
        s, rest = torch.sigmoid(z), torch.sigmoid(-z)
        return 24 * U * s * (1 + z.abs() * rest) + z.abs().clamp_max(200.0) * 2.0 ** -148
    return torch.full_like(z, 6 * U)


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("act", [a for a in ACTS if a != libgq.GQ_ACT_NONE])
def test_slope_of_every_value(dev, dtype, act):
    Z = all_values(dev, DT[dtype]).view(-1, 256)
    n, d_out = Z.shape
    gen, Q, codebook, codes, table, W = layer(dev, 8, d_out, 4, DT[dtype], 1)
    X = torch.zeros(n, 8, device=dev, dtype=DT[dtype])
    for size in (1.0, -0.75):
        dY = torch.full_like(Z, size)
        dZ = libgq.gq_linear_grad(dY, X, codes, table, 4, Z=Z, activation=act, need_x=False, need_table=False, need_bias=False)[0]
        libgq.gq_check()
        z = Z.double()
        slope = torch.where(z < -800.0, 0.0, torch.where(z > 800.0, 1.0, slope64(z.clamp(-800.0, 800.0), act)))
        within(dZ, size * slope, rounded(size * slope, abs(size) * slope_tolerance(z, act), DT[dtype]))
