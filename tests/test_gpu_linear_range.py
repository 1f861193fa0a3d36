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


@pytest.mark.parametrize("d_in", [264, 8, 128])
def test_infinite_gradients_leave_unused_levels_alone(dev, d_in):
    """A level that no weight has gets no gradient, an infinite dZ in its channel or not: nothing of what fills a tile up reaches it."""
    n, d_out, m = 6, 40, 4
    gen, Q, codebook, codes, table, W = layer(dev, d_in, d_out, m, torch.float16, 2)
    Q.clamp_min_(1)                                       # the code of the padding; no weight has it
    Q[:, 0], Q[:, 1] = 1, 2
    Q[:, 2:][Q[:, 2:] == 3] = 1                           # nor level 3
    codes, table = libgq.gq_linear_pack(Q, codebook, torch.float16)
    X = torch.rand(n, d_in, generator=gen, device=dev).add_(0.5).half()
    dY = torch.randn(n, d_out, generator=gen, device=dev).half()
    ws = libgq.alloc_workspace(libgq.gq_linear_grad_workspace_bytes(n, d_in, d_out), dev)
    want = libgq.gq_linear_grad(dY, X, codes, table, m, ws, need_x=False)
    dY[2, 7], dY[4, 30] = float("inf"), float("-inf")
    got = libgq.gq_linear_grad(dY, X, codes, table, m, ws, need_x=False)
    libgq.gq_check()
    for j, value in ((7, float("inf")), (30, float("-inf"))):
        assert got[2][j].tolist() == [0.0, value, value, 0.0] and float(got[3][j]) == value
    rest = [j for j in range(d_out) if j not in (7, 30)]
    assert torch.equal(got[2][rest], want[2][rest]) and torch.equal(got[3][rest], want[3][rest])
