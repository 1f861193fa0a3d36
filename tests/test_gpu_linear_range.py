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


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("n", [1, 12, 40, 600])
@pytest.mark.parametrize("act", ACTS)
def test_activation_of_every_value(dev, dtype, n, act):
    """The pre-activation is the bias where X is zero, so a channel can have any value.  SiLU: an exponential good to (2 + 1.2 |z|) units in
    the last place, a sum and a quotient, and 0 instead of numbers smaller than |z| 2^-126.  GELU: z / 2 times what is good to 5 u."""
    bias = all_values(dev, DT[dtype])
    d_out = bias.numel()
    codes = torch.zeros(d_out, 16, dtype=torch.uint8, device=dev)
    table = torch.zeros(d_out, 16, dtype=DT[dtype], device=dev)
    X, Z = torch.zeros(n, 8, device=dev, dtype=DT[dtype]), torch.empty(n, d_out, device=dev, dtype=DT[dtype])
    Y = libgq.gq_linear(X, codes, table, 16, bias=bias, activation=act, Z=Z)
    libgq.gq_check()
    assert torch.equal(Z, bias.expand(n, d_out)) and torch.equal(Y, Y[:1].expand(n, d_out))
    z = bias.double()
    y = torch.where(z < -800.0, 0.0, torch.where(z > 800.0, z if act != libgq.GQ_ACT_NONE else 0.0, act64(z.clamp(-800.0, 800.0), act)))
    if act == libgq.GQ_ACT_NONE:
        y = z
    tol = torch.zeros_like(z)
    if act == libgq.GQ_ACT_SILU:
        tol = 2 * U * ((2 + 1.2 * z.abs()) * torch.sigmoid(-z) + 5) * y.abs() + torch.where(z < 0, z.abs().clamp_max(200.0) * 2.0 ** -126, 0.0)
    elif act == libgq.GQ_ACT_GELU:
        tol = 0.5 * z.abs().clamp_max(15.0) * 5 * U + 4 * U * y.abs()
    within(Y[0], y, rounded(y, tol, DT[dtype]))


@pytest.mark.parametrize("n", [1, 40])
def test_activation_of_infinities(dev, n):
    """ReLU has its limits; SiLU and GELU are 0 times infinity at minus infinity, which is NaN, as in torch."""
    bias = torch.tensor([float("inf"), float("-inf"), float("nan")] * 8, device=dev).bfloat16()
    codes, table = torch.zeros(24, 16, dtype=torch.uint8, device=dev), torch.zeros(24, 16, dtype=torch.bfloat16, device=dev)
    X = torch.zeros(n, 8, device=dev, dtype=torch.bfloat16)
    for act in ACTS:
        Y = libgq.gq_linear(X, codes, table, 16, bias=bias, activation=act).float()
        assert bool((Y[:, 0::3] == float("inf")).all()) and bool(Y[:, 2::3].isnan().all())
        if act in (libgq.GQ_ACT_NONE, libgq.GQ_ACT_RELU):
            assert bool((Y[:, 1::3] == (0.0 if act == libgq.GQ_ACT_RELU else float("-inf"))).all())
        else:
            assert bool(Y[:, 1::3].isnan().all())
    libgq.gq_check()


def same(a, b):
    return torch.equal(a.view(torch.int16) if a.element_size() == 2 else a, b.view(torch.int16) if b.element_size() == 2 else b)


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("n,d_in,d_out", [(2, 200, 72), (7, 200, 312), (15, 136, 264), (40, 200, 312), (300, 2056, 264), (700, 264, 2056)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_one_token_that_is_no_number(dev, dtype, n, d_in, d_out, bad):
    """The other tokens' rows, and the other channels' sums, are what they are without it, bit for bit."""
    act, m, at, j = libgq.GQ_ACT_SILU, 16, n // 2, d_out // 3
    gen, Q, codebook, codes, table, W = layer(dev, d_in, d_out, m, DT[dtype], n)
    X = torch.randn(n, d_in, generator=gen, device=dev).to(DT[dtype])
    dY, Z = (torch.randn(n, d_out, generator=gen, device=dev).to(DT[dtype]) for _ in range(2))
    ws = libgq.alloc_workspace(libgq.gq_linear_grad_workspace_bytes(n, d_in, d_out), dev)
    rest, others = [i for i in range(n) if i != at], [c for c in range(d_out) if c != j]

    def forward(X):
        z = torch.empty(n, d_out, device=dev, dtype=X.dtype)
        return libgq.gq_linear(X, codes, table, m, activation=act, Z=z), z
    X2 = X.clone()
    X2[at, ::3] = bad
    for a, b in zip(forward(X), forward(X2)):
        assert same(a[rest], b[rest]) and not bool(b[at].isfinite().any())

    def backward(dY, Z):
        return libgq.gq_linear_grad(dY, X, codes, table, m, ws, Z=Z, activation=act)
    want = backward(dY, Z)
    for which in range(2):
        pair = [dY.clone(), Z.clone()]
        pair[which][at, j] = bad
        got = backward(*pair)
        libgq.gq_check()
        assert same(got[0][rest], want[0][rest]) and same(got[1][rest], want[1][rest])
        assert torch.equal(got[2][others], want[2][others]) and torch.equal(got[3][others], want[3][others])
        assert not bool(got[3][j].isfinite())
