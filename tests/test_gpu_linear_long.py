"""Products at the longest dimensions there are, 2^20 inputs or outputs, with the tolerances of test_gpu_linear.py."""
import pytest
import torch

from paper_2505_07004_b200 import api as libgq
from test_gpu_linear import STEP, check_backward, check_forward, layer, rounded, within

pytestmark = pytest.mark.gpu
LONG = 1 << 20


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available()
    return torch.device("cuda:0")


@pytest.mark.parametrize("n", [2, 9, 40, 300])
@pytest.mark.parametrize("d_in,d_out", [(LONG, 72), (LONG - 24, 264), (64, LONG), (136, LONG - 8)])
def test_longest_layers(dev, n, d_in, d_out):
    check_forward(dev, n, d_in, d_out, 16, torch.float16, libgq.GQ_ACT_RELU, True, True, 8)
    torch.cuda.empty_cache()
    check_backward(dev, n, d_in, d_out, 7, torch.bfloat16, libgq.GQ_ACT_RELU, 0)
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n,d_out", [(4, 8192), (32, 8192), (32, 256), (600, 8192)])
def test_sums_of_one_sign(dev, n, d_out):
    """Terms of one sign are the worst case of an accumulation that truncates: K / 16 steps that lose up to 2^-23 of the sum each."""
    d_in = 28672
    gen, Q, codebook, codes, table, W = layer(dev, d_in, 64, 16, torch.float16, 1)
    Q = torch.randint(0, 16, (d_out, d_in), generator=gen, device=dev, dtype=torch.uint8)
    codebook = (0.1 + torch.rand(d_out, 16, generator=gen, device=dev)) * (64 / d_in)
    codes, table = libgq.gq_linear_pack(Q, codebook, torch.float16)
    X = (0.1 + torch.rand(n, d_in, generator=gen, device=dev)).half()
    Y = libgq.gq_linear(X, codes, table, 16)
    libgq.gq_check()
    rows = torch.randperm(d_out, generator=gen, device=dev)[:256]
    z = X.double() @ table[rows].double().gather(1, Q[rows].long()).t()
    within(Y[:, rows], z, rounded(z, (d_in / 16 + 72) * STEP * z, torch.float16))
