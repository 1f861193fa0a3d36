"""More tiles than CTA pairs: barriers, phases and accumulators carried over several units of a pair, whole tiles followed by halves."""
import pytest
import torch

from paper_2505_07004_b200 import api as libgq
from test_gpu_linear import check_backward, check_forward

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available()
    return torch.device("cuda:0")


# contractions of two to nine k-steps of 64: fewer than the ring's four stages, as many, more, and no multiple
KDIMS = [72, 200, 264, 520]
# tokens (the last tile of 512 has one half or two) and rows: 5, 9, 11 and 12 row tiles of 256 times 17 token tiles are 85, 153, 187 and
# 204 tiles; 74 pairs take 11, 5, 39 and 56 of them in the last round, the first two of these as halves
SHAPES = [(8200, 2248), (8492, 2248), (8492, 2816), (8200, 3064), (8492, 1096)]


def several_rounds(dev, n, rows):
    """A pair is two SMs, so there are at most half as many pairs as SMs: some pair has a second unit."""
    tiles = ((n + 511) // 512) * ((rows + 255) // 256)
    assert tiles > torch.cuda.get_device_properties(dev).multi_processor_count // 2, tiles


@pytest.mark.parametrize("kdim", KDIMS)
@pytest.mark.parametrize("n,rows", SHAPES)
def test_forward_over_several_units(dev, n, rows, kdim):
    several_rounds(dev, n, rows)
    check_forward(dev, n, kdim, rows, 16 if kdim in (72, 264) else 7, torch.bfloat16, libgq.GQ_ACT_SILU, True, True, 8, seed=kdim)


@pytest.mark.parametrize("kdim", KDIMS)
@pytest.mark.parametrize("n,rows", SHAPES)
def test_backward_over_several_units(dev, n, rows, kdim):
    """The rows are the inputs' features here and the contraction goes over the channels.  (The gradient of the levels has a unit per 256
    features and 1024 tokens: 9 times 5 to 12.)"""
    several_rounds(dev, n, rows)
    check_backward(dev, n, rows, kdim, 16 if kdim in (72, 264) else 7, torch.float16, libgq.GQ_ACT_GELU, 8, seed=kdim)


def test_units_repeat_themselves(dev):
    """The same bits every time, whatever runs beside it."""
    n, d_in, d_out, m = 8492, 520, 2248, 16
    gen = torch.Generator(device=dev).manual_seed(1)
    Q = torch.randint(0, m, (d_out, d_in), generator=gen, device=dev, dtype=torch.uint8)
    codes, table = libgq.gq_linear_pack(Q, 0.1 * torch.randn(d_out, m, generator=gen, device=dev))
    X = torch.randn(n, d_in, generator=gen, device=dev).bfloat16()
    R = torch.randn(n, d_out, generator=gen, device=dev).bfloat16()
    ws = libgq.alloc_workspace(libgq.gq_linear_grad_workspace_bytes(n, d_in, d_out), dev)

    def chain():
        Y = libgq.gq_linear(X, codes, table, m, activation=libgq.GQ_ACT_GELU, residual=R)
        return [Y] + list(libgq.gq_linear_grad(Y, X, codes, table, m, ws, Z=R, activation=libgq.GQ_ACT_GELU))
    want = [t.clone() for t in chain()]
    side = torch.cuda.Stream()
    for _ in range(10):
        with torch.cuda.stream(side):
            torch.randn(1 << 22, device=dev).sort()
        assert all(torch.equal(a, b) for a, b in zip(want, chain()))
    torch.cuda.synchronize()
    libgq.gq_check()
