"""QuantizedLinear as part of a model."""
import copy

import pytest
import torch

from paper_2505_07004_b200 import api as libgq
from paper_2505_07004_b200.quantized import QuantizedLinear

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available()
    return torch.device("cuda:0")


def make(dev, dtype=torch.bfloat16, train_levels=False, act=libgq.GQ_ACT_SILU, d_in=72, d_out=40, m=16):
    gen = torch.Generator(device=dev).manual_seed(d_in + m)
    Q = torch.randint(0, m, (d_out, d_in), generator=gen, device=dev, dtype=torch.uint8)
    codebook = 0.1 * torch.randn(d_out, m, generator=gen, device=dev)
    return QuantizedLinear(Q, codebook, 0.1 * torch.randn(d_out, generator=gen, device=dev), act, dtype, train_levels)


MOVES = [lambda m: m.half(), lambda m: m.bfloat16(), lambda m: m.float(), lambda m: m.to(torch.float64), lambda m: m.to("cuda:0"),
         lambda m: m.to("cuda:0", torch.float16).float(), lambda m: m.cpu().to("cuda:0"), lambda m: copy.deepcopy(m).half()]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("train_levels", [False, True])
@pytest.mark.parametrize("move", range(len(MOVES)))
def test_casting_a_model_leaves_the_layer_its_numbers(dev, dtype, train_levels, move):
    """Module.to and its like change parameters' types; levels, bias and codes of the layer stay what they are."""
    layer = make(dev, dtype, train_levels)
    if train_levels:
        layer.codebook.grad = torch.ones_like(layer.codebook)
    x = torch.randn(9, 72, device=dev).to(dtype)
    want = layer(x).detach()
    kept = {k: (v.dtype, v.clone()) for k, v in layer.state_dict().items()}
    model = MOVES[move](torch.nn.Sequential(layer))
    for k, v in model[0].state_dict().items():
        assert v.dtype == kept[k][0] and torch.equal(v, kept[k][1])
    if train_levels:
        assert model[0].codebook.grad is None or model[0].codebook.grad.dtype == torch.float32
    got = model(x).detach()
    assert torch.equal(got, want.to(got.dtype))
    y = x.clone().requires_grad_()
    model(y).float().sum().backward()
    assert y.grad.dtype == dtype and bool(y.grad.isfinite().all())
    libgq.gq_check()
