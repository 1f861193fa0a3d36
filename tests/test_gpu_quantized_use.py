"""QuantizedLinear as part of a model."""
import copy

import pytest
import torch

from paper_2505_07004_b200 import api as libgq
from paper_2505_07004_b200.capture import GuidedHessianCapture
from paper_2505_07004_b200.loss import end_loss
from paper_2505_07004_b200.quantized import QuantizedLinear, quantise

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


class Net(torch.nn.Module):
    def __init__(self):
        super().__init__()
        self.embed = torch.nn.Embedding(96, 64)
        self.up = torch.nn.Linear(64, 128)
        self.down = torch.nn.Linear(128, 64, bias=False)
        self.head = torch.nn.Linear(64, 96, bias=False)

    def forward(self, ids):
        h = self.embed(ids)
        return self.head(h + self.down(torch.nn.functional.silu(self.up(h))))


@pytest.mark.parametrize("model_dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("layer_dtype", [torch.bfloat16, torch.float16])
def test_layers_of_a_model_of_another_type(dev, model_dtype, layer_dtype):
    """A layer that takes a torch.nn.Linear's place returns that layer's type, so that the layers behind it find what they did."""
    torch.manual_seed(1)
    net = Net().to(dev)
    batches = [(torch.randint(0, 96, (2, 33), device=dev), torch.randint(0, 96, (2, 33), device=dev))]
    H = GuidedHessianCapture({"up": net.up, "down": net.down}, 2).calibrate(net, batches)
    net = net.to(model_dtype)
    for name in ("up", "down"):
        setattr(net, name, quantise(getattr(net, name), H[name], dtype=layer_dtype))
    logits = net(batches[0][0])
    assert logits.dtype == model_dtype and net.up(net.embed(batches[0][0])).dtype == model_dtype
    end_loss(logits, batches[0][1]).backward()
    assert net.embed.weight.grad.dtype == model_dtype and bool(net.embed.weight.grad.isfinite().all())
    for other in (torch.float32, torch.bfloat16):         # and follows the model
        assert net.to(other)(batches[0][0]).dtype == other
    assert QuantizedLinear(torch.zeros(8, 8, dtype=torch.uint8, device=dev), torch.zeros(8, 4, device=dev), dtype=layer_dtype)(
        torch.zeros(1, 8, device=dev)).dtype == layer_dtype      # by itself: its own type
    libgq.gq_check()


@pytest.mark.parametrize("train_levels", [False, True])
@pytest.mark.parametrize("act", [libgq.GQ_ACT_NONE, libgq.GQ_ACT_GELU])
def test_inputs_are_kept_only_for_the_levels_gradient(dev, train_levels, act):
    layer = make(dev, train_levels=train_levels, act=act)
    layer.bias.requires_grad_(True)
    x = torch.randn(3, 5, 72, device=dev).bfloat16().requires_grad_()
    kept = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(tuple(t.shape)) or t, lambda t: t):
        y = layer(x)
    assert ((15, 72) in kept) == train_levels and ((15, 40) in kept) == (act != libgq.GQ_ACT_NONE)
    y.backward(torch.ones_like(y))
    # the same gradients from the call itself, which is given X
    dY, X = torch.ones(15, 40, device=dev).bfloat16(), x.detach().view(15, 72)
    table = layer.table if not train_levels else layer.make_table(layer.codebook)
    Z = torch.empty_like(dY) if act != libgq.GQ_ACT_NONE else None
    libgq.gq_linear(X, layer.codes, table, layer.m, bias=layer.bias.detach(), activation=act, Z=Z)
    ws = libgq.alloc_workspace(libgq.gq_linear_grad_workspace_bytes(15, 72, 40), dev)
    _, dX, d_table, d_bias = libgq.gq_linear_grad(dY, X, layer.codes, table, layer.m, ws, Z=Z, activation=act)
    assert torch.equal(x.grad.view(15, 72), dX) and torch.equal(layer.bias.grad, d_bias.bfloat16())
    assert not train_levels or torch.equal(layer.codebook.grad, d_table)
    without = libgq.gq_linear_grad(dY, None, layer.codes, table, layer.m, ws, Z=Z, activation=act, need_table=False, d_in=72)
    assert torch.equal(without[1], dX) and without[2] is None and torch.equal(without[3], d_bias)
    libgq.gq_check()


def test_gradients_without_inputs_refuse(dev):
    layer = make(dev)
    dY = torch.ones(3, 40, device=dev).bfloat16()
    ws = libgq.alloc_workspace(libgq.gq_linear_grad_workspace_bytes(3, 72, 40), dev)
    with pytest.raises(ValueError, match="X"):
        libgq.gq_linear_grad(dY, None, layer.codes, layer.table, 16, ws, d_in=72)
    with pytest.raises(ValueError, match="d_in"):
        libgq.gq_linear_grad(dY, None, layer.codes, layer.table, 16, ws, need_table=False)
    with pytest.raises(ValueError, match="d_in"):
        libgq.gq_linear_grad(dY, torch.ones(3, 72, device=dev).bfloat16(), layer.codes, layer.table, 16, ws, d_in=80)
    with pytest.raises(ValueError, match="codes"):
        libgq.gq_linear_grad(dY, None, layer.codes, layer.table, 16, ws, need_table=False, d_in=104)
    with pytest.raises(ValueError, match="table"):
        libgq.gq_linear_grad(dY.half(), None, layer.codes, layer.table, 16, ws, need_table=False, d_in=72)


def test_no_pre_activation_without_a_graph(dev, monkeypatch):
    """An evaluation under no_grad neither allocates nor writes what only a backward pass reads."""
    layer = make(dev, train_levels=True)
    x = torch.randn(6, 72, device=dev).bfloat16().requires_grad_()
    given, call = [], libgq.gq_linear
    monkeypatch.setattr(libgq, "gq_linear", lambda *a, **k: given.append(k.get("Z")) or call(*a, **k))
    want = layer(x)
    with torch.no_grad():
        got = layer(x)
    with torch.inference_mode():
        again = layer(x.detach())
    assert given[0] is not None and given[1] is None and given[2] is None
    assert torch.equal(got, want) and torch.equal(again, want) and not got.requires_grad


def test_calibration_on_an_iterator(dev):
    """Both passes see the batches of a generator too."""
    torch.manual_seed(2)
    net = Net().to(dev).bfloat16()
    batches = [(torch.randint(0, 96, (b, 17), device=dev), torch.randint(0, 96, (b, 17), device=dev)) for b in (3, 2, 1)]
    names = ("up", "down")
    want = GuidedHessianCapture({k: getattr(net, k) for k in names}, 4).calibrate(net, batches)
    for once in (iter(batches), (b for b in batches), zip([b[0] for b in batches], [b[1] for b in batches])):
        got = GuidedHessianCapture({k: getattr(net, k) for k in names}, 4).calibrate(net, once)
        assert set(got) == set(names)
        for k in names:
            # sums over the batches' tokens in the same order, but for the order of two writers of a tile
            assert bool(((got[k] - want[k]).abs() <= 2.0 ** -16 * want[k].diagonal(dim1=1, dim2=2).amax(1)[:, None, None]).all())


def test_a_layer_without_a_forward_pass_is_an_error(dev):
    torch.manual_seed(2)
    net = Net().to(dev).bfloat16()
    cap = GuidedHessianCapture({"up": net.up, "down": net.down}, 4)
    ids, targets = torch.randint(0, 96, (2, 17), device=dev), torch.randint(0, 96, (2, 17), device=dev)
    with cap.saliency_pass():
        end_loss(net(ids), targets).backward()
    with pytest.raises(RuntimeError, match="saliency blocks but 0 forward calls"):
        cap.finalize()
    with cap.hessian_pass(), torch.no_grad():
        net.up(net.embed(ids))
    with pytest.raises(RuntimeError, match="down"):
        cap.finalize()
