"""Layers that compute with the quantiser's result, the end loss under autograd, and a run of them together: a model is calibrated,
quantised, calibrated again through its quantised layers and scored."""
import copy

import numpy as np
import pytest
import torch

from oracle import gq_oracle as orc
from paper_2505_07004_b200 import api as libgq
from paper_2505_07004_b200 import synth
from paper_2505_07004_b200.capture import GuidedHessianCapture
from paper_2505_07004_b200.loss import end_loss, token_logprobs
from paper_2505_07004_b200.quantized import QuantizedLinear, quantise

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available()
    return torch.device("cuda:0")


def near(got, want, tol):
    """Within the tolerance, one rounding to bf16 (2^-8 relative) and 400 steps of fp32 sums of the largest entry."""
    tol = 1.01 * (tol + 2.0 ** -8 * want.abs() + 400 * 2.0 ** -23 * want.abs().max())
    assert bool(((got.double() - want).abs() <= tol).all()), ((got.double() - want).abs() / tol).max().item()


@pytest.mark.parametrize("act,fn", [(libgq.GQ_ACT_NONE, lambda z: z), (libgq.GQ_ACT_GELU, torch.nn.functional.gelu),
                                    (libgq.GQ_ACT_SILU, torch.nn.functional.silu)])
def test_layer_and_its_gradients(dev, act, fn):
    torch.manual_seed(act)
    d_in, d_out, m = 136, 72, 8
    Q = torch.randint(0, m, (d_out, d_in), device=dev, dtype=torch.uint8)
    codebook = (0.1 * torch.randn(d_out, m, device=dev)).bfloat16().float()      # levels that bf16 holds: both sides have the same weights
    layer = QuantizedLinear(Q, codebook, 0.1 * torch.randn(d_out, device=dev), act, train_levels=True)
    x = torch.randn(3, 7, d_in, device=dev).bfloat16().requires_grad_()
    r = torch.randn(3, 7, d_out, device=dev).bfloat16().requires_grad_()
    G = torch.randn(3, 7, d_out, device=dev).bfloat16()
    seen = []
    handle = layer.register_pre_activation_hook(lambda dz: seen.append(dz.clone()))
    y = layer(x, r)
    y.backward(G)
    handle.remove()

    x64, r64, cb64, b64 = (t.detach().double().requires_grad_() for t in (x, r, codebook, layer.bias))
    z64 = x64 @ cb64.gather(1, Q.long()).t() + b64
    z64.retain_grad()
    y64 = fn(z64) + r64
    y64.backward(G.double())
    near(y, y64.detach(), 0.0)
    # dZ = G f'(Z) with Z rounded to bf16: f' moves by at most max |f''| 2^-8 |z| (GELU: |f''| <= 0.8, SiLU: 0.5), and dZ is rounded.  What
    # follows from dZ is off by at most the sums of that.
    off = 2.0 ** -8 * (z64.grad.abs() + (0.0 if act == libgq.GQ_ACT_NONE else 0.8) * z64.detach().abs() * G.double().abs())
    near(seen[0], z64.grad, off)
    near(x.grad, x64.grad, off @ cb64.detach().gather(1, Q.long()).abs())
    per_weight = off.view(-1, d_out).t() @ x64.detach().view(-1, d_in).abs()
    near(layer.codebook.grad, cb64.grad, torch.zeros_like(cb64).scatter_add_(1, Q.long(), per_weight))
    near(layer.bias.grad, b64.grad, off.sum((0, 1)))
    assert torch.equal(r.grad, G)
    y2 = layer(x.detach(), r.detach())
    assert torch.equal(y2, y)
    libgq.gq_check()


def test_layer_takes_any_layout(dev):
    torch.manual_seed(1)
    Q = torch.randint(0, 16, (64, 40), device=dev, dtype=torch.uint8)
    layer = QuantizedLinear(Q, 0.1 * torch.randn(64, 16, device=dev))
    x = torch.randn(5, 6, 40, device=dev).bfloat16()
    want = layer(x)
    odd = torch.zeros(5 * 6 * 43 + 3, device=dev, dtype=torch.bfloat16)[3:].view(30, 43)[:, :40]
    odd.copy_(x.view(30, 40))
    assert torch.equal(layer(odd), want.view(30, 64))                    # rows that are not 16-byte aligned
    assert torch.equal(layer(odd[7:8]), want.view(30, 64)[7:8])          # one row with an odd leading dimension
    assert torch.equal(layer(x.transpose(0, 1)), want.transpose(0, 1))
    assert torch.equal(layer(x.float()), want)
    one = layer(x[2, 3])
    assert one.shape == (64,)
    assert layer(x[:0]).shape == (0, 6, 64)
    with pytest.raises(ValueError, match="features"):
        layer(x[..., :32])
    z = x.clone().requires_grad_()
    layer(z).sum().backward()                                            # an expanded gradient
    w = z.detach().clone().requires_grad_()
    layer(w).backward(torch.ones(5, 6, 64, device=dev, dtype=torch.bfloat16))
    assert torch.equal(z.grad, w.grad)


def test_end_loss_matches_autograd_in_64_bits(dev):
    torch.manual_seed(2)
    x = (3 * torch.randn(4, 9, 501, device=dev)).requires_grad_()
    t = torch.randint(0, 501, (4, 9), device=dev)
    t[1, 3:] = -100
    w = torch.rand(4, 9, device=dev)
    loss = end_loss(x, t, w)
    loss.backward()
    x64 = x.detach().double().requires_grad_()
    per = torch.nn.functional.cross_entropy(x64.view(-1, 501), t.view(-1), reduction="none", ignore_index=-100)
    want = (per * w.double().view(-1)).sum()
    want.backward()
    # logp: (vocab / 512 + 69) 2^-24 and its rounding (at most 20 in size), 36 of them
    assert abs(float(loss.detach().double() - want.detach())) <= 36 * (70 + 40) * 2.0 ** -24
    assert bool(((x.grad.double() - x64.grad).abs() <= 128 * 2.0 ** -24 * (x64.grad.abs() + 1e-6)).all())
    assert torch.count_nonzero(x.grad[1, 3:]) == 0
    logp, entropy, top_logp, top_ids = token_logprobs(x, t, top=3)
    assert logp.shape == t.shape and entropy.shape == t.shape and top_logp.shape == (4, 9, 3) and top_ids.shape == (4, 9, 3)
    (entropy.sum()).backward()                                           # without a gradient for logp
    p = torch.softmax(x64.detach(), -1)
    H = -(p * p.log()).sum(-1, keepdim=True)
    both = x64.grad - p * (p.log() + H)
    assert bool(((x.grad.double() - both).abs() <= 256 * 2.0 ** -24 * (x64.grad.abs() + p * (p.log().abs() + H) + 1e-6)).all())
    with pytest.raises(ValueError, match="targets"):
        token_logprobs(x, t[:3])


class Net(torch.nn.Module):
    def __init__(self):
        super().__init__()
        self.embed = torch.nn.Embedding(96, 64)
        self.up = torch.nn.Linear(64, 128)
        self.down = torch.nn.Linear(128, 64, bias=False)
        self.head = torch.nn.Linear(64, 96, bias=False)

    def forward(self, ids):
        h = self.embed(ids)
        up = self.up(h)
        if not isinstance(self.up, QuantizedLinear):
            up = torch.nn.functional.gelu(up)
        h = self.down(up, h) if isinstance(self.down, QuantizedLinear) else h + self.down(up)
        return self.head(h)


def test_calibrate_quantise_and_calibrate_again(dev):
    torch.manual_seed(3)
    net = Net().to(dev).bfloat16()
    batches = [(torch.randint(0, 96, (b, 33), device=dev), torch.randint(0, 96, (b, 33), device=dev)) for b in (3, 2)]
    names, g = ("up", "down"), 4
    H = GuidedHessianCapture({k: getattr(net, k) for k in names}, g).calibrate(net, batches)
    assert all(p.grad is None for p in net.parameters())

    small = copy.deepcopy(net)
    small.up = quantise(net.up, H["up"], activation=libgq.GQ_ACT_GELU)
    small.down = quantise(net.down, H["down"])
    small.embed.weight.requires_grad_(False)              # nothing below the first quantised layer requires a gradient
    # what independent hooks see
    seen_x, seen_dz = {k: [] for k in names}, {k: [] for k in names}
    spies = []
    for k in names:
        mod = getattr(small, k)
        spies.append(mod.register_pre_activation_hook(lambda dz, k=k: seen_dz[k].append(dz.clone())))
        spies.append(mod.register_forward_pre_hook(lambda _m, inp, k=k: seen_x[k].append(inp[0].detach().reshape(-1, inp[0].shape[-1]))))
    cap = GuidedHessianCapture({k: getattr(small, k) for k in names}, g)
    H2 = cap.calibrate(small, batches)
    for s in spies:
        s.remove()
    # the same network in 64 bits, with the weights that the quantised layers hold
    W = {k: mod.table.double().gather(1, torch.stack((mod.codes & 15, mod.codes >> 4), 2).view(mod.d_out, -1)[:, :mod.d_in].long())
         for k, mod in (("up", small.up), ("down", small.down))}
    for i, (ids, targets) in enumerate(batches):
        h = small.embed.weight.double()[ids]
        z_up = h @ W["up"].t() + small.up.bias.double()
        z_up.requires_grad_()
        z_down = torch.nn.functional.gelu(z_up) @ W["down"].t()
        z_down.retain_grad()
        logits = (h + z_down) @ small.head.weight.double().t()
        torch.nn.functional.cross_entropy(logits.view(-1, 96), targets.view(-1), reduction="sum").backward()
        for k, z in (("up", z_up), ("down", z_down)):
            # bf16 all the way: logits, their gradient and two products, each rounded
            err = (seen_dz[k][i].double() - z.grad).norm() / z.grad.norm()
            assert err <= 5 * 2.0 ** -8, (k, err.item())
    for k in names:
        # every module ran twice (both passes); the saliency pass saw the first half
        xs = seen_x[k][:len(batches)]
        s_o = np.concatenate([orc.saliency_strided(synth.bf16_bits(t.cpu()).reshape(tuple(t.shape)), "bf16", g, 1e3) for t in seen_dz[k]], axis=1)
        s_g = torch.cat(cap.s[k], dim=1).cpu().numpy().astype(np.float64)
        assert np.all(np.abs(s_g - s_o) <= 1e-4 * np.abs(s_o) + 1e-30)
        H_o = orc.hessian(np.concatenate([synth.bf16_bits(t.cpu()) for t in xs]), s_o)
        H_g = H2[k].cpu().numpy().astype(np.float64)
        for q in range(g):
            assert np.linalg.norm(H_g[q] - H_o[q]) <= 5e-3 * np.linalg.norm(H_o[q])
    # scores of the quantised network: finite, alternatives in falling order
    logp, entropy, top_logp, _ = token_logprobs(small(batches[0][0]).detach(), batches[0][1], top=4)
    assert bool(logp.isfinite().all()) and bool((entropy >= 0).all()) and bool((top_logp[..., :-1] >= top_logp[..., 1:]).all())
    libgq.gq_check()


def test_captured_step_replays(dev):
    """Scores and the layer's forward and backward pass recorded into one graph (gradients by torch.autograd.grad, which leaves no
    leaf's accumulation in the recording) and replayed on other inputs."""
    torch.manual_seed(4)
    Q = torch.randint(0, 16, (96, 64), device=dev, dtype=torch.uint8)
    layer = QuantizedLinear(Q, 0.1 * torch.randn(96, 16, device=dev), activation=libgq.GQ_ACT_SILU, train_levels=True)
    x = torch.randn(20, 64, device=dev).bfloat16().requires_grad_()
    t = torch.randint(0, 96, (20,), device=dev)

    def step():
        loss = end_loss(layer(x), t)
        return [loss] + list(torch.autograd.grad(loss, [x, layer.codebook]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step()
    with torch.no_grad():
        x.copy_(torch.randn(20, 64, device=dev))
        t.copy_(torch.randint(0, 96, (20,), device=dev))
    graph.replay()
    torch.cuda.synchronize()
    got = [k.clone() for k in kept]
    want = step()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    libgq.gq_check()
