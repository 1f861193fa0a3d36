"""Layers that compute with the quantiser's result: :class:`QuantizedLinear` holds the packed codes and the levels of a layer and runs
gq_linear forward, gq_linear_grad backward; :func:`quantise` makes one from a ``torch.nn.Linear`` and its guided Hessians by Algorithm 2."""
from __future__ import annotations

from typing import Optional

import torch
from torch.autograd.function import once_differentiable

from . import api


def _tokens(t: torch.Tensor, dtype) -> torch.Tensor:
    """[n, width] of a type with 16-byte rows, as the kernels read matrices; a copy only where the layout is another one."""
    t = t.reshape(-1, t.shape[-1]).to(dtype)
    if t.shape[0] == 1:
        t = t[0][None]                   # whatever the leading dimension was
    if (t.shape[1] > 1 and t.stride(1) != 1) or t.stride(0) % 8 != 0 or t.stride(0) < t.shape[1] or t.data_ptr() % 16 != 0:
        t = t.clone(memory_format=torch.contiguous_format)
    return t


class _QuantizedLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, codebook, bias, residual, _anchor, layer, graph):
        X = _tokens(x, layer.dtype)
        table = layer.table if layer.table is not None else layer.make_table(codebook)
        R = _tokens(residual, layer.dtype) if residual is not None else None
        keep = graph and any(ctx.needs_input_grad)           # (an input may require a gradient that no graph is made for)
        Z = X.new_empty((X.shape[0], layer.d_out)) if keep and layer.activation != api.GQ_ACT_NONE else None
        Y = api.gq_linear(X, layer.codes, table, layer.m, bias=bias, activation=layer.activation, residual=R, Z=Z)
        if keep:
            ctx.layer = layer
            ctx.shapes = x.shape, x.dtype, None if residual is None else (residual.shape, residual.dtype), None if bias is None else bias.dtype
            ctx.save_for_backward(X if ctx.needs_input_grad[1] else None, table, Z)      # (only the levels' gradient reads X)
        return Y.view(*x.shape[:-1], layer.d_out).to(layer.out_dtype)

    @staticmethod
    @once_differentiable
    def backward(ctx, grad):
        layer, (X, table, Z) = ctx.layer, ctx.saved_tensors
        shape, dtype, residual, bias_dtype = ctx.shapes
        need_x, need_table, need_bias, need_residual = ctx.needs_input_grad[:4]
        dY = _tokens(grad, layer.dtype)
        workspace = None
        if need_table or need_bias:
            workspace = api.alloc_workspace(api.gq_linear_grad_workspace_bytes(dY.shape[0], layer.d_in, layer.d_out), dY.device)
        dZ, dX, d_table, d_bias = api.gq_linear_grad(dY, X, layer.codes, table, layer.m, workspace, Z=Z, activation=layer.activation,
                                                     need_x=need_x, need_table=need_table, need_bias=need_bias, d_in=layer.d_in)
        for hook in list(layer.pre_activation_hooks.values()):
            hook(dZ.view(*shape[:-1], layer.d_out))
        if dX is not None:
            dX = dX.view(shape).to(dtype)
        d_residual = grad.reshape(residual[0]).to(residual[1]) if need_residual else None
        return dX, d_table, d_bias.to(bias_dtype) if need_bias else None, d_residual, None, None, None


class _Handle:
    def __init__(self, hooks, key):
        self.hooks, self.key = hooks, key

    def remove(self):
        self.hooks.pop(self.key, None)


class QuantizedLinear(torch.nn.Module):
    """``activation(x W_hat^T + bias) + residual`` with ``W_hat[j, c] = codebook[j, Q[j, c]]``.

    ``Q`` (uint8 ``[d_out, d_in]``) and ``codebook`` (fp32 ``[d_out, m]``) as gq_lnq leaves them; activations, bias and residual are computed
    with in ``dtype`` (bfloat16 or float16), to which the levels are rounded.  Without ``train_levels`` the layout is made once; with it the
    levels are a parameter, rounded at every forward pass, and get a gradient (the codes stay).  Inputs may have any floating type; outputs
    have ``out_dtype`` (``dtype`` unless given), which is all that Module.to(dtype) and its like change: levels and bias keep theirs."""

    def __init__(self, Q: torch.Tensor, codebook: torch.Tensor, bias: Optional[torch.Tensor] = None, activation: int = api.GQ_ACT_NONE,
                 dtype=torch.bfloat16, train_levels: bool = False, out_dtype: Optional[torch.dtype] = None):
        super().__init__()
        codes, table = api.gq_linear_pack(Q.contiguous(), codebook.float().contiguous(), dtype)
        self.d_out, self.d_in = int(Q.shape[0]), int(Q.shape[1])
        self.m, self.activation, self.dtype = int(codebook.shape[1]), int(activation), dtype
        self.out_dtype = dtype if out_dtype is None else out_dtype
        self.register_buffer("codes", codes)
        self.register_buffer("table", None if train_levels else table)
        self.codebook = torch.nn.Parameter(codebook.detach().float().clone()) if train_levels else None
        self.bias = None if bias is None else torch.nn.Parameter(bias.detach().to(dtype).clone(), requires_grad=train_levels)
        self.pre_activation_hooks = {}
        self._next_hook = 0

    def _apply(self, fn, recurse=True):
        """Module.to, .half() and their like move the layer, but do not cast it: levels, bias and codebook belong to ``dtype``.  The type
        of its outputs follows the model's."""
        def move(t):
            moved = fn(t)
            return moved if moved.dtype == t.dtype else t.to(moved.device)
        out_dtype = fn(torch.empty(0, dtype=self.out_dtype, device=self.codes.device)).dtype
        super()._apply(move, recurse)
        self.out_dtype = out_dtype
        return self

    def make_table(self, codebook: torch.Tensor) -> torch.Tensor:
        table = torch.zeros((self.d_out, 16), dtype=self.dtype, device=codebook.device)
        table[:, :self.m] = codebook.detach()
        return table

    def register_pre_activation_hook(self, hook) -> _Handle:
        """``hook(dZ)`` is called in every backward pass with the gradient of the pre-activation ``[..., d_out]``, the dl/dZ that the
        saliency step reduces (a module's backward hook sees the gradient behind activation and residual)."""
        key = self._next_hook
        self._next_hook += 1
        self.pre_activation_hooks[key] = hook
        return _Handle(self.pre_activation_hooks, key)

    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
        if x.shape[-1] != self.d_in:
            raise ValueError("the layer takes %d features, not %d" % (self.d_in, x.shape[-1]))
        # hooks want the gradient even where nothing below the layer does: something that requires one keeps it in the graph
        graph = torch.is_grad_enabled()
        anchor = torch.empty(0, device=x.device, requires_grad=True) if self.pre_activation_hooks and graph else None
        return _QuantizedLinear.apply(x, self.codebook, self.bias, residual, anchor, self, graph)

    def extra_repr(self) -> str:
        return "d_in=%d, d_out=%d, m=%d, activation=%d, dtype=%s" % (self.d_in, self.d_out, self.m, self.activation, self.dtype)


def quantise(linear: torch.nn.Linear, H: torch.Tensor, m: int = 16, T: int = 2, K: int = 4, dtype=torch.bfloat16, train_levels: bool = False,
             activation: int = api.GQ_ACT_NONE) -> QuantizedLinear:
    """Algorithm 2 on a layer's weights with its guided Hessians (``[g, d_in, d_in]`` from ``GuidedHessianCapture``), started from ``m``
    equally spaced levels per channel, and the layer that computes with the result.  Its outputs have the type of the layer's weights, so
    that the layers behind it find what they did."""
    W = linear.weight.detach().float().contiguous()
    lo, hi = W.amin(1, keepdim=True), W.amax(1, keepdim=True)
    step = (hi - lo) / max(m - 1, 1)
    Q = torch.where(step > 0, torch.round((W - lo) / torch.where(step > 0, step, torch.ones_like(step))), torch.zeros_like(W))
    Q = Q.clamp_(0, m - 1).to(torch.uint8)
    workspace = api.alloc_workspace(api.gq_lnq_workspace_bytes(W.shape[1], W.shape[0], H.shape[0], m), W.device)
    _, Q, codebook = api.gq_lnq(W, Q, m, H, T, K, workspace)
    return QuantizedLinear(Q, codebook, linear.bias, activation, dtype, train_levels, linear.weight.dtype)
