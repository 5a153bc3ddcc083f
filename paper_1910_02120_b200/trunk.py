"""Layer norm with a gradient for torch trunks in front of the partitioned layers.  Both passes run in the CUDA library
(ist_layer_norm_forward, ist_layer_norm_backward); the optimizer for such a trunk is api.AdamW."""
from __future__ import annotations

from typing import Optional

import torch
from torch.autograd import forward_ad

from . import api


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, groups, y_dtype):
        y, mean, rstd = api.ist_layer_norm_forward(x, weight, bias, eps, groups=groups, y_dtype=y_dtype)
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.groups, ctx.shapes = groups, [None if t is None else t.shape for t in (weight, bias)]
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        if not dy.is_contiguous():                        # an expanded gradient has no row stride
            dy = dy.contiguous()
        dx, dweight, dbias = api.ist_layer_norm_backward(
            dy, x, weight, mean, rstd, groups=ctx.groups, want_dx=ctx.needs_input_grad[0],
            want_dweight=ctx.needs_input_grad[1], want_dbias=ctx.needs_input_grad[2])
        if dweight is not None:
            dweight = dweight.view(ctx.shapes[0])
        if dbias is not None:
            dbias = dbias.view(ctx.shapes[1])
        return dx, dweight, dbias, None, None, None


def _check_leaves(tensors) -> None:
    """Refuses a capture whose backward pass torch could not capture.  A leaf's accumulation node lives as long as any
    graph that leads to it and stays with the stream it was made on: a backward pass captured while an eager graph of the leaf is
    alive would synchronise with that stream and break the capture.  So every call notes its stream at the node.
    Nodes that only other operations have used carry no note; for these torch's own rule holds, that the leaves of a captured
    backward pass are not in a live eager graph."""
    stream = torch.cuda.current_stream()
    for t in tensors:
        if t is not None and t.requires_grad and t.grad_fn is None and t.is_cuda:
            made_on = torch.autograd.graph.get_gradient_edge(t).node.metadata.setdefault("ist_stream", stream)
            if made_on != stream and torch.cuda.is_current_stream_capturing():
                raise api.IstError(api.IST_ERR_STATE, "layer_norm is captured while an eager graph of the same leaf is alive: "
                                   "free that graph first, or capture with t.detach().requires_grad_() in the leaf's place")


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
               groups: int = 1, y_dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """Layer norm over the last dimension with gradients for x, weight and bias; see api.ist_layer_norm_forward.
    A gradient of a gradient and forward-mode differentiation are refused."""
    if forward_ad._current_level >= 0 and any(t is not None and forward_ad.unpack_dual(t).tangent is not None for t in (x, weight, bias)):
        raise api.IstError(api.IST_ERR_UNSUPPORTED, "layer_norm has no forward-mode derivative")
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (x, weight, bias)):
        y = _LayerNorm.apply(x, weight, bias, eps, groups, y_dtype)
        _check_leaves((x, weight, bias))          # behind the call: y's graph keeps the leaves' nodes
        return y
    return api.ist_layer_norm_forward(x, weight, bias, eps, groups=groups, y_dtype=y_dtype, want_stats=False)[0]
