"""torch.autograd integration of the convolution (plumbing around the C ABI, no arithmetic of its own).

    graph = Graph(n_nodes, senders, receivers)            # prepared once per neighbour list
    out = conv(plan, graph, x, sh, w)                     # differentiable in x, sh, w, to second order
    out = conv_radial(plan, graph, x, sh, h, W)           # weights from the radial layer; first order
    out = conv_vec(plan, graph, x, edge_vec, w)           # harmonics from the edge vectors; first order
    h = layer_norm(linear(rbf, W0, b0), g0, c0, act=E3J_ACT_SILU)   # the radial network's hidden layers; first order

The backward is e3j_conv_bwd; it is itself a differentiable function (of x, sh, w and the incoming cotangent), whose
backward is e3j_conv_bwd_bwd -- what force training needs (a loss on gradients of the energy).  Third derivatives are
not provided.
"""
from __future__ import annotations

import torch

from . import (E3J_ACT_NONE, e3j_conv_bwd, e3j_conv_bwd_bwd, e3j_conv_fwd, e3j_conv_radial_bwd, e3j_conv_radial_fwd,
               e3j_conv_vec_bwd, e3j_conv_vec_fwd, e3j_graph_prepare, e3j_graph_validate, e3j_layer_norm_bwd, e3j_layer_norm_fwd,
               e3j_linear_bwd, e3j_linear_fwd)


class Graph:
    """Receiver-sorted edge list with the index arrays the kernels want (e3j_graph_prepare), on the device."""

    def __init__(self, n_nodes: int, senders: torch.Tensor, receivers: torch.Tensor, validate: bool = True):
        """validate: check on the device, before anything indexes with them, that the ids lie in [0, n_nodes) and the
        receivers do not decrease (one small kernel and a synchronisation per edge list).  The compute calls
        trust the list: an id outside the range makes them read or write outside their arrays."""
        self.n_nodes = int(n_nodes)
        self.senders = senders.to(torch.int32).contiguous()
        self.receivers = receivers.to(torch.int32).contiguous()
        if validate and e3j_graph_validate(self.n_nodes, self.senders, self.receivers) != 0:
            raise ValueError("edge list: an id outside [0, n_nodes) or receivers that decrease")
        self.rowptr, self.sender_perm, self.colptr = e3j_graph_prepare(self.n_nodes, self.senders, self.receivers)


def _c(t):
    return None if t is None else t.contiguous()


class _ConvBackward(torch.autograd.Function):
    @staticmethod
    def forward(ctx, plan, graph, x, sh, w, grad_out):
        ctx.plan, ctx.graph = plan, graph
        ctx.save_for_backward(x, sh, w, grad_out)
        return e3j_conv_bwd(plan, x, sh, w, graph.senders, graph.receivers, grad_out, graph.rowptr, graph.sender_perm,
                            graph.colptr)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, ct_x, ct_sh, ct_w):
        x, sh, w, grad_out = ctx.saved_tensors
        g = ctx.graph
        gg_out, g_x, g_sh, g_w = e3j_conv_bwd_bwd(ctx.plan, x, sh, w, g.senders, g.receivers, grad_out, g.rowptr,
                                                  g.sender_perm, g.colptr, _c(ct_x), _c(ct_sh), _c(ct_w))
        return None, None, g_x, g_sh, g_w, gg_out


class _Conv(torch.autograd.Function):
    @staticmethod
    def forward(ctx, plan, graph, x, sh, w):
        ctx.plan, ctx.graph = plan, graph
        ctx.save_for_backward(x, sh, w)
        return e3j_conv_fwd(plan, x, sh, w, graph.senders, graph.receivers, graph.rowptr)

    @staticmethod
    def backward(ctx, grad_out):
        x, sh, w = ctx.saved_tensors
        gx, gsh, gw = _ConvBackward.apply(ctx.plan, ctx.graph, x, sh, w, grad_out.contiguous())
        return None, None, gx, gsh, gw


def conv(plan, graph: Graph, x: torch.Tensor, sh: torch.Tensor, w: torch.Tensor) -> torch.Tensor:
    """out[n_nodes, D, N_q] = message-passing convolution of x [n_nodes, d, N_q] with harmonics sh [n_edges, d'] and
    edge weights w [n_edges, P, N_q] over `graph` (float32 CUDA tensors)."""
    return _Conv.apply(plan, graph, x.contiguous(), sh.contiguous(), w.contiguous())


class _ConvRadial(torch.autograd.Function):
    @staticmethod
    def forward(ctx, plan, graph, x, sh, h, W):
        ctx.plan, ctx.graph = plan, graph
        ctx.save_for_backward(x, sh, h, W)
        return e3j_conv_radial_fwd(plan, x, sh, h, W, graph.senders, graph.receivers, graph.rowptr)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_out):
        x, sh, h, W = ctx.saved_tensors
        g = ctx.graph
        need = ctx.needs_input_grad[2:]
        gx, gsh, gh, gW = e3j_conv_radial_bwd(ctx.plan, x, sh, h, W, g.senders, g.receivers, grad_out.contiguous(), g.rowptr,
                                              g.sender_perm, g.colptr, grad_x=need[0], grad_sh=need[1], grad_h=need[2],
                                              grad_W=need[3])
        return None, None, gx, gsh, gh, gW


class _ConvVec(torch.autograd.Function):
    @staticmethod
    def forward(ctx, plan, graph, x, edge_vec, w):
        ctx.plan, ctx.graph = plan, graph
        ctx.save_for_backward(x, edge_vec, w)
        return e3j_conv_vec_fwd(plan, x, edge_vec, w, graph.senders, graph.receivers, graph.rowptr)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_out):
        x, edge_vec, w = ctx.saved_tensors
        g = ctx.graph
        need = ctx.needs_input_grad[2:]
        gx, gvec, gw = e3j_conv_vec_bwd(ctx.plan, x, edge_vec, w, g.senders, g.receivers, grad_out.contiguous(), g.rowptr,
                                        g.sender_perm, g.colptr, grad_x=need[0], grad_vec=need[1], grad_w=need[2])
        return None, None, gx, gvec, gw


def conv_radial(plan, graph: Graph, x, sh, h, W) -> torch.Tensor:
    """The convolution with the edge weights given as the radial network's last layer, w = h W (first derivatives)."""
    return _ConvRadial.apply(plan, graph, x.contiguous(), sh.contiguous(), h.contiguous(), W.contiguous())


def conv_vec(plan, graph: Graph, x, edge_vec, w) -> torch.Tensor:
    """The convolution with the harmonics taken from the edge vectors [n_edges, 3] (first derivatives)."""
    return _ConvVec.apply(plan, graph, x.contiguous(), edge_vec.contiguous(), w.contiguous())


def _kept(ctx, n_real):
    """A copy of a padded list's count of real rows for the backward: the next list may be prepared in the same buffer before it."""
    return None if n_real is None or not any(ctx.needs_input_grad) else n_real.clone()


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, W, b, residual, act, n_real):
        y = e3j_linear_fwd(x, W, b, residual, act, n_real)
        ctx.act = act
        ctx.save_for_backward(x, W, b, _kept(ctx, n_real))
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_y):
        x, W, b, n_real = ctx.saved_tensors
        grad_y, need = grad_y.contiguous(), ctx.needs_input_grad
        gx, gW, gb = e3j_linear_bwd(x, W, b, grad_y, ctx.act, n_real, grad_x=need[0], grad_W=need[1], grad_b=need[2])
        gr = grad_y if need[3] else None
        if gr is not None and n_real is not None:   # padding rows of the result do not depend on anything
            real = torch.arange(gr.shape[0], device=gr.device).unsqueeze(1) < n_real
            gr = torch.where(real, gr, torch.zeros_like(gr))
        return gx, gW, gb, gr, None, None


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, act, n_real):
        y = e3j_layer_norm_fwd(x, weight, bias, eps, act, n_real)
        ctx.eps, ctx.act = eps, act
        ctx.save_for_backward(x, weight, bias, _kept(ctx, n_real))
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_y):
        x, weight, bias, n_real = ctx.saved_tensors
        need = ctx.needs_input_grad
        gx, gw, gb = e3j_layer_norm_bwd(x, weight, bias, grad_y.contiguous(), ctx.eps, ctx.act, n_real, grad_x=need[0],
                                        grad_weight=need[1], grad_bias=need[2])
        return gx, gw, gb, None, None, None


def linear(x, W, b=None, residual=None, act: int = E3J_ACT_NONE, n_real=None) -> torch.Tensor:
    """act(x W + b) + residual: x [rows, n_in], W [n_in, n_out] (float32 or bfloat16, first derivatives); saves x, W and b for the
    backward, nothing else.  n_real as in e3j_linear_fwd; its value at the time of the call counts for the backward too."""
    return _Linear.apply(x.contiguous(), W.contiguous(), _c(b), _c(residual), act, n_real)


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, act: int = E3J_ACT_NONE, n_real=None) -> torch.Tensor:
    """Layer norm over the columns of x [rows, n] with an activation behind it (first derivatives); saves its inputs only.  n_real as in linear."""
    return _LayerNorm.apply(x.contiguous(), _c(weight), _c(bias), eps, act, n_real)
