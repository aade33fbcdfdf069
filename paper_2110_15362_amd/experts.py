"""The operators of a feed-forward sublayer of several experts: the choice of each token's experts and the order of the rows that it makes, the gated
projections and the product back with each row's own expert, and the sum of a token's rows, on device tensors.

A row stands for one token at one of its experts.  A ``Plan`` says which rows there are and in which order: by expert, and within an expert by token.  How
many rows an expert has stays on the device: nothing waits for the host.

Two layers, as in ``block``.  The ``bt_...`` functions are the C calls of ``include/bittrain.h`` with tensors for pointers: the caller owns all buffers, the arguments are
checked, the kernels are enqueued on the stream (the current one unless given) and nothing is synchronised.  ``route``, ``plan_of``, ``gated_linear``, ``linear`` and
``combine`` are what a training program calls: they allocate and take part in autograd.  There is no CPU fallback: if the library is missing every
call raises.

A sublayer is

    weights, plan = experts.route(x @ w_router.t(), 2)
    h = experts.gated_linear(x, plan, w_gate, w_up, "silu")
    out = experts.combine(experts.linear(h, plan, w_down), plan, weights)

With ReLU gates what ``gated_linear`` keeps for backward is zero wherever a gate is closed, like its output, so that ``autograd.BitmapStash`` keeps all three
compressed.
"""
import ctypes

import torch

from . import bittrain as bt
from .block import ACTIVATIONS, _activation, _check_device, _code, _elsewhere, _keep, _plain, _scratch, lib as _block_lib

BT_MAX_EXPERTS, BT_MAX_CHOSEN = 1024, 32

# the library's functions, in the order of the table in csrc/call.cpp
_CALLS = ("bt_route_workspace_bytes", "bt_route_forward", "bt_route_order", "bt_route_backward", "bt_expert_gated_workspace_bytes", "bt_expert_gated_forward",
          "bt_expert_gated_backward", "bt_expert_linear_workspace_bytes", "bt_expert_linear_forward", "bt_expert_linear_backward", "bt_combine_forward",
          "bt_combine_backward")

_lib = None
_call = None


def lib():
    """The loaded library; raises if it has not been built."""
    global _lib, _call
    if _lib is None:
        L = _block_lib()
        u64, sz = ctypes.c_uint64, ctypes.c_size_t
        L.bt_route_workspace_bytes.restype, L.bt_route_workspace_bytes.argtypes = sz, [u64, u64, u64]
        from . import _call as call
        call.bind_experts(tuple(ctypes.cast(getattr(L, f), ctypes.c_void_p).value for f in _CALLS))
        _call = call                          # first: other threads go by _lib
        _lib = L
    return _lib


def _native():
    if _lib is None:
        lib()
    return _call


# ---- the plan ----------------------------------------------------------------------------------------------------------

class Plan:
    """Who goes where: index [tokens, chosen], a token's experts (-1: none); slots, of the same shape, the row of each; source [tokens * chosen], the token of each row (-1: a
    row of no expert, which come last); offsets [experts + 1], expert e having the rows from offsets[e] on, up to offsets[e + 1].  32-bit integers on one device."""

    __slots__ = ("index", "slots", "source", "offsets", "tokens", "chosen", "experts")

    def __init__(self, index, slots, source, offsets):
        for name, t in (("index", index), ("slots", slots), ("source", source), ("offsets", offsets)):
            if t.dtype != torch.int32:
                raise TypeError("%s must hold 32-bit integers (torch.int32), not %s" % (name, t.dtype))
            if not t.is_contiguous():
                raise ValueError("%s must be contiguous" % name)
            if t.device != index.device:
                raise ValueError("all tables must live on one device")
        if index.dim() != 2 or slots.shape != index.shape or source.shape != (index.numel(),) or offsets.dim() != 1:
            raise ValueError("index and slots must be [tokens, chosen], source [tokens * chosen], offsets [experts + 1]")
        self.index, self.slots, self.source, self.offsets = index, slots, source, offsets
        (self.tokens, self.chosen), self.experts = index.shape, offsets.shape[0] - 1
        _check_numbers(self.tokens, self.experts, self.chosen)

    @property
    def rows(self):
        return self.tokens * self.chosen

    @property
    def device(self):
        return self.index.device

    def _tables(self):
        return self.index, self.slots, self.source, self.offsets


def _check_numbers(tokens, experts, chosen):
    if not 1 <= experts <= BT_MAX_EXPERTS or not 1 <= chosen <= min(experts, BT_MAX_CHOSEN):
        raise ValueError("of %d to %d experts a token may use 1 to %d, and no more than there are: not %d of %d" % (1, BT_MAX_EXPERTS, BT_MAX_CHOSEN, chosen, experts))
    if tokens * chosen >= 1 << 31:
        raise ValueError("tokens * chosen must be below 2^31")


def new_plan(tokens, experts, chosen, device="cuda"):
    """A plan whose tables are yet to be written, by bt_route_forward or, from its index, bt_route_order."""
    _check_numbers(tokens, experts, chosen)
    empty = lambda *shape: torch.empty(shape, dtype=torch.int32, device=device)  # noqa: E731
    return Plan(empty(tokens, chosen), empty(tokens, chosen), empty(tokens * chosen), empty(experts + 1))


def new_route_workspace(tokens, experts, chosen, device="cuda"):
    """Workspace for bt_route_forward and bt_route_order; None if they need none."""
    size = int(lib().bt_route_workspace_bytes(tokens, experts, chosen))
    return _scratch(size, device) if size else None


def bt_route_forward(logits, plan, weights, workspace=None, normalise=True, stream=None):
    """Writes the plan's tables and weights (float32 [tokens, chosen]) from logits [tokens, experts]: of each token the experts with the largest logits (of equal ones the lowest
    numbers; never one whose logit is -infinity), and the softmax there, over those chosen (normalise) or over all."""
    _native().route_forward(logits, weights, *plan._tables(), workspace, normalise, stream)


def bt_route_order(plan, workspace=None, stream=None):
    """Writes slots, source and offsets from the plan's index."""
    _native().route_order(*plan._tables(), workspace, stream)


def bt_route_backward(grad_weights, logits, plan, weights, grad_logits, normalise=True, stream=None):
    """The gradient of the logits (with normalise they are not read and may be None)."""
    _native().route_backward(grad_weights, weights, grad_logits, *plan._tables(), logits, normalise, stream)


# ---- the products -------------------------------------------------------------------------------------------------------

def _product_workspace(gated, plan, d, f, dtype, ordered, backward, device):
    lib()
    size = max(_call.experts_workspace(gated, plan.tokens, plan.experts, plan.chosen, d, f, _code(dtype), bool(ordered), b) for b in range(2 if backward else 1))
    return _scratch(size, plan.device if device is None else device) if size else None


def new_gated_workspace(plan, d, f, dtype, ordered=False, backward=False, device=None):
    """Workspace for bt_expert_gated_forward (and bt_expert_gated_backward) with weights [experts, f, d]; None if it needs none."""
    return _product_workspace(1, plan, d, f, dtype, ordered, backward, device)


def bt_expert_gated_forward(x, plan, w_gate, w_up, activation, h, gate=None, up=None, workspace=None, ordered=False, stream=None):
    """h = act(x w_gate^T) * (x w_up^T) with the weights of each row's expert: x [tokens, d], or with `ordered` [rows, d] in the plan's order; weights [experts, f, d]; h
    [rows, f]; activation "relu", "silu" or "gelu_tanh".  gate and up (like h, or None): what bt_expert_gated_backward needs of it."""
    _native().expert_gated_forward(x, w_gate, w_up, h, *plan._tables(), gate, up, workspace, _activation(activation), ordered, stream)


def bt_expert_gated_backward(grad_h, x, plan, w_gate, w_up, gate, up, activation, grad_x, grad_w_gate, grad_w_up, workspace, ordered=False, stream=None):
    """The gradients of x and the weights; grad_x, or both of grad_w_gate and grad_w_up, may be None: not wanted."""
    _native().expert_gated_backward(grad_h, x, w_gate, w_up, gate, up, *plan._tables(), grad_x, grad_w_gate, grad_w_up, workspace, _activation(activation), ordered, stream)


def new_linear_workspace(plan, d_in, d_out, dtype, ordered=True, backward=False, device=None):
    """Workspace for bt_expert_linear_forward (and bt_expert_linear_backward) with weights [experts, d_out, d_in]; None if it needs none."""
    return _product_workspace(0, plan, d_in, d_out, dtype, ordered, backward, device)


def bt_expert_linear_forward(x, plan, w, y, workspace=None, ordered=True, stream=None):
    """y = x w^T with the weight of each row's expert: x [rows, d_in] in the plan's order, or without `ordered` [tokens, d_in]; w [experts, d_out, d_in]; y [rows, d_out]."""
    _native().expert_linear_forward(x, w, y, *plan._tables(), workspace, ordered, stream)


def bt_expert_linear_backward(grad_y, x, plan, w, grad_x, grad_w, workspace=None, ordered=True, stream=None):
    """The gradients of x and w, each None if not wanted."""
    _native().expert_linear_backward(grad_y, x, w, *plan._tables(), grad_x, grad_w, workspace, ordered, stream)


# ---- a token's rows -----------------------------------------------------------------------------------------------------

def bt_combine_forward(y, plan, weights, out, stream=None):
    """out [tokens, cols]: a token's rows of y [rows, cols], times weights (float32 [tokens, chosen], or None: 1), added up."""
    _native().combine_forward(y, out, *plan._tables(), weights, stream)


def bt_combine_backward(grad_out, y, plan, weights, grad_y, grad_weights, stream=None):
    """The gradients of y and the weights, each None if not wanted."""
    _native().combine_backward(grad_out, y, *plan._tables(), weights, grad_y, grad_weights, stream)


# ---- with autograd ------------------------------------------------------------------------------------------------------

def _on(t, function, *args):
    """function(*args) with t's device as the current one."""
    if _elsewhere(t):
        with torch.cuda.device(t.device):
            return function(*args)
    return function(*args)


def _check_plan(plan, first, *tensors):
    if not isinstance(plan, Plan):
        raise TypeError("plan must be a Plan, as route and plan_of make them")
    _check_device(first, plan.index, *tensors)


class _Route(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, plan, normalise, keep):
        logits = _plain(logits)
        weights = torch.empty(plan.index.shape, dtype=torch.float32, device=logits.device)
        bt_route_forward(logits, plan, weights, new_route_workspace(plan.tokens, plan.experts, plan.chosen, logits.device), normalise)
        if keep:
            ctx.plan, ctx.normalise, ctx.like = plan, normalise, (logits.shape, logits.dtype)
            ctx.save_for_backward(None if normalise else logits, weights, plan.index)
        return weights

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_weights):
        return _on(grad_weights, _Route._gradient, ctx, _plain(grad_weights)), None, None, None

    @staticmethod
    def _gradient(ctx, grad_weights):
        logits, weights, _ = ctx.saved_tensors
        shape, dtype = ctx.like
        grad = torch.empty(shape, dtype=dtype, device=grad_weights.device)
        bt_route_backward(grad_weights, logits, ctx.plan, weights, grad, ctx.normalise)
        return grad


def route(logits, chosen, normalise=True):
    """(weights, plan) for logits [tokens, experts]: the plan by which each token goes to the `chosen` experts with the largest logits (of equal ones the lowest numbers), and its
    weights for them, float32 [tokens, chosen]: the softmax over those chosen, or without `normalise` over all, with the gradient of the logits.  An expert whose logit is
    -infinity is never chosen: a token may so have fewer experts, or none (padding), and weights of 0."""
    if logits.dim() != 2:
        raise ValueError("logits must be [tokens, experts]")
    _check_device(logits)
    _code(logits.dtype)
    plan = _on(logits, new_plan, logits.shape[0], logits.shape[1], chosen, logits.device)
    weights = _on(logits, _Route.apply, logits, plan, bool(normalise), _keep(logits))
    return weights, plan


def _numbers(index, experts):
    """The experts of `index` in 32 bits, -1 where there is none."""
    if index.dtype not in (torch.int32, torch.int64):      # (a type of few bits holds neither -1 nor the number of experts for sure)
        index = index.long()
    return torch.where((index >= 0) & (index < experts), index, -1).int()


def plan_of(index, experts):
    """The plan for experts that were chosen otherwise: index [tokens, chosen], integers; a number that is no expert's stands for none."""
    if index.dim() != 2 or index.dtype.is_floating_point or index.dtype.is_complex or index.dtype == torch.bool:
        raise ValueError("index must be [tokens, chosen], of integers")
    if not index.is_cuda:
        raise ValueError("these operators take tensors in device memory")

    def make():
        tokens, chosen = index.shape
        plan = new_plan(tokens, experts, chosen, index.device)
        plan.index = _numbers(index, experts).contiguous()
        bt_route_order(plan, new_route_workspace(tokens, experts, chosen, index.device))
        return plan
    return _on(index, make)


class _GatedLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_gate, w_up, plan, activation, ordered, keep):
        x, w_gate, w_up = _plain(x), _plain(w_gate), _plain(w_up)
        d, f = w_gate.shape[2], w_gate.shape[1]
        h = x.new_empty(plan.rows, f)
        gate, up = (torch.empty_like(h), torch.empty_like(h)) if keep else (None, None)
        bt_expert_gated_forward(x, plan, w_gate, w_up, activation, h, gate, up, new_gated_workspace(plan, d, f, x.dtype, ordered), ordered)
        if keep:
            ctx.plan, ctx.activation, ctx.ordered = plan, activation, ordered
            ctx.save_for_backward(x, w_gate, w_up, gate, up)
        return h

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_h):
        return _on(grad_h, _GatedLinear._gradients, ctx, _plain(grad_h))

    @staticmethod
    def _gradients(ctx, grad_h):
        x, w_gate, w_up, gate, up = ctx.saved_tensors
        needs, plan = ctx.needs_input_grad, ctx.plan
        grad_x = torch.empty_like(x) if needs[0] else None
        grads = (torch.empty_like(w_gate), torch.empty_like(w_up)) if needs[1] or needs[2] else (None, None)
        workspace = new_gated_workspace(plan, w_gate.shape[2], w_gate.shape[1], x.dtype, ctx.ordered, backward=True)
        bt_expert_gated_backward(grad_h, x, plan, w_gate, w_up, gate, up, ctx.activation, grad_x, *grads, workspace, ctx.ordered)
        return grad_x, grads[0] if needs[1] else None, grads[1] if needs[2] else None, None, None, None, None


def gated_linear(x, plan, w_gate, w_up, activation="relu", ordered=False):
    """act(x w_gate^T) * (x w_up^T) with the weights of each row's expert, with its gradient: [rows, f], rows of no expert zeros.  x [tokens, d], or with `ordered`
    [rows, d] in the plan's order; weights [experts, f, d], all of one type.  In 16 bits what is kept for backward, and the factors of the gradients, are rounded to them."""
    _activation(activation)
    _check_plan(plan, x, w_gate, w_up)
    _check_weight(plan, x, w_gate, "w_gate")
    return _on(x, _GatedLinear.apply, x, w_gate, w_up, plan, activation, bool(ordered), _keep(x, w_gate, w_up))


def _check_weight(plan, x, w, name):
    if w.dim() != 3 or w.shape[0] != plan.experts:
        raise ValueError("%s must be a matrix for each of the plan's %d experts" % (name, plan.experts))
    if x.dim() != 2:
        raise ValueError("x must be a matrix, with a row for each token or, ordered, each of the plan's rows")


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, plan, ordered, keep):
        x, w = _plain(x), _plain(w)
        y = x.new_empty(plan.rows, w.shape[1])
        bt_expert_linear_forward(x, plan, w, y, new_linear_workspace(plan, w.shape[2], w.shape[1], x.dtype, ordered), ordered)
        if keep:
            ctx.plan, ctx.ordered = plan, ordered
            ctx.save_for_backward(x, w)
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_y):
        return _on(grad_y, _Linear._gradients, ctx, _plain(grad_y))

    @staticmethod
    def _gradients(ctx, grad_y):
        x, w = ctx.saved_tensors
        grad_x, grad_w = (torch.empty_like(t) if need else None for t, need in zip((x, w), ctx.needs_input_grad))
        workspace = new_linear_workspace(ctx.plan, w.shape[2], w.shape[1], x.dtype, ctx.ordered, backward=True)
        bt_expert_linear_backward(grad_y, x, ctx.plan, w, grad_x, grad_w, workspace, ctx.ordered)
        return grad_x, grad_w, None, None, None


def linear(x, plan, w, ordered=True):
    """x w^T with the weight of each row's expert, with its gradient: [rows, d_out], rows of no expert zeros.  x [rows, d_in] in the plan's order, or without `ordered`
    [tokens, d_in]; w [experts, d_out, d_in], of the same type."""
    _check_plan(plan, x, w)
    _check_weight(plan, x, w, "w")
    return _on(x, _Linear.apply, x, w, plan, bool(ordered), _keep(x, w))


class _Combine(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y, weights, plan, keep):
        y, weights = _plain(y), _plain(weights)
        out = y.new_empty(plan.tokens, y.shape[1])
        bt_combine_forward(y, plan, weights, out)
        if keep:
            ctx.plan = plan
            ctx.save_for_backward(y, weights)
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_out):
        return _on(grad_out, _Combine._gradients, ctx, _plain(grad_out))

    @staticmethod
    def _gradients(ctx, grad_out):
        y, weights = ctx.saved_tensors
        grad_y, grad_weights = (torch.empty_like(t) if need else None for t, need in zip((y, weights), ctx.needs_input_grad))
        bt_combine_backward(grad_out, y, ctx.plan, weights, grad_y, grad_weights)
        return grad_y, grad_weights, None, None


def combine(y, plan, weights=None):
    """[tokens, cols]: a token's rows of y [rows, cols], times its weights (float32 [tokens, chosen], or None: 1), added up, with the gradients of both; zeros for a token without
    experts."""
    _check_plan(plan, y, weights)
    if y.dim() != 2:
        raise ValueError("y must be a matrix with a row for each of the plan's")
    if weights is not None and weights.dim() > 1 and weights.shape[-1] != plan.chosen:
        raise ValueError("weights must be [tokens, chosen]")
    return _on(y, _Combine.apply, y, weights, plan, _keep(y, weights))
