"""The operators of a feed-forward sublayer: gated projections, the norms around a block with its gate and residual sum, and
the clipping of gradients, on device tensors.

Two layers.  The ``bt_...`` functions are the C calls of ``include/bittrain.h`` with tensors for pointers: the caller owns all
buffers, the arguments are checked, the kernels are enqueued on the stream (the current one unless given) and nothing is
synchronised.  ``gated_linear``, ``residual_norm``, ``rms_norm`` and ``clip_grad_norm_`` are what a training program calls: they allocate
and take part in autograd.  There is no CPU fallback: if the library is missing every call raises.

What ``gated_linear`` saves for backward with ReLU gates is zero wherever a gate is closed, like its output, so that
``autograd.BitmapStash`` keeps all three compressed.
"""
import ctypes
import os

import torch

from . import bittrain as bt

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libbittrain.so")

# bt_activation of the C header
ACTIVATIONS = {"relu": 0, "silu": 1, "gelu_tanh": 2}
BT_MAX_NORM_COLS = 16384

_SUPPORTED = (torch.float32, torch.float16, torch.bfloat16)

# the library's functions, in the order of the table in csrc/call.cpp
_CALLS = ("bt_gated_workspace_bytes", "bt_gated_forward", "bt_gated_backward", "bt_residual_norm_workspace_bytes", "bt_residual_norm_forward",
          "bt_residual_norm_backward", "bt_clip_workspace_bytes", "bt_grad_norm", "bt_clip_grads")

_lib = None
_call = None


def lib():
    """The loaded library; raises if it has not been built."""
    global _lib, _call
    if _lib is None:
        bt.lib()                              # (checks that what has been built is there and belongs to this torch)
        L = ctypes.CDLL(_LIB_PATH)
        u64, sz, ci = ctypes.c_uint64, ctypes.c_size_t, ctypes.c_int
        L.bt_gated_workspace_bytes.restype, L.bt_gated_workspace_bytes.argtypes = sz, [u64, u64, u64, ci, ci]
        L.bt_residual_norm_workspace_bytes.restype, L.bt_residual_norm_workspace_bytes.argtypes = sz, [u64, u64, u64, ci]
        L.bt_clip_workspace_bytes.restype, L.bt_clip_workspace_bytes.argtypes = sz, [sz]
        from . import _call as call
        call.bind_block(tuple(ctypes.cast(getattr(L, f), ctypes.c_void_p).value for f in _CALLS))
        _call = call                          # first: other threads go by _lib
        _lib = L
    return _lib


def _native():
    if _lib is None:
        lib()
    return _call


def _activation(name):
    try:
        return ACTIVATIONS[name]
    except (KeyError, TypeError):
        raise ValueError("activation must be one of %s, not %r" % (", ".join(sorted(ACTIVATIONS)), name)) from None


def _code(dtype):
    if dtype not in _SUPPORTED:
        raise TypeError("these operators handle float32, float16 and bfloat16, not %s" % dtype)
    return bt.dtype_code(dtype)


def _scratch(size, device):
    return torch.empty(size, dtype=torch.uint8, device=device)


# ---- gated projections ---------------------------------------------------------------------------------------------

def new_gated_workspace(rows, d, f, dtype, backward=False, device="cuda"):
    """Workspace for bt_gated_forward (bt_gated_backward) of x [rows, d] with weights [f, d]; None if it needs none."""
    size = int(lib().bt_gated_workspace_bytes(rows, d, f, _code(dtype), 0))
    if backward:
        size = max(size, int(lib().bt_gated_workspace_bytes(rows, d, f, _code(dtype), 1)))
    return _scratch(size, device) if size else None


def bt_gated_forward(x, w_gate, w_up, activation, h, gate=None, up=None, workspace=None, stream=None):
    """h = act(x w_gate^T) * (x w_up^T): x [..., d], weights [f, d], h [..., f]; activation "relu", "silu" or "gelu_tanh".  gate and up (like
    h, or None): what bt_gated_backward needs of it."""
    _native().gated_forward(x, w_gate, w_up, h, gate, up, workspace, _activation(activation), stream)


def bt_gated_backward(grad_h, x, w_gate, w_up, gate, up, activation, grad_x, grad_w_gate, grad_w_up, workspace, stream=None):
    """The gradients of x and the weights; grad_x, or both of grad_w_gate and grad_w_up, may be None: not wanted."""
    _native().gated_backward(grad_h, x, w_gate, w_up, gate, up, grad_x, grad_w_gate, grad_w_up, workspace, _activation(activation), stream)


# ---- norms around a block -----------------------------------------------------------------------------------------

def new_residual_norm_workspace(rows, cols, gate_rows, dtype, device="cuda"):
    """Workspace for bt_residual_norm_backward on [rows, cols]; gate_rows 0 if there is no gate."""
    return _scratch(int(lib().bt_residual_norm_workspace_bytes(rows, cols, gate_rows, _code(dtype))), device)


def bt_residual_norm_forward(x, block, post_weight, gate, pre_weight, out, y, stats, eps, scale=1.0, residual_scale=1.0, stream=None):
    """out = residual_scale * x + scale * gate * norm(block) * post_weight and y = norm(out) * pre_weight, norm(t) = t / sqrt(mean(t^2) + eps)
    over the last dimension.  x, block, out, y [..., cols], weights [cols], gate [gate_rows, cols] with gate_rows dividing the rows.  Without block
    (None, as out, post_weight and gate then) y = norm(x) * pre_weight.  post_weight None: block without its norm; gate None: 1;
    pre_weight and y None: out alone.  stats: float32 [2, rows] for backward, or None."""
    _native().residual_norm_forward(x, block, post_weight, gate, pre_weight, out, y, stats, eps, scale, residual_scale, stream)


def bt_residual_norm_backward(grad_out, grad_y, out, block, post_weight, gate, pre_weight, stats, grad_x, grad_block, grad_post_weight, grad_gate,
                              grad_pre_weight, workspace, scale=1.0, residual_scale=1.0, stream=None):
    """The gradients of x, block, gate and both weights (each None if not wanted) from those of out and y (None: 0); out: as the forward pass
    left it, x if there was no block."""
    _native().residual_norm_backward(grad_out, grad_y, out, block, post_weight, gate, pre_weight, stats, grad_x, grad_block, grad_post_weight, grad_gate,
                                     grad_pre_weight, workspace, scale, residual_scale, stream)


# ---- clipping -------------------------------------------------------------------------------------------------------

def new_clip_workspace(grads, device="cuda"):
    """Workspace for bt_grad_norm and bt_clip_grads on a list of as many tensors as `grads` has."""
    return _scratch(int(lib().bt_clip_workspace_bytes(len(grads))), device)


def bt_grad_norm(grads, norm, workspace, stream=None):
    """norm (float32[1]) = sqrt(sum of squares of all elements of the tensors in the list `grads`, whose types may differ)."""
    _native().grad_norm(grads, norm, workspace, stream)


def bt_clip_grads(grads, outs, max_norm, norm, workspace, eps=1e-6, stream=None):
    """The same, and outs[i] = grads[i] * min(1, max_norm / (norm + eps)); outs may be grads itself."""
    _native().clip_grads(grads, outs, norm, workspace, max_norm, eps, stream)


# ---- with autograd --------------------------------------------------------------------------------------------------

def _elsewhere(t):
    return t.device.index is not None and t.device.index != torch.cuda.current_device()


def _check_device(first, *tensors):
    if not first.is_cuda:
        raise ValueError("these operators take tensors in device memory")
    for t in tensors:
        if t is not None and t.device != first.device:
            raise ValueError("all tensors must live on one device")


def _plain(t):
    """`t` as the kernels read it: dense and with its values in memory."""
    return None if t is None else t.contiguous().resolve_neg()


def _keep(*tensors):
    """Whether a backward pass will want something of a call on `tensors`.  (Inside of a Function gradients are always off, and its needs_input_grad
    does not know of no_grad.)"""
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


class _GatedLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_gate, w_up, activation, keep):
        x, w_gate, w_up = _plain(x), _plain(w_gate), _plain(w_up)
        rows, d, f = x.shape[:-1].numel(), x.shape[-1], w_gate.shape[0]
        h = x.new_empty(x.shape[:-1] + (f,))
        gate, up = (torch.empty_like(h), torch.empty_like(h)) if keep else (None, None)
        workspace = new_gated_workspace(rows, d, f, x.dtype, device=x.device)
        bt_gated_forward(x, w_gate, w_up, activation, h, gate, up, workspace)
        if keep:
            ctx.activation = activation
            ctx.save_for_backward(x, w_gate, w_up, gate, up)
        return h

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_h):
        x, w_gate, w_up, gate, up = ctx.saved_tensors
        if _elsewhere(x):
            with torch.cuda.device(x.device):
                return _GatedLinear._gradients(ctx, _plain(grad_h), x, w_gate, w_up, gate, up)
        return _GatedLinear._gradients(ctx, _plain(grad_h), x, w_gate, w_up, gate, up)

    @staticmethod
    def _gradients(ctx, grad_h, x, w_gate, w_up, gate, up):
        grad_x = torch.empty_like(x) if ctx.needs_input_grad[0] else None
        weights = ctx.needs_input_grad[1] or ctx.needs_input_grad[2]
        grad_w_gate, grad_w_up = (torch.empty_like(w_gate), torch.empty_like(w_up)) if weights else (None, None)
        rows = x.shape[:-1].numel()
        workspace = new_gated_workspace(rows, x.shape[-1], w_gate.shape[0], x.dtype, backward=True, device=x.device)
        bt_gated_backward(grad_h, x, w_gate, w_up, gate, up, ctx.activation, grad_x, grad_w_gate, grad_w_up, workspace)
        return grad_x, grad_w_gate if ctx.needs_input_grad[1] else None, grad_w_up if ctx.needs_input_grad[2] else None, None, None


def gated_linear(x, w_gate, w_up, activation="relu"):
    """act(x w_gate^T) * (x w_up^T): the gated half of a feed-forward block, with its gradient.  x [..., d], weights [f, d], all of one type."""
    _activation(activation)
    _check_device(x, w_gate, w_up)
    args = x, w_gate, w_up, activation, _keep(x, w_gate, w_up)
    if _elsewhere(x):
        with torch.cuda.device(x.device):
            return _GatedLinear.apply(*args)
    return _GatedLinear.apply(*args)


class _ResidualNorm(torch.autograd.Function):
    """(x, block, post_weight, gate, pre_weight) -> (out, y), either None where there is none."""

    @staticmethod
    def forward(ctx, x, block, post_weight, gate, pre_weight, eps, scale, residual_scale, keep):
        x, block, post_weight, gate, pre_weight = (_plain(t) for t in (x, block, post_weight, gate, pre_weight))
        rows = x.shape[:-1].numel()
        out = None if block is None else torch.empty_like(x)
        y = None if pre_weight is None else torch.empty_like(x)
        stats = torch.empty(2, rows, dtype=torch.float32, device=x.device) if keep else None
        bt_residual_norm_forward(x, block, post_weight, gate, pre_weight, out, y, stats, eps, scale, residual_scale)
        if keep:
            ctx.scales = scale, residual_scale
            ctx.set_materialize_grads(False)
            ctx.save_for_backward(x if block is None else out, block, post_weight, gate, pre_weight, stats)
        return out, y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_out, grad_y):
        saved = ctx.saved_tensors
        if _elsewhere(saved[0]):
            with torch.cuda.device(saved[0].device):
                return _ResidualNorm._gradients(ctx, _plain(grad_out), _plain(grad_y), *saved)
        return _ResidualNorm._gradients(ctx, _plain(grad_out), _plain(grad_y), *saved)

    @staticmethod
    def _gradients(ctx, grad_out, grad_y, out, block, post_weight, gate, pre_weight, stats):
        if grad_out is None and grad_y is None:
            return (None,) * 9
        needs, scale, residual_scale = ctx.needs_input_grad, *ctx.scales
        like = lambda t, i: torch.empty_like(t) if t is not None and needs[i] else None  # noqa: E731
        grads = like(out, 0), like(block, 1), like(post_weight, 2), like(gate, 3), like(pre_weight, 4)
        if grad_y is None:                    # y did not go into what is differentiated
            if grads[4] is not None:
                grads[4].zero_()
            pre_weight = None
        rows, cols = out.shape[:-1].numel(), out.shape[-1]
        workspace = new_residual_norm_workspace(rows, cols, 0 if gate is None else gate.numel() // max(cols, 1), out.dtype, device=out.device)
        bt_residual_norm_backward(grad_out, grad_y, out, block, post_weight, gate, pre_weight, stats, grads[0], grads[1], grads[2], grads[3],
                                  grads[4] if grad_y is not None else None, workspace, scale, residual_scale)
        return grads + (None, None, None, None)


def _gate_matrix(gate, shape):
    """A gate of shape [cols], [..., 1, cols] (one for each sequence) or [..., cols] as [gate_rows, cols], for x of `shape`.  Refused is one that broadcasting
    would spread over x in another order than its rows are taken in."""
    if gate is None:
        return None
    cols, lead, over = shape[-1], list(gate.shape[:-1]), list(shape[:-1])
    while lead and lead[-1] == 1:
        lead.pop()
    if lead != over[:len(lead)] and gate.shape[:-1].numel() != shape[:-1].numel():      # (with a row for each row of x there is one order)
        if gate.dim() <= len(shape) and all(a in (1, b) for a, b in zip(reversed(gate.shape), reversed(shape))):
            raise ValueError("gate %s lacks leading dimensions of x %s: expand it to the shape of x" % (tuple(gate.shape), tuple(shape)))
    return gate.reshape(gate.shape[:-1].numel(), cols)


def residual_norm(x, block, post_weight=None, gate=None, pre_weight=None, eps=1e-6, scale=1.0, residual_scale=1.0):
    """What stands between two blocks: (out, y) with out = residual_scale * x + scale * gate * norm(block) * post_weight, the residual stream, and
    y = norm(out) * pre_weight, the input of the next block (None without pre_weight), with their gradients.  gate: [cols], or [..., cols] with a
    number of rows that divides that of x, row r of x taking gate row r * gate_rows // rows: a row for each of B sequences of x [B, T, cols] is
    gate [B, cols] or [B, 1, cols].  A gate that lacks leading dimensions of x, such as [1, T, cols] or (with T other than B) [T, cols], is refused:
    gate.expand(x.shape) has a row for each row."""
    if block is None:
        raise TypeError("residual_norm needs a block: rms_norm is the norm alone")
    _check_device(x, block, post_weight, gate, pre_weight)
    if block.shape != x.shape:
        raise ValueError("block must have the shape of x")
    if gate is not None and (gate.dim() == 0 or gate.shape[-1] != x.shape[-1]):
        raise ValueError("gate must have the last dimension of x")
    args = x, block, post_weight, _gate_matrix(gate, x.shape), pre_weight, eps, scale, residual_scale, _keep(x, block, post_weight, gate, pre_weight)
    if _elsewhere(x):
        with torch.cuda.device(x.device):
            return _ResidualNorm.apply(*args)
    return _ResidualNorm.apply(*args)


def rms_norm(x, weight, eps=1e-6):
    """x / sqrt(mean(x^2) + eps) * weight over the last dimension: the norm before the first block."""
    if weight is None:
        raise TypeError("rms_norm needs a weight")
    _check_device(x, weight)
    args = x, None, None, None, weight, eps, 1.0, 1.0, _keep(x, weight)
    if _elsewhere(x):
        with torch.cuda.device(x.device):
            return _ResidualNorm.apply(*args)[1]
    return _ResidualNorm.apply(*args)[1]


def clip_grad_norm_(parameters, max_norm, eps=1e-6):
    """Scales the gradients of the parameters in place so that their norm is at most max_norm; returns the norm that they had, on the device
    (float32[1]; infinite or NaN where a gradient is).  A parameter that is given twice counts once, and so does a gradient that several parameters share;
    gradients must not overlap otherwise.  Nothing waits for the device."""
    if isinstance(parameters, torch.Tensor):
        parameters = [parameters]
    # (One tensor twice would be scaled twice, or once, by workgroups that do not know of each other.)
    grads = list({id(g): g for g in (p.grad for p in parameters) if g is not None}.values())
    if not grads:
        raise ValueError("no parameter has a gradient")
    _check_device(*grads)
    dense = [g if g.is_contiguous() and not g.is_neg() else g.contiguous().resolve_neg() for g in grads]
    with torch.cuda.device(grads[0].device):
        norm = torch.empty(1, dtype=torch.float32, device=grads[0].device)
        bt_clip_grads(dense, dense, max_norm, norm, new_clip_workspace(dense, device=grads[0].device), eps)
        for g, d in zip(grads, dense):
            if g is not d:
                g.copy_(d)
    return norm
