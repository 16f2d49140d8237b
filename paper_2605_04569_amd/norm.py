"""The root-mean-square norm with the residual's addition: functions and a module over the C ABI's isa_rms_norm,
isa_rms_norm_8bit and isa_rms_norm_backward.  Plumbing only: views, output tensors and torch.autograd glue.

    h = x + residual;   y = h / sqrt(mean(h^2) + eps) * weight      over the last dimension

Tensors are bf16 or fp32 of any shape; those whose rows do not lie at one distance from each other (after the leading
dimensions are taken in the order of x's strides) are copied first.
"""
import torch

from . import binding as B


def _order(x):
    """Leading dimensions by falling stride, or None if they are in that order already: the rows of a transposed view
    are then taken as they lie in memory."""
    n = x.dim() - 1
    if n < 2:
        return None
    order = sorted(range(n), key=lambda d: (-x.stride(d), d))
    return None if order == list(range(n)) else order + [n]


def _as_rows(t, order):
    """`t` with its leading dimensions in `order`, as a tensor whose rows lie at one distance from each other."""
    if order is not None:
        t = t.permute(order)
    return t if t.is_contiguous() or B._row_stride(t) is not None else t.contiguous()


def _back(t, order):
    if order is None:
        return t
    inverse = [0] * len(order)
    for i, d in enumerate(order):
        inverse[d] = i
    return t.permute(inverse)


def _new(t):
    return torch.empty_like(t) if t.is_contiguous() else torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _check(x, weight, residual):
    shape = x.shape
    if len(shape) < 1 or shape[-1] < 1:
        raise ValueError("x needs a last dimension")
    if residual is not None and (residual.shape != shape or residual.dtype != x.dtype):
        raise ValueError("the residual has x's shape and type")
    if weight is not None and weight.shape != shape[-1:]:
        raise ValueError("the weight has one number for every channel")


def _forward(x, weight, residual, eps, want_rstd):
    """(y, h or None, rstd or None, x and residual as rows), all in the dimension order of the rows."""
    order = _order(x)
    x = _as_rows(x, order)
    y, h, rstd = _new(x), None, None
    if residual is not None:
        residual = _as_rows(residual, order)
        h = torch.empty_like(y)
    if want_rstd:
        rstd = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    B.isa_rms_norm(x, weight, y, residual, h, rstd, eps)
    return y, h, rstd, order, x, residual


class _ResidualRMSNormFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, residual, eps):
        weight = None if weight is None else weight.contiguous()
        y, h, rstd, order, xr, rr = _forward(x, weight, residual, eps, True)
        ctx.order = order
        ctx.set_materialize_grads(False)
        # the backward pass adds x and residual again: h is stored rounded
        ctx.save_for_backward(xr, rr, weight, rstd)
        return _back(y, order) if h is None else (_back(y, order), _back(h, order))

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, dh=None):
        x, residual, weight, rstd = ctx.saved_tensors
        need_x, need_w, need_r, _ = ctx.needs_input_grad
        if dy is None:                                 # only h was used
            return (dh if need_x else None, torch.zeros_like(weight) if need_w and weight is not None else None,
                    dh if need_r else None, None)
        order = ctx.order
        dx = _new(x)
        dw = torch.empty_like(weight) if need_w and weight is not None else None
        B.isa_rms_norm_backward(x, residual, weight, rstd, _as_rows(dy, order), dx, None if dh is None else _as_rows(dh, order), dw)
        dx = _back(dx, order)
        return dx if need_x else None, dw, dx if need_r else None, None


def residual_rms_norm(x, weight=None, residual=None, eps=1e-6):
    """y, or (y, h) with a residual; differentiable in x, weight and residual."""
    _check(x, weight, residual)
    if (torch.is_grad_enabled() and (x.requires_grad or (weight is not None and weight.requires_grad) or
                                     (residual is not None and residual.requires_grad))) or B._recorded():
        return _ResidualRMSNormFunction.apply(x, weight, residual, eps)
    y, h, _, order, _, _ = _forward(x, None if weight is None else weight.contiguous(), residual, eps, False)
    return _back(y, order) if residual is None else (_back(y, order), _back(h, order))


def residual_rms_norm_8bit(x, weight=None, residual=None, eps=1e-6, group=0):
    """(y8, scales), or (y8, scales, h) with a residual: y in e4m3, y = y8 * scale of its row (group 0; scales has a last
    dimension of 1) or of its 128 channels (group 128).  For inference: not differentiable."""
    _check(x, weight, residual)
    B._require(group in (0, 128) and (group == 0 or x.shape[-1] % 128 == 0), "group is 0, or 128 and divides the channels")
    if B._recorded():
        return _ResidualRMSNorm8Function.apply(x, weight, residual, eps, group)
    return _eight_bit(x, weight, residual, eps, group)


def _eight_bit(x, weight, residual, eps, group):
    order = _order(x)
    xr = _as_rows(x.detach(), order)
    rr = None if residual is None else _as_rows(residual.detach(), order)
    y8 = torch.empty(xr.shape, dtype=torch.float8_e4m3fn, device=x.device)
    scales = torch.empty((*xr.shape[:-1], x.shape[-1] // group if group else 1), dtype=torch.float32, device=x.device)
    h = None if residual is None else torch.empty(xr.shape, dtype=x.dtype, device=x.device)
    B.isa_rms_norm_8bit(xr, None if weight is None else weight.detach().contiguous(), y8, scales, rr, h, eps, group)
    y8, scales = _back(y8, order), _back(scales, order)
    return (y8, scales) if residual is None else (y8, scales, _back(h, order))


class _ResidualRMSNorm8Function(torch.autograd.Function):
    """What a trace records of residual_rms_norm_8bit, and what refuses forward-mode derivatives of it."""
    @staticmethod
    def forward(ctx, x, weight, residual, eps, group):
        out = _eight_bit(x, weight, residual, eps, group)
        ctx.mark_non_differentiable(*out)
        return out


class ResidualRMSNorm(torch.nn.Module):
    """residual_rms_norm with a learned weight; `eight_bit` is its form for projections in 8 bits."""

    def __init__(self, channels, eps=1e-6, device=None, dtype=None):
        super().__init__()
        self.eps = eps
        self.weight = torch.nn.Parameter(torch.ones(channels, device=device, dtype=dtype))

    def forward(self, x, residual=None):
        return residual_rms_norm(x, self.weight, residual, self.eps)

    def eight_bit(self, x, residual=None, group=0):
        return residual_rms_norm_8bit(x, self.weight, residual, self.eps, group)
