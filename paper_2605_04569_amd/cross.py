"""Cross attention to an encoder's states: a function and a module over the C ABI's isa_cross_attention and
isa_cross_attention_backward.  Plumbing only: copies of tensors whose layout the library does not take, output tensors, scratch
(from torch's allocator, so a call belongs to no particular stream) and torch.autograd glue.

    out[b, h, i] = sum_j softmax_j(scale q[b, h, i] . k[b, h', j]) v[b, h', j],   h' = h // (H // H_kv),   over the valid keys j

q [B, H, S_q, D], k and v [B, H_kv, S_k, D], bf16 or fp32, D 64 or 128, any strides with a contiguous last dimension.
"""
import torch

from . import binding as B


def _layout(t):
    """`t`, or a copy if the library does not take its strides or address."""
    if t.is_contiguous() and not t.data_ptr() & 15:
        return t
    sb, sh, st = B._strides(t)
    if t.numel() == 0 or (t.stride(3) == 1 and not (sb | sh | st) & 7 and st < 1 << 22 and not t.data_ptr() & 15):
        return t
    return t.contiguous() if not t.is_contiguous() else t.clone()


def _like(t):
    """An empty tensor of t's shape; dense, with its heads and tokens in t's order."""
    if t.is_contiguous():
        return torch.empty_like(t)
    if t.stride(1) < t.stride(2):                      # as a projection leaves them
        n = t.shape
        return torch.empty((n[0], n[2], n[1], n[3]), dtype=t.dtype, device=t.device).transpose(1, 2)
    return torch.empty(t.shape, dtype=t.dtype, device=t.device)


_LENGTHS = (torch.int32, torch.int64, torch.int16, torch.int8, torch.uint8, torch.uint16, torch.uint32)      # what 64 bits hold


def _masks(q, k, kv_len, key_mask):
    if kv_len is not None:
        B._require(kv_len.dtype in _LENGTHS, "kv_len: whole numbers, unsigned ones up to 32 bits")
        B._require(kv_len.shape == (q.shape[0],) and kv_len.is_cuda, "kv_len: one whole number a batch item, on the GPU")
        if kv_len.dtype in (torch.int64, torch.uint32):
            kv_len = kv_len.to(torch.int64).clamp(0, k.shape[2])
        kv_len = kv_len.to(torch.int32).contiguous()
    if key_mask is not None:
        B._require(key_mask.shape == (q.shape[0], k.shape[2]) and key_mask.is_cuda and key_mask.dtype in (torch.bool, torch.uint8),
                   "key_mask: truth values [B, S_k], on the GPU")
        if key_mask.stride(1) != 1:
            key_mask = key_mask.contiguous()
    return kv_len, key_mask


class _CrossAttentionFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, kv_len, key_mask, scale):
        q, k, v = _layout(q), _layout(k), _layout(v)
        out = _like(q)
        lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device)
        B.isa_cross_attention(q, k, v, out, kv_len, key_mask, scale, lse)
        ctx.save_for_backward(q, k, v, out, lse, kv_len, key_mask)
        ctx.scale = scale
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_out):
        q, k, v, out, lse, kv_len, key_mask = ctx.saved_tensors
        need_q, need_k, need_v = ctx.needs_input_grad[:3]
        dq = _like(q)                                  # (and the rows' deltas, which dk and dv want)
        dk, dv = (_like(k), _like(v)) if need_k or need_v else (None, None)
        B.isa_cross_attention_backward(q, k, v, out, lse, _layout(d_out), dq, dk, dv, kv_len, key_mask, ctx.scale)
        return dq if need_q else None, dk if need_k else None, dv if need_v else None, None, None, None


def cross_attention(q, k, v, kv_len=None, key_mask=None, scale=None):
    """Differentiable in q, k and v.  kv_len: None or whole numbers [B], the keys of every batch item; key_mask: None or truth values
    [B, S_k], the keys that are attended to.  Where both are given a key has to pass both.  A query whose batch item has no valid
    key gets zeros.  scale: 1 / sqrt(D) unless given."""
    shape_q, shape_k = q.shape, k.shape
    if len(shape_q) != 4 or len(shape_k) != 4 or v.shape != shape_k:
        raise ValueError("q, k and v have four dimensions, k and v one shape")
    if shape_k[0] != shape_q[0] or shape_k[3] != shape_q[3] or shape_k[1] < 1 or shape_q[1] % shape_k[1]:
        raise ValueError("k and v have q's batch items and channels, and heads that divide q's")
    if q.dtype != k.dtype or q.dtype != v.dtype:
        raise ValueError("q, k and v have one type")
    if kv_len is not None or key_mask is not None:
        kv_len, key_mask = _masks(q, k, kv_len, key_mask)
    scale = float(shape_q[3] ** -0.5 if scale is None else scale)
    if (torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or v.requires_grad)) or B._recorded():
        return _CrossAttentionFunction.apply(q, k, v, kv_len, key_mask, scale)
    q, k, v = _layout(q), _layout(k), _layout(v)
    return B.isa_cross_attention(q, k, v, _like(q), kv_len, key_mask, scale)


class CrossAttention(torch.nn.Module):
    """cross_attention as a module; it holds no weights and, between calls, nothing else."""

    def __init__(self, scale=None):
        super().__init__()
        self.scale = scale

    def forward(self, q, k, v, kv_len=None, key_mask=None):
        return cross_attention(q, k, v, kv_len, key_mask, self.scale)
