"""A learning pass over whole sequences for torch programs: differentiable calls around include/vla_learn.h.

Sequences of different lengths are packed one behind the other; ``start`` (int32 [sequences + 1] on the GPU) has the first
row of each and the end of the last (``Rows.start`` of a page plan is one).  ``prompt_attention`` is the causal attention
of every row to its sequence, ``block_norm`` what lies between two blocks.  All compute is in libvla.so, on torch's current
stream; nothing waits for the GPU.
"""
from __future__ import annotations

from typing import Optional

import torch
from torch.autograd.function import once_differentiable

from . import vla as V
from .paged import _code, _ok, _on_gpu, _ptr, _rows_of, _stream


def _starts(start: torch.Tensor) -> int:
    if start.dim() != 1 or start.dtype != torch.int32 or not start.is_contiguous() or start.shape[0] < 2:
        raise ValueError("start: int32 [sequences + 1], contiguous")
    return start.shape[0] - 1


def _heads(t: torch.Tensor, hd: int) -> int:
    return t.shape[1] if t.dim() == 3 else t.shape[-1] // hd


class _PromptAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, start, head_dim, scale):
        if not q.dtype == k.dtype == v.dtype or not q.shape[0] == k.shape[0] == v.shape[0]:
            raise ValueError("q, k and v have one type and the same rows")
        n_seq, n = _starts(start), q.shape[0]
        H, Hk = _heads(q, head_dim), _heads(k, head_dim)
        _on_gpu(q, k, v, start)
        ld = [_rows_of(q, H, head_dim), _rows_of(k, Hk, head_dim), _rows_of(v, Hk, head_dim)]
        out = torch.empty(n, H, head_dim, dtype=q.dtype, device=q.device)
        lse = torch.empty(n, H, dtype=torch.float32, device=q.device)
        _ok(V.vla_prompt_attn(q.data_ptr(), ld[0], k.data_ptr(), ld[1], v.data_ptr(), ld[2], _code(q), n, H, Hk, head_dim, start.data_ptr(),
                              n_seq, scale, out.data_ptr(), H * head_dim, lse.data_ptr(), _stream()))
        ctx.save_for_backward(q, k, v, start, out, lse)
        ctx.shape = H, Hk, head_dim, scale, ld
        ctx.mark_non_differentiable(lse)
        return out, lse

    @staticmethod
    @once_differentiable
    def backward(ctx, d_out, _):
        q, k, v, start, out, lse = ctx.saved_tensors
        H, Hk, hd, scale, ld = ctx.shape
        n = q.shape[0]
        _on_gpu(d_out)
        d_out = d_out.contiguous()
        if d_out.data_ptr() & 15:
            d_out = d_out.clone()
        d = torch.empty(n, (H + 2 * Hk) * hd, dtype=q.dtype, device=q.device)
        dq, dk, dv = d[:, :H * hd], d[:, H * hd:(H + Hk) * hd], d[:, (H + Hk) * hd:]
        workspace = torch.empty(V.vla_prompt_attn_grad_workspace_bytes(n, H, Hk, hd), dtype=torch.uint8, device=q.device)
        _ok(V.vla_prompt_attn_grad(q.data_ptr(), ld[0], k.data_ptr(), ld[1], v.data_ptr(), ld[2], _code(q), n, H, Hk, hd, start.data_ptr(),
                                   start.shape[0] - 1, scale, out.data_ptr(), H * hd, lse.data_ptr(), d_out.data_ptr(), H * hd,
                                   dq.data_ptr(), d.stride(0), dk.data_ptr(), d.stride(0), dv.data_ptr(), d.stride(0),
                                   workspace.data_ptr(), workspace.numel(), _stream()))
        return dq.view(q.shape), dk.view(k.shape), dv.view(v.shape), None, None, None


def prompt_attention(q, k, v, start, head_dim: int, scale: Optional[float] = None, want_lse: bool = False):
    """Causal attention of packed sequences: q [rows, heads, head_dim] or [rows, heads * head_dim] with dense rows, k and v
    likewise with a divisor of its heads, fp16 or bf16, views of one q|k|v buffer among them.  Returns [rows, heads, head_dim] (and
    the log-sums, which have no gradient).  Rows of no sequence give zeros."""
    out, lse = _PromptAttention.apply(q, k, v, start, int(head_dim), float(head_dim ** -0.5 if scale is None else scale))
    return (out, lse) if want_lse else out


def _dense(t: Optional[torch.Tensor], n: int, dim: int, what: str) -> int:
    if t is None:
        return dim
    if t.shape != (n, dim) or (dim > 1 and t.stride(1) != 1):
        raise ValueError(f"{what}: [rows, channels] with dense rows expected, got {tuple(t.shape)} with strides {t.stride()}")
    return t.stride(0) if n > 1 else dim  # (rows that overlap, a stride below the channels, are refused by the call)


class _BlockNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y, h, pre_gain, post_gain, gate, residual_scale, eps, dtype):
        ctx.set_materialize_grads(False)
        n, dim = h.shape if h.dim() == 2 else (0, 0)
        if h.dim() != 2 or dim < 1:
            raise ValueError("h: [rows, channels]")
        for g in (pre_gain, post_gain):
            if g is not None and (g.dtype, g.shape, g.is_contiguous()) != (torch.bfloat16, (dim,), True):
                raise ValueError("gains: bf16 [channels]")
        if y is not None and gate is not None and gate.dtype != y.dtype:
            raise ValueError("a gate has the type of the block's output")
        if gate is not None and gate.dim() == 1 and (gate.shape[0] != dim or not gate.is_contiguous()):
            raise ValueError("gate: [channels] or [rows, channels]")
        _on_gpu(y, h, pre_gain, post_gain, gate)
        if gate is not None and gate.dim() == 2 and gate.shape == (n, dim) and gate.stride(0) < dim and (dim == 1 or gate.stride(1) == 1):
            gate = gate.contiguous()  # (one row for all, as a view: its gradient is one of each row, and stride 0 means [channels] to the call)
        ldy, ldh = _dense(y, n, dim, "y"), _dense(h, n, dim, "h")
        ldg = 0 if gate is None or gate.dim() == 1 else _dense(gate, n, dim, "gate")
        act = dtype if y is None else y.dtype
        e = lambda dtype: torch.empty(n, dim, dtype=dtype, device=h.device)  # noqa: E731
        h_out, x = e(h.dtype) if y is not None else None, e(act)
        code = _code(x)
        rstd = torch.empty(n, 2, dtype=torch.float32, device=h.device)
        _ok(V.vla_block_norm(_ptr(y), ldy, code, h.data_ptr(), ldh, _code(h), n, dim, _ptr(post_gain), _ptr(gate), ldg, residual_scale,
                             pre_gain.data_ptr(), eps, _ptr(h_out), dim, x.data_ptr(), dim, rstd.data_ptr(), _stream()))
        ctx.save_for_backward(y, h if y is None else h_out, pre_gain, post_gain, gate, rstd)
        ctx.residual_scale = residual_scale
        ctx.lds = ldy, ldh if y is None else dim, ldg
        if y is None:
            return x, None
        return x, h_out

    @staticmethod
    @once_differentiable
    def backward(ctx, d_x, d_h_out):
        y, h, pre_gain, post_gain, gate, rstd = ctx.saved_tensors
        n, dim = h.shape
        ldy, ldh, ldg = ctx.lds
        d_x = torch.zeros(n, dim, dtype=h.dtype if y is None else y.dtype, device=h.device) if d_x is None else d_x.contiguous()
        d_h_out = d_h_out.contiguous() if d_h_out is not None else None
        _on_gpu(d_x, d_h_out)
        e = lambda dtype, *s: torch.empty(*s, dtype=dtype, device=h.device)  # noqa: E731
        d_h, d_y = e(h.dtype, n, dim), e(y.dtype, n, dim) if y is not None else None
        d_pre, d_post = e(torch.float32, dim), e(torch.float32, dim) if post_gain is not None else None
        d_gate = None if gate is None else e(gate.dtype, n, dim) if ldg else e(torch.float32, dim)
        workspace = e(torch.uint8, V.vla_block_norm_grad_workspace_bytes(n, dim))
        _ok(V.vla_block_norm_grad(_ptr(y), ldy, _code(d_x), h.data_ptr(), ldh, _code(h), n, dim, _ptr(post_gain), _ptr(gate), ldg,
                                  ctx.residual_scale, pre_gain.data_ptr(), rstd.data_ptr(), d_x.data_ptr(), dim, _ptr(d_h_out), dim,
                                  d_h.data_ptr(), dim, _ptr(d_y), dim, _ptr(d_gate), dim, _ptr(d_post), d_pre.data_ptr(),
                                  workspace.data_ptr(), workspace.numel(), _stream()))
        cast = lambda g, t: g if g is None or g.dtype == t.dtype else g.to(t.dtype)  # noqa: E731
        return d_y, d_h, cast(d_pre, pre_gain), cast(d_post, post_gain), cast(d_gate, gate), None, None, None


def block_norm(y, h, pre_gain, post_gain=None, gate=None, residual_scale: float = 1.0, eps: float = 1e-6):
    """Between two blocks: ``h_out = h + residual_scale * gate * norm(y)`` and ``x = norm(h_out)``, the norms with their gains (bf16
    [channels]; without `post_gain` y is added as it is).  `gate`: [channels], [rows, channels] (an expanded row among them) or None, of
    y's type.
    Returns (x, h_out), both differentiable."""
    if y is None:
        raise ValueError("y: the block's output (first_norm takes the stream alone)")
    return _BlockNorm.apply(y, h, pre_gain, post_gain, gate, float(residual_scale), float(eps), None)


def first_norm(h, pre_gain, eps: float = 1e-6, dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """The first block's input, norm(h) with its gain (bf16 [channels]): of type `dtype` where h is float32, else (and by default) of h's."""
    return _BlockNorm.apply(None, h, pre_gain, None, None, 1.0, float(eps), dtype or h.dtype)[0]


def check() -> None:
    """Waits for the current stream and raises for what its operators found on the device (sequence starts among it)."""
    rc, bits = V.vla_op_read_status(_stream())
    _ok(rc)
    if bits:
        raise V.VlaError(V.VLA_ERR_DEVICE_STATUS, f"status bits {bits:#x}")
