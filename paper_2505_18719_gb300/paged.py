"""Paged contexts and token log-probs for torch programs: tensors and streams around include/vla_lm.h.

``PagedCache`` holds the pool, the tables and the descriptors of every layer, ``token_logprobs`` is
differentiable.  All compute is in libvla.so, on torch's current stream; nothing waits for the GPU except
``PagedCache.check`` and the methods that return Python numbers.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch
from torch.autograd.function import once_differentiable

from . import vla as V

_CODE = {torch.float32: V.VLA_F32, torch.float16: V.VLA_F16, torch.bfloat16: V.VLA_BF16}


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


_capturing = torch.cuda.is_current_stream_capturing


def _ptr(t: Optional[torch.Tensor]) -> int:
    return t.data_ptr() if t is not None else 0


def _ok(rc: int) -> None:
    if rc != V.VLA_OK:
        raise V.VlaError(rc, V.vla_last_error())


def _on_gpu(*tensors: Optional[torch.Tensor]) -> None:
    for t in tensors:
        if t is not None and t.device.index != torch.cuda.current_device():
            raise ValueError(f"a tensor of the current GPU expected, got one on {t.device}")


def _code(t: torch.Tensor) -> int:
    if t.dtype not in _CODE:
        raise ValueError(f"float32, float16 or bfloat16 expected, got {t.dtype}")
    return _CODE[t.dtype]


def _rows_of(t: torch.Tensor, heads: int, hd: int) -> int:
    """Row stride of [rows, heads, hd] or [rows, heads * hd] whose rows are dense (a lone row's or head's does not count)."""
    if (t.dim() not in (2, 3) or t.shape[-1] != (hd if t.dim() == 3 else heads * hd) or t.stride(-1) != 1 or
            (t.dim() == 3 and (t.shape[1] != heads or (heads > 1 and t.stride(1) != hd)))):
        raise ValueError(f"rows of {heads} heads of {hd} expected, got {tuple(t.shape)} with strides {t.stride()}")
    return t.stride(0) if t.shape[0] > 1 else heads * hd


class Rows(NamedTuple):
    """The rows of one step: environment, position and cache slot of each (-1: padding), and each environment's first row."""
    env: torch.Tensor
    pos: torch.Tensor
    slot: torch.Tensor
    start: torch.Tensor


class PagedCache:
    """Keys and values of `layers` layers for `n_env` contexts that share `n_pages` pages of `page_size` positions.

    A step is ``rows = cache.plan(new_len, max_rows)`` and then, layer by layer, ``cache.append`` and ``cache.attend``.

    ``attend`` may run on several streams at once: each stream has a workspace of its own from its first call on.  Calls
    captured into CUDA graphs share ``workspace``, so the replays of one cache's graphs follow one another.
    """

    def __init__(self, n_env: int, n_pages: int, page_size: int, layers: int, n_heads: int, head_dim: int,
                 max_positions: int, dtype: torch.dtype = torch.float16, device="cuda"):
        i32 = dict(dtype=torch.int32, device=device)
        self.n_env, self.n_pages, self.page_size, self.n_heads, self.head_dim = n_env, n_pages, page_size, n_heads, head_dim
        self.max_pages = (max_positions + page_size - 1) // page_size
        # one buffer: keys and values of a page side by side, layer after layer
        self.data = torch.empty(layers, n_pages, 2, n_heads, page_size, head_dim, dtype=dtype, device=device)
        page = 2 * n_heads * page_size * head_dim
        self.layers = [V.VlaPagedKv(x[0, 0].data_ptr(), x[0, 1].data_ptr(), _CODE[dtype], n_pages, page_size, n_heads, head_dim, page,
                                    page_size * head_dim, head_dim) for x in self.data]
        self.table = torch.full((n_env, self.max_pages), -1, **i32)
        self.pool = torch.arange(n_pages - 1, -1, -1, **i32)
        self.n_free = torch.full((1,), n_pages, **i32)
        self.ctx = torch.zeros(n_env, **i32)
        nbytes = V.vla_paged_attn_workspace_bytes(head_dim)
        if not nbytes:
            raise V.VlaError(V.VLA_ERR_UNSUPPORTED, f"heads of {head_dim}")
        self.workspace = torch.zeros(nbytes, dtype=torch.uint8, device=device)
        self._stream_workspaces: dict[int, torch.Tensor] = {}

    def _workspace(self, stream: int) -> torch.Tensor:
        """Partial results and tickets of calls that may overlap must not mix (zeroed in the order of the stream that uses it)."""
        if _capturing():
            return self.workspace
        workspace = self._stream_workspaces.get(stream)
        if workspace is None:
            workspace = self._stream_workspaces[stream] = torch.zeros_like(self.workspace)
        return workspace

    def plan(self, new_len: torch.Tensor, max_rows: int, release: Optional[torch.Tensor] = None) -> Rows:
        """Takes pages for `new_len` (int32 [n_env] on the GPU) more tokens of each context; `release` (same shape)
        marks the contexts that start over first.  `max_rows` bounds the step's rows (a fixed number can be captured)."""
        for t in (new_len, release):
            if t is not None and (t.dtype, t.shape, t.is_contiguous()) != (torch.int32, (self.n_env,), True):
                raise ValueError("new_len and release: int32 [n_env], contiguous")
        _on_gpu(self.data, new_len, release)
        e = lambda n: torch.empty(n, dtype=torch.int32, device=self.ctx.device)  # noqa: E731
        rows = Rows(e(max_rows), e(max_rows), e(max_rows), e(self.n_env + 1))
        _ok(V.vla_page_plan(self.ctx.data_ptr(), new_len.data_ptr(), _ptr(release), self.n_env, self.page_size, self.table.data_ptr(),
                            self.max_pages, self.pool.data_ptr(), self.n_pages, self.n_free.data_ptr(), self.ctx.data_ptr(),
                            self.n_free.data_ptr(), rows.start.data_ptr(), rows.env.data_ptr(), rows.pos.data_ptr(),
                            rows.slot.data_ptr(), max_rows, _stream()))
        return rows

    def append(self, layer: int, q, k, v, rows: Rows, rope=None, interleaved: bool = False, q_gain=None, k_gain=None,
               eps: float = 1e-6) -> torch.Tensor:
        """Normalises (with gains) and rotates (with a table of ``rope_table``) q and k, files k and v; returns the queries."""
        hd = self.head_dim
        heads = q.shape[1] if q.dim() == 3 else q.shape[1] // hd
        if not q.dtype == k.dtype == v.dtype:
            raise ValueError("q, k and v have one type")
        for g in (q_gain, k_gain):
            if g is not None and (g.dtype, g.shape, g.is_contiguous()) != (torch.bfloat16, (hd,), True):
                raise ValueError("gains: bf16 [head_dim]")
        if not q.shape[0] == k.shape[0] == v.shape[0] == rows.pos.shape[0]:
            raise ValueError("q, k, v and the plan have the same rows")
        if rope is not None and (rope.dtype, rope.dim(), rope.shape[-1], rope.is_contiguous()) != (torch.float32, 3, 2, True):
            raise ValueError("rope: float32 [positions, rope_dim / 2, 2]")
        _on_gpu(self.data, q, k, v, rows.pos, rope, q_gain, k_gain)
        out = torch.empty(q.shape[0], heads, hd, dtype=q.dtype, device=q.device)
        _ok(V.vla_rope_append(q.data_ptr(), _rows_of(q, heads, hd), k.data_ptr(), _rows_of(k, self.n_heads, hd), v.data_ptr(),
                              _rows_of(v, self.n_heads, hd), _code(q), q.shape[0], heads, self.layers[layer], _ptr(q_gain),
                              _ptr(k_gain), eps, _ptr(rope), rope.shape[0] if rope is not None else 0,
                              2 * rope.shape[1] if rope is not None else 0, interleaved, rows.pos.data_ptr(), rows.slot.data_ptr(),
                              out.data_ptr(), heads * hd, _stream()))
        return out

    def attend(self, layer: int, q: torch.Tensor, rows: Rows, scale: Optional[float] = None, want_lse: bool = False):
        """Each row's attention over its context up to its own position: [rows, heads, head_dim] (and the log-sums)."""
        hd = self.head_dim
        heads = q.shape[1] if q.dim() == 3 else q.shape[1] // hd
        if q.shape[0] != rows.pos.shape[0]:
            raise ValueError("q and the plan have the same rows")
        _on_gpu(self.data, q, rows.pos)
        out = torch.empty(q.shape[0], heads, hd, dtype=q.dtype, device=q.device)
        lse = torch.empty(q.shape[0], heads, dtype=torch.float32, device=q.device) if want_lse else None
        stream = _stream()
        workspace = self._workspace(stream)
        _ok(V.vla_paged_attn(q.data_ptr(), _rows_of(q, heads, hd), _code(q), q.shape[0], heads, self.layers[layer],
                             self.table.data_ptr(), self.max_pages, self.n_env, rows.env.data_ptr(), rows.pos.data_ptr(),
                             hd ** -0.5 if scale is None else scale, out.data_ptr(), heads * hd, _ptr(lse), workspace.data_ptr(),
                             workspace.numel(), stream))
        return (out, lse) if want_lse else out

    def free_pages(self) -> int:
        return int(self.n_free.item())

    @staticmethod
    def check() -> None:
        """Waits for the current stream and raises for what its operators found on the device."""
        rc, bits = V.vla_op_read_status(_stream())
        _ok(rc)
        if bits:
            raise V.VlaError(V.VLA_ERR_DEVICE_STATUS, f"status bits {bits:#x}")


def rope_table(n_pos: int, rope_dim: int, theta: float = 1e4, device="cuda", **scaling) -> torch.Tensor:
    """(cos, sin) f32 [n_pos, rope_dim / 2, 2]; `scaling` as in ``vla_rope_table`` (kind, factor, original_len, low, high, amplitude)."""
    t = torch.empty(n_pos, rope_dim // 2, 2, dtype=torch.float32, device=device)
    _on_gpu(t)
    _ok(V.vla_rope_table(t.data_ptr(), n_pos, rope_dim, theta, stream=_stream(), **scaling))
    return t


class _TokenLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, temperature, top_k):
        if logits.dim() != 2 or logits.stride(1) != 1 or (tokens.dtype, tokens.shape, tokens.is_contiguous()) != (torch.int32, logits.shape[:1], True):
            raise ValueError("logits [rows, vocab] with dense rows, tokens int32 [rows]")
        _on_gpu(logits, tokens)
        n, vocab = logits.shape
        f = lambda *s: torch.empty(*s, dtype=torch.float32, device=logits.device)  # noqa: E731
        logprob, entropy, lse, top = f(n), f(n), f(n), f(n, top_k)
        ids = torch.empty(n, top_k, dtype=torch.int32, device=logits.device)
        _ok(V.vla_token_logprobs(logits.data_ptr(), logits.stride(0) if n > 1 else vocab, _code(logits), n, vocab, tokens.data_ptr(), temperature, top_k,
                                 logprob.data_ptr(), entropy.data_ptr(), lse.data_ptr(), ids.data_ptr() if top_k else 0,
                                 top.data_ptr() if top_k else 0, _stream()))
        ctx.save_for_backward(logits, tokens, lse, entropy)
        ctx.temperature = temperature
        ctx.mark_non_differentiable(lse, ids, top)
        return logprob, entropy, lse, ids, top

    @staticmethod
    @once_differentiable
    def backward(ctx, g_logprob, g_entropy, *_):
        logits, tokens, lse, entropy = ctx.saved_tensors
        n, vocab = logits.shape
        g_logprob, g_entropy = g_logprob.contiguous(), g_entropy.contiguous()
        d = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        _ok(V.vla_token_logprobs_grad(logits.data_ptr(), logits.stride(0) if n > 1 else vocab, _code(logits), n, vocab, tokens.data_ptr(),
                                      ctx.temperature, lse.data_ptr(), entropy.data_ptr(), g_logprob.data_ptr(), g_entropy.data_ptr(),
                                      d.data_ptr(), vocab, _stream()))
        return d, None, None, None


class TokenLogprobs(NamedTuple):
    logprob: torch.Tensor       # of each row's token, 0 where it is -1
    entropy: torch.Tensor
    lse: torch.Tensor
    top_ids: torch.Tensor
    top_logprobs: torch.Tensor


def token_logprobs(logits, tokens, temperature: float = 1.0, top_k: int = 0) -> TokenLogprobs:
    """Log-probs of `tokens` (int32 [rows], -1: none) under softmax(logits / temperature), with entropies and the `top_k`
    best ids.  Log-probs and entropies have gradients; rows without a token get none."""
    return TokenLogprobs(*_TokenLogprobs.apply(logits, tokens, float(temperature), int(top_k)))
