"""Packed attention and its gradient write what is theirs and nothing else: every output and the workspace lie inside larger buffers, with
numbers between the rows, behind well-formed and malformed sequence starts."""
import pytest
import torch

from paper_2505_18719_gb300 import vla as V
from tests.test_gpu_learn import CODE, TYPE, stream
from tests.test_gpu_lm_ops import gen, ints, normal, status

pytestmark = pytest.mark.gpu

MARK = 0x5A


class Inside:
    """rows x width of `dtype` with `gap` elements between its rows, `around` bytes before and behind; what is not its own keeps MARK."""

    def __init__(self, rows, width, dtype, gap=0, around=8192):
        size = torch.empty(0, dtype=dtype).element_size()
        ld, self.around = width + gap, around
        nbytes = rows * ld * size
        self.raw = torch.full((2 * around + nbytes,), MARK, dtype=torch.uint8, device="cuda")
        self.rows = self.raw[around:around + nbytes].view(dtype).view(rows, ld)[:, :width]
        own = torch.zeros_like(self.raw, dtype=torch.bool)
        own[around:around + nbytes].view(rows, ld * size)[:, :width * size] = True
        self.other = ~own

    def untouched(self):
        return bool((self.raw[self.other] == MARK).all())


STARTS = [[0, 90], [5, 40, 40, 80], [0, 50, 40, 90], [-3, 50, 90], [0, 50, 91], [0, 1 << 30], [10, -5, 90], [-(1 << 30), 1 << 30, 7], [200, 300],
          [90, 0], [0, 90, 0, 90, 0, 90]]


@pytest.mark.parametrize("starts", STARTS)
@pytest.mark.parametrize("act,H,Hk,hd", [("f16", 4, 2, 64), ("bf16", 2, 2, 128), ("f16", 8, 1, 128)])
def test_nothing_outside_the_outputs_is_written(starts, act, H, Hk, hd):
    rows, dt, g = 90, TYPE[act], gen(90)
    q, k, v, d_out = [normal(g, rows, n * hd, dtype=dt) for n in (H, Hk, Hk, H)]
    at = ints(starts)
    out, lse = Inside(rows, H * hd, dt, gap=8), Inside(rows, H, torch.float32)
    d_q, d_k, d_v = Inside(rows, H * hd, dt, gap=16), Inside(rows, Hk * hd, dt, gap=8), Inside(rows, Hk * hd, dt, gap=24)
    n = V.vla_prompt_attn_grad_workspace_bytes(rows, H, Hk, hd)
    ws = Inside(1, n, torch.uint8)
    common = (q.data_ptr(), H * hd, k.data_ptr(), Hk * hd, v.data_ptr(), Hk * hd, CODE[act], rows, H, Hk, hd, at.data_ptr(), len(starts) - 1, hd ** -0.5)
    copies = [t.clone() for t in (q, k, v, d_out)]
    assert V.vla_prompt_attn(*common, out.rows.data_ptr(), out.rows.stride(0), lse.rows.data_ptr(), stream()) == 0
    formed = all(0 <= a <= b <= rows for a, b in zip(starts[:-1], starts[1:]))
    assert status() == (0 if formed else V.VLA_STATUS_SEQUENCES)
    kept = out.rows.clone()
    assert V.vla_prompt_attn_grad(*common, out.rows.data_ptr(), out.rows.stride(0), lse.rows.data_ptr(), d_out.data_ptr(), H * hd,
                                  d_q.rows.data_ptr(), d_q.rows.stride(0), d_k.rows.data_ptr(), d_k.rows.stride(0), d_v.rows.data_ptr(),
                                  d_v.rows.stride(0), ws.rows.data_ptr(), n, stream()) == 0
    assert status() == (0 if formed else V.VLA_STATUS_SEQUENCES)
    for name, b in (("out", out), ("lse", lse), ("d_q", d_q), ("d_k", d_k), ("d_v", d_v), ("workspace", ws)):
        assert b.untouched(), name
    same = lambda a, b: torch.equal(a.view(torch.int16), b.view(torch.int16))  # noqa: E731
    assert same(out.rows.contiguous(), kept.contiguous())
    for t, c in zip((q, k, v, d_out), copies):
        assert torch.equal(t, c)
