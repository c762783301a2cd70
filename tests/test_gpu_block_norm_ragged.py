"""Gradient of the block norm on tensors that begin at every offset and lie tight between others, against plain 64-bit forms; tolerances
in learn_reference.py.  What lies around the tensors is no number and stays as it is."""
import math

import pytest
import torch

from tests.test_gpu_learn import Norm
from tests.test_gpu_lm_ops import status

pytestmark = pytest.mark.gpu


class Tight(Norm):
    """Every tensor begins `offset` elements behind a 16-byte border; `gap` numbers lie between its rows."""

    def __init__(self, offset, gap, *args, **kw):
        super().__init__(*args, **kw)
        self.buffers = []

        def place(t, at):
            if t is None:
                return None
            rows, dim = t.shape if t.dim() == 2 else (1, t.shape[0])
            ld = dim + gap if t.dim() == 2 else dim
            buf = torch.full((at + rows * ld + 64,), math.nan, dtype=t.dtype, device="cuda")
            view = buf[at:at + rows * ld].view(rows, ld)[:, :dim]
            view.copy_(t.view(rows, dim))
            outside = torch.ones_like(buf, dtype=torch.bool)
            outside[at:at + rows * ld].view(rows, ld)[:, :dim] = False
            self.buffers.append((buf, outside))
            return view if t.dim() == 2 else view[0]

        self.y, self.h, self.gate = place(self.y, offset), place(self.h, offset + 1), place(self.gate, offset + 2)
        self.d_x, self.d_h_out = place(self.d_x, offset + 3), place(self.d_h_out, offset + 4)
        self.new = lambda dtype: place(torch.full((self.rows, self.dim), 7.0, dtype=dtype, device="cuda"), offset + 5)

    def check(self, **kw):
        super().check(**kw)
        assert status() == 0
        for buf, outside in self.buffers:
            assert bool(torch.isnan(buf[outside]).all())


@pytest.mark.parametrize("act,stream_type", [("bf16", "f32"), ("f16", "f16"), ("f32", "f32")])
@pytest.mark.parametrize("offset", range(8))
@pytest.mark.parametrize("gap", [0, 1, 8])
def test_gradients_of_tight_rows(offset, gap, act, stream_type):
    for rows, dim in ((1, 1), (9, 1), (5, 2), (4, 3), (3, 7), (2, 8), (1, 9), (3, 15), (2, 17), (3, 33), (2, 255)):
        Tight(offset, gap, 80 + dim, rows, dim, act, stream_type, True, "row").check()
    Tight(offset, gap, 99, 700, 41, act, stream_type, False, "channel").check(with_h_out=False)


@pytest.mark.parametrize("dim", [2049, 4100, 8193, 12345])
def test_gradients_of_long_tight_rows(dim):
    for offset in (1, 4, 7):
        Tight(offset, 0, dim, 4, dim, "bf16", "bf16", True, "row").check()
        Tight(offset, 3, dim, 3, dim, "f16", "f32", True, "none").check()
