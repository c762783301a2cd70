"""Gates of the block norm that are broadcast views: the gradient comes back in the shape that went in."""
import pytest
import torch

from paper_2505_18719_gb300 import learn as L
from tests.test_gpu_lm_ops import gen, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,dim", [(45, 264), (7, 33), (1, 64), (5, 1)])
def test_an_expanded_gate(rows, dim):
    g = gen(70)
    h, y = normal(g, rows, dim), normal(g, rows, dim, dtype=torch.bfloat16)
    pre = post = (1 + 0.2 * normal(g, dim)).bfloat16()
    wx, wh = normal(g, rows, dim, dtype=torch.bfloat16), normal(g, rows, dim)
    base = normal(g, *((dim,) if dim > 1 else ()), dtype=torch.bfloat16)  # (one channel: of no strides at all)

    def gradients(gate_of):
        leaves = [t.detach().clone().requires_grad_() for t in (y, h, pre, post, base)]
        gate = gate_of(leaves[4])
        x, h_out = L.block_norm(leaves[0], leaves[1], leaves[2], leaves[3], gate, residual_scale=0.3)
        return x, h_out, torch.autograd.grad((x * wx).float().sum() + (h_out * wh).sum(), [*leaves, gate])

    x, h_out, got = gradients(lambda t: t.expand(rows, dim))
    x2, h2, want = gradients(lambda t: t.expand(rows, dim).contiguous())
    assert got[-1].shape == (rows, dim) and got[-2].shape == base.shape
    assert torch.equal(x, x2) and torch.equal(h_out, h2)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_a_gate_of_equal_channels_is_refused():
    h, y, gain = torch.ones(4, 16, device="cuda"), torch.ones(4, 16, dtype=torch.bfloat16, device="cuda"), torch.ones(16, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        L.block_norm(y, h, gain, gate=y[:, :1].expand(4, 16))
