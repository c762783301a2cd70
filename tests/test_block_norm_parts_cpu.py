"""The CTAs that share the rows of a block norm's gradient are resident at once: their number, which the workspace's size shows, times their
threads' registers fits the SMs."""
import pytest

from paper_2505_18719_gb300 import vla as V

SMS, REGISTERS, A_THREAD = 152, 65536, 128


@pytest.mark.parametrize("dim", [*range(8, 4097, 8)])
def test_all_parts_are_resident(dim):
    parts, rest = divmod(V.vla_block_norm_grad_workspace_bytes(1 << 20, dim), 3 * 4 * dim)
    assert rest == 0 and parts % SMS == 0
    threads = -(-dim // (256 if dim <= 2048 else 512)) * 32  # 16-byte accesses: 8 elements a thread, 16 above 2048 channels
    assert parts // SMS * threads * A_THREAD <= REGISTERS
