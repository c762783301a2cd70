"""fp32 queries of any size over an fp16 cache: a score keeps 22 bits of its products whatever the queries' scale."""
import pytest
import torch

from tests.test_gpu_lm_ops import attend_call, attend_check, attend_state, gen, normal, status, workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,Hk,hd", [(4, 4, 64), (12, 2, 64), (1, 1, 128), (16, 4, 128), (10, 1, 128)])
@pytest.mark.parametrize("std", [1e-30, 1e-8, 1e-4, 1e-2, 1.0, 1e4, 1e8, 1e30])
def test_paged_attn_queries_of_any_size(H, Hk, hd, std):
    lengths = [1, 0, 2, 33, 300, 129, 64]
    q, k, v, table, env, pos = attend_state(H * hd, lengths, H, Hk, hd, "f32", "f16", 16, "head", q_std=1.0)
    q = q * std
    scale = hd ** -0.5 / std
    out, lse = attend_call(q, k, v, table, env, pos, "f32", "f16", scale, workspace(hd))
    attend_check(q, k, v, table, 16, env, pos, "f32", "f16", out, lse, scale)
    assert status() == 0


def test_paged_attn_queries_of_each_heads_own_size():
    # heads (and rows) of one call far apart in size, some of them zero; a head's channels apart by 2^12
    H, hd = 8, 128
    q, k, v, table, env, pos = attend_state(5, [300, 77, 128, 1, 2000], H, 4, hd, "f32", "f16", 16, "head", q_std=1.0)
    q[:, 1] *= 2.0 ** -20
    q[:, 2] *= 2.0 ** 9
    q[1] *= 2.0 ** -9
    q[:, 3] = 0.0
    q[:, 4, ::2] *= 2.0 ** -12
    q[0, 5, 7] = 0.0
    out, lse = attend_call(q, k, v, table, env, pos, "f32", "f16", 0.05, workspace(hd))
    attend_check(q, k, v, table, 16, env, pos, "f32", "f16", out, lse, 0.05)
    assert status() == 0
