"""Packed attention where scores or values are infinite or no numbers, against plain 64-bit forms; tolerances in learn_reference.py."""
import math

import pytest
import torch

from tests import learn_reference as R
from tests.test_gpu_learn import Prompt
from tests.test_gpu_lm_ops import status, within

pytestmark = pytest.mark.gpu


def tail_reference(p, a, b, first):
    """What rows first .. b - 1 of the sequence a .. b get when keys before `first` have no weight: the sequence that begins there."""
    part = [p.heads(t)[first:b] for t in (p.q, p.k, p.v)]
    return R.prompt(*part, [0, b - first], p.scale, p.act)


@pytest.mark.parametrize("act", ["f16", "bf16"])
@pytest.mark.parametrize("H,Hk,hd", [(4, 2, 64), (2, 2, 128)])
@pytest.mark.parametrize("n,hidden", [(300, 63), (300, 64), (300, 200), (1500, 80), (1500, 81), (1500, 700)])
@pytest.mark.parametrize("level", [0.0, -9.0, -20.0, -60.0, -400.0])
def test_prompt_attention_behind_keys_that_score_minus_infinity(act, H, Hk, hd, n, hidden, level):
    # `hidden` keys of no weight come first, whole blocks of them; the others score `level` give or take a few
    p = Prompt(50, [n], H, Hk, hd, act)
    q, k = p.heads(p.q), p.heads(p.k)
    q[:, :, 0] = 1.0
    k[:, :, 0] = level / p.scale
    k[:hidden, :, 0] = -math.inf
    out, lse = p.forward()
    assert status() == 0
    want, w_lse, t_out, t_lse = tail_reference(p, 0, n, hidden)
    within(p.heads(out)[hidden:], want, t_out, "out")
    within(lse[hidden:], w_lse, t_lse, "lse")
    # a row all of whose keys have no weight
    assert bool((out[:hidden] == 0).all()) and bool((lse[:hidden] == -math.inf).all())


def test_prompt_attention_first_block_far_below_the_next():
    # the reference of the running softmax follows a first block at -infinity and one far below the third
    p = Prompt(51, [300], 2, 2, 64, "f16")
    q, k = p.heads(p.q), p.heads(p.k)
    q[:, :, 0] = 1.0
    k[:, :, 0] = torch.linspace(-200, -20, 300, device="cuda")[:, None].half() / p.scale
    k[:64, :, 0] = -math.inf
    out, lse = p.forward()
    want, w_lse, t_out, t_lse = tail_reference(p, 0, 300, 64)
    within(p.heads(out)[64:], want, t_out, "out")
    within(lse[64:], w_lse, t_lse, "lse")
    assert status() == 0
