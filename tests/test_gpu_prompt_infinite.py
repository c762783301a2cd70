"""Packed attention where scores or values are infinite or no numbers, against plain 64-bit forms; tolerances in learn_reference.py."""
import math

import pytest
import torch

from paper_2505_18719_gb300 import vla as V
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


def rows_reference(p, a, rows):
    """(out, lse, tolerances) of the given rows of the sequence from a on that 32-bit dot products compute, keys one by one, in 64 bits.
    A channel in which a row sees a value that is no number has none itself."""
    q, k, v = [p.heads(t).to(R.F64) for t in (p.q, p.k, p.v)]
    out, t_out = [torch.zeros(len(rows), p.H, p.hd, dtype=R.F64, device="cuda") for _ in range(2)]
    lse, t_lse = [torch.zeros(len(rows), p.H, dtype=R.F64, device="cuda") for _ in range(2)]
    at = torch.tensor(rows, device="cuda")
    n = max(rows) + 1 - a
    for h in range(p.H):
        K, W = k[a:a + n, h // (p.H // p.Hk)], v[a:a + n, h // (p.H // p.Hk)]
        seen = torch.arange(a, a + n, device="cuda")[None] <= at[:, None]
        s = torch.where(seen, p.scale * q[at, h] @ K.T, -math.inf)
        w = torch.softmax(s, -1)
        number = torch.isfinite(W)
        out[:, h] = torch.where(seen.to(R.F64) @ (~number).to(R.F64) > 0, math.nan, w @ torch.where(number, W, 0.0))
        lse[:, h] = torch.logsumexp(s, -1)
        # a score: a rounding for each of its products and sums; sums over the keys, whose roundings fall either way; the result's own
        e_s = torch.where(seen, p.scale * q[at, h].abs() @ K.abs().T, 0.0).amax(-1, keepdim=True) * (p.hd + 4) * R.E
        size = w @ torch.where(number, W, 0.0).abs()
        t_out[:, h] = R.U[p.act] * out[:, h].abs() + (2 * e_s + 2 * (8 + n ** 0.5) * R.E) * size + R.TINY[p.act]
        t_lse[:, h] = e_s.squeeze(-1) + (8 + n ** 0.5) * R.E + 4 * R.E * lse[:, h].abs()
    return out, lse, t_out, t_lse


@pytest.fixture
def short_waits():
    # 2 ms a wait, of 1 s: shorter than what is computed again below takes
    assert V.vla_test_set_wait_limit_ns(2_000_000) == 0
    yield
    V.vla_test_set_wait_limit_ns(0)


@pytest.mark.parametrize("act", ["f16", "bf16"])
def test_rows_computed_again_keep_no_other_sequence_waiting(act, short_waits):
    # a NaN in the last value of a long sequence: the rows before it in its tile are computed again, over all their keys, while the
    # other warps of that CTA wait with the rows of the next sequence
    p = Prompt(52, [16384, 8192], 4, 2, 64, act)
    want, w_lse = p.forward()
    assert status() == 0
    bad = 16383
    p.heads(p.v)[bad] = math.nan
    out, lse = p.forward()
    assert status() == 0
    rest = [i for i in (*range(bad // 128 * 128), *range(bad + 1, p.rows))]
    assert torch.equal(out[rest], want[rest]) and torch.equal(lse[rest], w_lse[rest])
    tile = list(range(bad // 128 * 128, bad))
    exact, e_lse, t_out, t_lse = rows_reference(p, 0, tile)
    within(p.heads(out)[tile], exact, t_out, "out")
    within(lse[tile], e_lse, t_lse, "lse")
    assert bool(torch.isnan(p.heads(out)[bad]).all())


@pytest.mark.parametrize("act,hd", [("f16", 64), ("bf16", 128)])
@pytest.mark.parametrize("n", [700, 1700])
@pytest.mark.parametrize("where", ["first channel", "first row", "here and there", "tile ends", "scattered"])
def test_a_value_without_a_number_shows_in_its_channel_from_its_row_on(n, where, act, hd):
    p = Prompt(53, [40, n, 90], 4, 2, hd, act)
    v = p.heads(p.v)
    clean = p.forward()
    if where == "first channel":
        v[40, :, 0] = math.nan
    elif where == "first row":
        v[40] = math.nan
    elif where == "here and there":  # (the second key-value head has one row only)
        v[40, 0, 0], v[40 + 130, 0, 1], v[40 + 300, 0], v[40 + n - 2, 1, 5] = [math.nan] * 4
    elif where == "tile ends":  # rows that see one in another channel, spoilt by the last of each tile
        v[40, :, 7] = math.nan
        for i in range(127, n, 128):
            v[40 + i, :, i // 128] = math.nan
    else:
        at = torch.randint(0, n, (20,), generator=torch.Generator().manual_seed(3))
        for i, r in enumerate(at.tolist()):
            v[40 + r, i % 2, (7 * i) % hd] = math.nan
    out, lse = p.forward()
    assert status() == 0
    rows = list(range(40, 40 + n))
    want, _, _, _ = rows_reference(p, 40, rows)
    numbers = torch.where(torch.isfinite(v), v, 0)
    _, _, tol, _ = R.prompt(p.heads(p.q), p.heads(p.k), numbers, p.start, p.scale, act)
    within(p.heads(out)[40:40 + n], want, tol[40:40 + n], "out")
    assert torch.equal(lse, clean[1]) or bool(((lse - clean[1]).abs() <= 1e-5 * (1 + clean[1].abs())).all())
    for part in (slice(0, 40), slice(40 + n, p.rows)):
        assert torch.equal(out[part], clean[0][part])


def test_values_near_the_largest_bf16():
    # sums of weights up to 2^8 with a reference that lags behind pass the largest number; the row itself does not
    p = Prompt(54, [900], 2, 1, 64, "bf16")
    q, k, v = p.heads(p.q), p.heads(p.k), p.heads(p.v)
    q[:] = 0
    q[:, :, 0] = 1
    k[:] = 0
    k[:, :, 0] = (torch.linspace(0, 5.0, 900, device="cuda")[:, None] / p.scale).bfloat16()
    v[:] = 1e34
    out, lse = p.forward()
    assert status() == 0
    want, w_lse, t_out, t_lse = R.prompt(q, k, v, p.start, p.scale, "bf16")
    within(p.heads(out), want, t_out, "out")
    within(lse, w_lse, t_lse, "lse")


def test_a_long_sequence_without_numbers_takes_no_longer(short_waits):
    p = Prompt(55, [16384, 300], 8, 2, 128, "bf16")

    def time():
        best = math.inf
        for _ in range(3):
            a, b = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
            a.record()
            got = p.forward()
            b.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(b))
        assert status() == 0
        return (*got, best)

    out, lse, ms = time()
    for name in ("v", "k", "q"):
        t = p.heads(getattr(p, name))
        keep = t[0].clone()
        for channels in (slice(None), slice(3, 4)):
            t[0, :, channels] = math.nan
            o2, l2, ms2 = time()
            assert torch.equal(o2[16384:], out[16384:]) and torch.equal(l2[16384:], lse[16384:])
            if name != "q":
                assert bool(torch.isnan(p.heads(o2)[:16384, :, channels]).all())
            assert ms2 < 10 * ms  # (each row computed again: 100 times)
            t[0] = keep
