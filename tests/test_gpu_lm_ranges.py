"""The token log-probs far from zero, against plain 64-bit forms.

A log-prob depends on differences of logits alone, so its tolerance here goes by the row's spread, not by how far from
zero the row lies: `E` = 2^-24 for every 32-bit rounding, 8 of them for a difference and its products, and those of a
sum of `vocab` weights as in test_gpu_lm_ops.py."""
import math

import pytest
import torch

from tests.test_gpu_lm_ops import E, F64, TINY, TYPE, U, gen, grad_call, ints, logprob_call, logprob_reference, normal, status, within

pytestmark = pytest.mark.gpu


def spread_of(x, T):
    """Largest less smallest finite logit of each row, over T."""
    z = x.to(F64)
    finite = torch.isfinite(z)
    top = torch.where(finite, z, -math.inf).amax(-1)
    low = torch.where(finite, z, math.inf).amin(-1)
    return ((top - low) / T).clamp(min=0.0)


def check_differences(x, tokens, T, top, got):
    want = logprob_reference(x, tokens, T, top)
    vocab = x.shape[1]
    tol = 8 * E * spread_of(x, T) + (32 + 4 * vocab ** 0.5) * E + 8 * E * math.log(vocab + 1)
    within(got["logprob"], want["logprob"], 2 * tol, "logprob")
    within(got["entropy"], want["entropy"], tol * (2 + math.log(vocab)), "entropy")
    # the log-sum itself has the size of the logits
    size = torch.where(torch.isfinite(x), x.to(F64), 0.0).abs().amax(-1) / T
    within(got["lse"], want["lse"], 8 * E * size + tol, "lse")
    if top:
        assert torch.equal(got["ids"].long(), want["ids"]), "ids"
        within(got["lps"], want["lps"], 2 * tol[:, None], "top log-probs")


# a row of one warp, of a CTA, of a CTA with all its rounds, and one cut over a cluster
VOCABS = [(6, 40), (9, 4099), (5, 32064), (3, 100003)]


@pytest.mark.parametrize("act", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,vocab", VOCABS)
@pytest.mark.parametrize("T", [1.0, 0.7, 1.5])
def test_token_logprobs_keep_their_bits_far_from_zero(act, rows, vocab, T):
    g = gen(vocab + 1)
    for far in (0.0, 31.0, 1e3, 1e4, 1e5, 1e6, 9e6, 3e7, 1e9) if act == "f32" else (0.0, 31.0, 1e3, 1e4):
        for sign in (-1.0, 1.0):
            x = (normal(g, rows, vocab, std=2.5) + sign * far).to(TYPE[act])
            tokens = torch.randint(0, vocab, (rows,), generator=g, device="cuda").to(torch.int32)
            got = logprob_call(x, tokens, T, 0, act)
            assert status() == 0
            check_differences(x, tokens, T, 0, got)


@pytest.mark.parametrize("rows,vocab", VOCABS)
@pytest.mark.parametrize("limit,T", [(11629079.5, 1.0), (11.6290795, 2.0 ** -20 * 1.048576), (2907269.75, 0.25)])
def test_token_logprobs_around_the_largest_reference(rows, vocab, limit, T):
    # rows whose logits lie on both sides of z log2(e) / T = -2^24, from which on differences are taken first
    T = float(torch.tensor(T, dtype=torch.float32))
    g = gen(vocab)
    steps = torch.randint(-3, 4, (rows, vocab), generator=g, device="cuda").to(torch.float32)
    for sign in (-1.0, 1.0):
        x = sign * limit + steps * T
        x[0] = -math.inf  # one weight of e^-1 beside the largest, from one thread (and slice) to another
        x[0, 0], x[0, vocab - 1] = sign * limit + 0.5 * T, sign * limit - 0.5 * T
        tokens = ints([vocab - 1] + list(range(1, rows)))
        got = logprob_call(x, tokens, T, 2, "f32")
        assert status() == 0
        check_differences(x, tokens, T, 2, got)


def check_gradient(x, tokens, T, g, h, act):
    rows, vocab = x.shape
    fwd = logprob_call(x, tokens, T, 0, act)
    d = grad_call(x, tokens, T, fwd["lse"], fwd["entropy"], g, h, act)
    want = logprob_reference(x, tokens, T, 0)
    lp, p, H = want["lp"], want["p"], want["entropy"][:, None]
    gg, hh = g.to(F64)[:, None], h.to(F64)[:, None]
    lp0 = torch.where(p > 0, lp, 0.0)
    exact = -gg * p - hh * p * (lp0 + H)
    exact.scatter_add_(1, tokens.long().clamp(min=0)[:, None], gg)
    kept = (tokens >= 0)[:, None]
    exact = torch.where(kept, exact / T, 0.0)
    # a log-sum of up to 128 is off by half of its last place, 2^-18
    eps = 2.0 ** -18 + 16 * E * (spread_of(x, T)[:, None] + H + 2) + 2 * (32 + 4 * vocab ** 0.5) * E
    tol = eps * p * (gg.abs() + hh.abs() * (lp0.abs() + H + 1) * (2 + math.log(vocab))) / T
    tol.scatter_add_(1, tokens.long().clamp(min=0)[:, None], 4 * E * gg.abs() / T)
    within(d, exact, torch.where(kept, tol + U[act] * exact.abs() + TINY[act], 0.0), "gradient")
    own = x.clone()
    assert torch.equal(grad_call(own, tokens, T, fwd["lse"], fwd["entropy"], g, h, act, out=own), d)
    assert status() == 0


# few long rows are cut: in place, CTAs write slices of a row that the others read first
GRAD_VOCABS = [(6, 40), (9, 4099), (700, 1000), (40, 32064), (2, 151937), (1, 600001)]


@pytest.mark.parametrize("act", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,vocab", GRAD_VOCABS)
@pytest.mark.parametrize("T", [1.0, 0.5, 0.7, 3.3])
def test_token_logprobs_grad_far_from_zero(act, rows, vocab, T):
    T = float(torch.tensor(T, dtype=torch.float32))
    gn = gen(vocab + 2)
    for far in (0.0, 31.0, 100.0, 1e3, 1e4, 1e6, 9e6, 3e7) if act == "f32" else (0.0, 31.0, 100.0, 1e3, 1e4):
        for sign in (-1.0, 1.0):
            x = (normal(gn, rows, vocab, std=2.0) + sign * far).to(TYPE[act])
            x[::3, :vocab // 3] = -math.inf
            tokens = vocab - 1 - torch.randint(0, vocab // 2, (rows,), generator=gn, device="cuda").to(torch.int32)
            if rows > 4:
                tokens[4] = -1
            check_gradient(x, tokens, T, normal(gn, rows), normal(gn, rows, std=0.3), act)


@pytest.mark.parametrize("act", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,vocab", GRAD_VOCABS)
@pytest.mark.parametrize("T", [1.0, 0.5, 0.7, 4.0, 1.3, 1e-6, 1e6])
def test_token_logprobs_grad_of_the_lowest_and_largest_values(act, rows, vocab, T):
    T = float(torch.tensor(T, dtype=torch.float32))
    # masks of a type's lowest value: one of several ids left, and rows of nothing else, whose log-sum is past 32 bits at T < 1
    gn = gen(vocab + 3)
    low = torch.finfo(TYPE[act]).min
    x = torch.full((rows, vocab), low, dtype=TYPE[act], device="cuda")
    x[1::3] = -low                                    # the same of the largest value
    x[2::3, vocab // 2:] = normal(gn, 1, vocab - vocab // 2, std=2.0).to(TYPE[act])
    tokens = vocab - 1 - torch.randint(0, vocab // 3, (rows,), generator=gn, device="cuda").to(torch.int32)
    fwd = logprob_call(x, tokens, T, 0, act)
    g, h = T * normal(gn, rows), T * normal(gn, rows, std=0.3)
    d = grad_call(x, tokens, T, fwd["lse"], fwd["entropy"], g, h, act)
    # equal logits (or equal ones beside weights of zero) are a difference of 0: the row's spread does not count
    z = x.to(F64)
    lp = torch.log_softmax((z - z.amax(-1, keepdim=True)) / T, -1)
    p = lp.exp()
    H = torch.special.entr(p).sum(-1, keepdim=True)
    lp0 = torch.where(p > 0, lp, 0.0)
    gg, hh = g.to(F64)[:, None], h.to(F64)[:, None]
    exact = -gg * p - hh * p * (lp0 + H)
    exact.scatter_add_(1, tokens.long()[:, None], gg)
    exact = exact / T
    spread = torch.where(p > 0, -lp, 0.0).amax(-1, keepdim=True)
    eps = 2.0 ** -18 + 16 * E * (spread + H + 2) + 2 * (32 + 4 * vocab ** 0.5) * E
    tol = eps * p * (gg.abs() + hh.abs() * (lp0.abs() + H + 1) * (2 + math.log(vocab))) / T
    tol.scatter_add_(1, tokens.long()[:, None], 4 * E * gg.abs() / T)
    within(d, exact, tol + U[act] * exact.abs() + TINY[act], "gradient")
    own = x.clone()
    assert torch.equal(grad_call(own, tokens, T, fwd["lse"], fwd["entropy"], g, h, act, out=own), d)
    assert status() == 0
