"""The learning example: every weight's gradient against 64-bit autograd, and what the operators do at the ends of their ranges
(the kernel for long sequences over short ones, rows further apart than 32 bits of bytes, many calls at once)."""
import math

import pytest
import torch

from examples import packed_learning as X
from paper_2505_18719_gb300 import paged as P
from tests import learn_reference as R
from tests.test_gpu_learn import HEADS, Prompt, starts_of
from tests.test_gpu_lm_ops import gen, ints, normal, status

pytestmark = pytest.mark.gpu
F64 = torch.float64


def dense_objective(policy, leaves, data, advantages):
    """The example's objective from elementary operations in 64 bits, around the log-probs that it has itself."""
    it = iter(leaves)
    embed, first, head = next(it), next(it), next(it)
    layers = [{k: next(it) for k in w} for w in policy.layers]
    ids, start, pos, tokens = data
    norm = lambda t, w: t / (t.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt() * w  # noqa: E731
    cos, sin = policy.rope[pos].to(F64).unbind(-1)

    def rotated(x):
        a, b = x.view(x.shape[0], -1, policy.hd).chunk(2, -1)
        return torch.cat([a * cos[:, None] - b * sin[:, None], b * cos[:, None] + a * sin[:, None]], -1)

    h = embed[ids]
    x = norm(h, first)
    widths = [policy.heads * policy.hd, policy.kv_heads * policy.hd, policy.kv_heads * policy.hd]
    bounds = start.tolist()
    for w in layers:
        q, k, v = (x @ w["qkv"].t()).split(widths, -1)
        q, k, v = rotated(q), rotated(k).repeat_interleave(2, 1), v.view(v.shape[0], -1, policy.hd).repeat_interleave(2, 1)
        parts = []
        for a, b in zip(bounds[:-1], bounds[1:]):
            s = torch.einsum("nhd,mhd->hnm", q[a:b], k[a:b]) * policy.hd ** -0.5
            s = s.masked_fill(torch.ones(b - a, b - a, dtype=torch.bool, device="cuda").triu(1), -math.inf)
            parts.append(torch.einsum("hnm,mhd->nhd", torch.softmax(s, -1), v[a:b]))
        parts.append(torch.zeros(q.shape[0] - bounds[-1], *q.shape[1:], dtype=F64, device="cuda"))
        y = torch.cat(parts).flatten(1) @ w["o"].t()
        h = h + 0.5 * w["attn_gate"] * norm(y, w["attn_norm"])
        x = norm(h, w["ffn_norm"])
        h = h + 0.5 * w["ffn_gate"] * (torch.nn.functional.silu(x @ w["up"].t()) @ w["down"].t())
        x = norm(h, w["next_norm"])
    lp = torch.log_softmax(x @ head.t(), -1)
    live = tokens >= 0
    chosen = torch.where(live, lp.gather(1, tokens.clamp(min=0).long()[:, None])[:, 0], 0.0)
    entropy = -(lp.exp() * lp).sum(-1)
    seq = torch.searchsorted(start[1:].long(), torch.arange(ids.shape[0], device="cuda"), right=True).clamp(max=len(bounds) - 2)
    change = torch.zeros(len(bounds) - 1, dtype=F64, device="cuda").index_add(0, seq, chosen - chosen.detach())
    ratio, adv = torch.exp(change), advantages.to(F64)
    clipped = torch.minimum(ratio * adv, ratio.clamp(0.8, 1.2) * adv).mean()
    return clipped + 0.01 * (entropy * live).sum() / live.sum()


def test_learning_step_gradients_reach_every_weight():
    policy, data = X.Decoder(), X.batch()
    with torch.no_grad():
        old = P.token_logprobs(policy.logits(*data[:3]), data[3]).logprob
    # (ratios of 1: inside the clip)
    advantages = torch.tensor([1.0, -0.5, 0.25, 0.8], device="cuda")
    value, grads = X.learning_step(policy, data, old, advantages)
    leaves = [t.detach().to(F64).requires_grad_() for t in policy.leaves()]
    want = torch.autograd.grad(dense_objective(policy, leaves, data, advantages), leaves)
    # about 60 bf16 roundings lie on a path from a weight to the objective and back, of random sign: 8 half-steps each way
    for t, a, b in zip(policy.leaves(), grads, want):
        assert a.shape == t.shape and a.dtype == t.dtype
        assert float((a.to(F64) - b).norm()) <= 16 * R.U["bf16"] * float(b.norm()), t.shape


@pytest.mark.parametrize("H,Hk,hd", HEADS)
@pytest.mark.parametrize("act", ["f16", "bf16"])
def test_long_and_short_sequences_in_one_batch(H, Hk, hd, act):
    # 800 rows a sequence on average: the kernel for long sequences, over lengths of 1, of part of a tile and of none too
    Prompt(50, [2700, 1, 129, 0, 1100, 81, 1589], H, Hk, hd, act, behind=2).check()


@pytest.mark.parametrize("seqs,length", [(5, 768), (5, 767), (2, 769)])
def test_around_the_mean_length_that_parts_the_kernels(seqs, length):
    Prompt(51, [length] * seqs, 4, 2, 128, "bf16").check()


def test_rows_whose_offsets_pass_32_bits():
    rows, H, Hk, hd, ld = 40000, 2, 1, 64, 65536  # 2.6e9 elements from the first row to the last
    g = gen(52)
    p = Prompt(53, [39000, 900], H, Hk, hd, "bf16", before=60, behind=40)
    near = [t.contiguous() for t in (p.q, p.k, p.v)]
    want = p.forward()
    want_grad = p.backward(*want)
    buffer = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda")
    far, at = [], 0
    for t in near:
        view = buffer.as_strided((rows, t.shape[1]), (ld, 1), at)
        view.copy_(t)
        far.append(view)
        at += t.shape[1]
    p.q, p.k, p.v = far
    got = p.forward()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all(torch.equal(a, b) for a, b in zip(p.backward(*got), want_grad))
    assert status() == 0
    del g


def test_many_calls_beside_other_work_give_equal_bits():
    side = torch.cuda.Stream()
    x = torch.randn(2048, 2048, device="cuda", dtype=torch.bfloat16)
    for lengths, H, Hk, hd, act in (([1500], 3, 1, 64, "bf16"), ([5, 300, 290, 288] * 6, 8, 8, 128, "f16"), ([3000, 77], 7, 1, 128, "bf16")):
        p = Prompt(54, lengths, H, Hk, hd, act)
        out = p.forward()
        grad = p.backward(*out)
        torch.cuda.synchronize()
        for i in range(40):
            if i % 3 == 0:
                with torch.cuda.stream(side):
                    x @ x
            assert all(torch.equal(a, b) for a, b in zip(p.forward(), out))
            assert all(torch.equal(a, b) for a, b in zip(p.backward(*out), grad))
    assert status() == 0


def test_a_captured_step_of_the_functions():
    from paper_2505_18719_gb300 import learn as L
    g = gen(55)
    x = normal(g, 300, 512, dtype=torch.bfloat16).requires_grad_()
    start = ints(starts_of([100, 150]))
    h = normal(g, 300, 256)
    gain = torch.ones(256, dtype=torch.bfloat16, device="cuda")

    def step():
        q, k, v = x.split([256, 128, 128], -1)
        y = L.prompt_attention(q, k, v, start, 64).flatten(1)
        z, s = L.block_norm(y, h, gain, gain)
        return torch.autograd.grad((z.float() + s).sum(), [x])[0]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        got.fill_(1.0)
        graph.replay()
        assert torch.equal(got, want)
