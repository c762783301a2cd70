"""Gradient of the packed attention in fp16 where gradients of very different sizes lie side by side, against plain 64-bit forms.

The kernels round dS to fp16 times a power of two that brings the largest it can be in a row (of d_q: a query's, over the keys it sees; of
d_k: a key's, over the queries that see it) to 2^13 at least and 2^15 at most.  Half the spacing of the smallest fp16 numbers is 2^-25, so
beside the relative half-step a dS is off by at most 2^-38 of that largest.  The rest is as in learn_reference.py."""
import math

import pytest
import torch

from paper_2505_18719_gb300 import vla as V
from tests import learn_reference as R
from tests.test_gpu_learn import Prompt
from tests.test_gpu_lm_ops import gen, status, within

pytestmark = pytest.mark.gpu

F64 = R.F64


def gradients(p, out, lse):
    """d_q, d_k, d_v in 64 bits from the given out and lse, and their tolerances."""
    H, Hk, hd, group = p.H, p.Hk, p.hd, p.H // p.Hk
    z = lambda n: torch.zeros(p.rows, n, hd, dtype=F64, device="cuda")  # noqa: E731
    dq, tq, dk, tk, dv, tv = z(H), z(H), z(Hk), z(Hk), z(Hk), z(Hk)
    q, k, v, o, g_out = [p.heads(t).to(F64) for t in (p.q, p.k, p.v, out, p.d_out)]
    lse = lse.to(F64)
    u, floor = 1.01 * R.U["f16"], 2.0 ** -38
    for a, b in zip(p.start[:-1], p.start[1:]):
        n = b - a
        if not n:
            continue
        seen = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
        s_n = R.sum_error(n * group)
        for g in range(Hk):
            K, W = k[a:b, g], v[a:b, g]
            heads = range(g * group, (g + 1) * group)
            size_g = torch.stack([g_out[a:b, h].norm(dim=-1) for h in heads]).amax(0)
            size_d = torch.stack([(g_out[a:b, h] * o[a:b, h]).sum(-1).abs() for h in heads]).amax(0)
            behind = lambda t: t.flip(0).cummax(0).values.flip(0)  # noqa: E731 (the largest of the queries from a key on)
            most_k = W.norm(dim=-1) * behind(size_g) + behind(size_d)
            most_v = W.norm(dim=-1).cummax(0).values
            for h in heads:
                Q, G, O, L = q[a:b, h], g_out[a:b, h], o[a:b, h], lse[a:b, h, None]  # noqa: E741
                w = torch.where(seen, torch.exp(torch.where(seen, p.scale * Q @ K.T - L, 0.0)), 0.0)
                e_p = torch.where(seen, p.scale * (Q.abs() @ K.abs().T) * (R.sum_error(hd) + 4 * R.E), 0.0) + 4 * R.E * L.abs() + 8 * R.E
                D = (G * O).sum(-1, keepdim=True)
                dp = G @ W.T
                e_d = (G.abs() @ W.abs().T + (G * O).abs().sum(-1, keepdim=True)) * R.sum_error(hd)
                ds = w * (dp - D)
                e_ds = (u + e_p) * ds.abs() + w * e_d
                least = lambda t: torch.where(seen, floor * t, 0.0)  # noqa: E731
                e_q = e_ds + least((G.norm(dim=-1) * most_v + D.squeeze(-1).abs())[:, None])
                e_k = e_ds + least(most_k[None])
                dq[a:b, h] = p.scale * ds @ K
                tq[a:b, h] = p.scale * (e_q + s_n * ds.abs()) @ K.abs()
                dk[a:b, g] += p.scale * ds.T @ Q
                tk[a:b, g] += p.scale * (e_k + s_n * ds.abs()).T @ Q.abs()
                dv[a:b, g] += w.T @ G
                tv[a:b, g] += ((u + e_p) * w + least(torch.ones_like(w)) + s_n * w).T @ G.abs()
    end = lambda x, t: t + R.U["f16"] * (x.abs() + t) + R.TINY["f16"]  # noqa: E731
    return (dq, dk, dv), (end(dq, tq), end(dk, tk), end(dv, tv))


def check(p):
    out, lse = p.forward()
    got = p.backward(out, lse)
    assert status() == 0
    want, tol = gradients(p, out, lse)
    for name, x, w, t in zip(("dq", "dk", "dv"), got, want, tol):
        within(p.heads(x), w, t, name)


SHAPES = [(4, 2, 64), (2, 2, 128), (8, 1, 128)]


@pytest.mark.parametrize("H,Hk,hd", SHAPES)
@pytest.mark.parametrize("lengths", [[300], [40, 1000, 7]])
def test_each_row_of_d_q_keeps_its_bits(H, Hk, hd, lengths):
    # rows of d_out from 1 to 1e-5 of the largest, side by side
    p = Prompt(60, lengths, H, Hk, hd, "f16", before=5, behind=9)
    p.d_out *= (3e3 * 10 ** (-5 * torch.rand(p.rows, 1, device="cuda", generator=gen(61)))).half()
    check(p)


@pytest.mark.parametrize("H,Hk,hd", SHAPES)
@pytest.mark.parametrize("lengths", [[300], [40, 1000, 7]])
def test_each_row_of_d_k_keeps_its_bits(H, Hk, hd, lengths):
    # d_out that falls along the sequences: late keys are seen by small gradients alone
    p = Prompt(62, lengths, H, Hk, hd, "f16", before=5, behind=9)
    for a, b in zip(p.start[:-1], p.start[1:]):
        p.d_out[a:b] *= (3e3 * 10 ** torch.linspace(0, -5, b - a, device="cuda")).half()[:, None]
    check(p)


@pytest.mark.parametrize("rows_of", ["values", "heads"])
def test_values_and_heads_of_very_different_sizes(rows_of):
    p = Prompt(63, [500, 20], 8, 4, 128, "f16")
    if rows_of == "values":  # one key's value far above all before it
        p.v *= 0.01
        p.v[300] *= 1e5
        p.d_out *= 0.3
    else:
        p.heads(p.d_out).mul_((3e3 * 10 ** -torch.linspace(0, 5, 8, device="cuda")).half()[:, None])
    check(p)


@pytest.mark.parametrize("H,Hk,hd", SHAPES)
def test_neighbours_change_no_bit_of_a_sequence(H, Hk, hd):
    p = Prompt(64, [20, 20, 300, 7, 150, 33], H, Hk, hd, "f16", before=3, behind=4)
    sizes = [3e3, 0.01, 1e-2, 2e3, 1.0, 0.02]
    for a, b, s in zip(p.start[:-1], p.start[1:], sizes):
        p.d_out[a:b] *= s
    check(p)
    out, lse = p.forward()
    want = p.backward(out, lse)
    for i in (1, 2, 4, 5):
        a, b = p.start[i], p.start[i + 1]
        d_out, v = p.d_out.clone(), p.v.clone()
        p.d_out *= 16.0
        p.v *= 8.0
        p.d_out[a:b], p.v[a:b] = d_out[a:b], v[a:b]
        o, l = p.forward()  # noqa: E741
        got = p.backward(o, l)
        for x, y in zip(got, want):
            assert torch.equal(x[a:b], y[a:b]), f"sequence {i}"
        p.d_out.copy_(d_out)
        p.v.copy_(v)


def test_the_workspace_holds_what_the_rows_need():
    # any content before, nothing written behind it
    p = Prompt(65, [100, 33], 4, 2, 64, "f16")
    out, lse = p.forward()
    n = V.vla_prompt_attn_grad_workspace_bytes(p.rows, p.H, p.Hk, p.hd)
    ws = torch.full((n + 4096,), 0x7F, dtype=torch.uint8, device="cuda")
    p.backward(out, lse, workspace=ws)
    assert bool((ws[n:] == 0x7F).all())


def test_rows_of_no_sequence_and_other_lengths_by_one_graph():
    # what lies around the sequences is no number; the same captured calls go over other starts
    p = Prompt(66, [70, 201, 0, 33], 6, 2, 64, "f16", before=45, behind=100)
    inside = torch.zeros(p.rows, dtype=torch.bool, device="cuda")
    inside[p.start[0]:p.start[-1]] = True
    want = p.backward(*p.forward())
    for t in (p.q, p.k, p.v, p.d_out):
        t[~inside] = math.nan
    out, lse = p.forward()
    for a, b in zip(p.backward(out, lse), want):
        assert torch.equal(a, b) and bool((a[~inside] == 0).all())
    for t in (p.q, p.k, p.v, p.d_out):
        t[~inside] = 0.5
    ws = torch.empty(V.vla_prompt_attn_grad_workspace_bytes(p.rows, p.H, p.Hk, p.hd), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, l = p.forward()  # noqa: E741
        d = p.backward(o, l, workspace=ws)
    for start in ([0, 449, 449, 449, 449], [3, 40, 300, 301, 420], p.start):
        p.start = start
        p.starts.copy_(torch.tensor(start, dtype=torch.int32))
        graph.replay()
        for a, b in zip(d, p.backward(*p.forward())):
            assert torch.equal(a, b)
    assert status() == 0
