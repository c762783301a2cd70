"""The learning pass over packed sequences (include/vla_learn.h) against plain 64-bit forms, at the lengths, head layouts, strides
and masks where it can go wrong; tolerances in learn_reference.py."""
import math

import pytest
import torch

from paper_2505_18719_gb300 import learn as L
from paper_2505_18719_gb300 import vla as V
from tests import learn_reference as R
from tests.test_gpu_lm_ops import gen, ints, normal, status, within

pytestmark = pytest.mark.gpu

TYPE, CODE, F64 = R.TYPE, R.CODE, R.F64


def stream():
    return torch.cuda.current_stream().cuda_stream


def starts_of(lengths, before=0):
    s = [before]
    for n in lengths:
        s.append(s[-1] + n)
    return s


class Prompt:
    """One packed batch: parts of one q|k|v buffer, or three of their own with gaps between the rows."""

    def __init__(self, seed, lengths, H, Hk, hd, act, before=0, behind=0, apart=False, std=1.0, scale=None):
        g = gen(seed)
        self.start = starts_of(lengths, before)
        self.rows, self.H, self.Hk, self.hd, self.act = self.start[-1] + behind, H, Hk, hd, act
        self.scale = hd ** -0.5 if scale is None else scale
        dt = TYPE[act]
        new = lambda heads, gap: normal(g, self.rows, heads * hd + gap, dtype=dt, std=std)  # noqa: E731
        if apart:
            q, k, v = new(H, 8), new(Hk, 16), new(Hk, 0)
            self.q, self.k, self.v = q[:, :H * hd], k[:, 16:], v
        else:
            x = new(H + 2 * Hk, 0)
            self.q, self.k, self.v = x[:, :H * hd], x[:, H * hd:(H + Hk) * hd], x[:, (H + Hk) * hd:]
        self.d_out = normal(g, self.rows, H * hd, dtype=dt)
        self.starts = ints(self.start)

    def heads(self, t):
        return t.reshape(self.rows, -1, self.hd)

    def forward(self, want_lse=True, **kw):
        out = torch.full((self.rows, self.H * self.hd), 7.0, dtype=TYPE[self.act], device="cuda")
        lse = torch.full((self.rows, self.H), 7.0, device="cuda") if want_lse else None
        rc = V.vla_prompt_attn(self.q.data_ptr(), self.q.stride(0), self.k.data_ptr(), self.k.stride(0), self.v.data_ptr(), self.v.stride(0),
                               CODE[self.act], self.rows, self.H, self.Hk, self.hd, self.starts.data_ptr(), len(self.start) - 1, self.scale,
                               out.data_ptr(), self.H * self.hd, lse.data_ptr() if want_lse else 0, stream())
        assert rc == 0, V.vla_last_error()
        return out, lse

    def backward(self, out, lse, d_out=None, workspace=None):
        d = [torch.full_like(t, 7.0, memory_format=torch.contiguous_format) for t in (self.q, self.k, self.v)]
        d_out = self.d_out if d_out is None else d_out
        n = V.vla_prompt_attn_grad_workspace_bytes(self.rows, self.H, self.Hk, self.hd)
        ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda") if workspace is None else workspace  # (NaN as numbers)
        rc = V.vla_prompt_attn_grad(self.q.data_ptr(), self.q.stride(0), self.k.data_ptr(), self.k.stride(0), self.v.data_ptr(), self.v.stride(0),
                                    CODE[self.act], self.rows, self.H, self.Hk, self.hd, self.starts.data_ptr(), len(self.start) - 1,
                                    self.scale, out.data_ptr(), self.H * self.hd, lse.data_ptr(), d_out.data_ptr(), self.H * self.hd,
                                    d[0].data_ptr(), d[0].stride(0), d[1].data_ptr(), d[1].stride(0), d[2].data_ptr(), d[2].stride(0),
                                    ws.data_ptr(), n, stream())
        assert rc == 0, V.vla_last_error()
        return d

    def check(self, grad=True):
        out, lse = self.forward()
        assert status() == 0
        args = self.heads(self.q), self.heads(self.k), self.heads(self.v), self.start, self.scale
        want, w_lse, t_out, t_lse = R.prompt(*args, self.act)
        within(self.heads(out), want, t_out, "out")
        within(lse, w_lse, t_lse, "lse")
        if not grad:
            return
        # the gradient on its own: from the formula's out and lse, rounded as a call before would have
        out, lse = want.to(out.dtype).reshape(self.rows, -1), w_lse.float()
        got = self.backward(out, lse)
        assert status() == 0
        want, tol = R.prompt_grad(*args, self.heads(out), lse, self.heads(self.d_out), self.act)
        for name, x, w, t in zip(("dq", "dk", "dv"), got, want, tol):
            within(self.heads(x), w, t, name)


HEADS = [(4, 4, 64), (6, 2, 64), (8, 1, 128), (7, 1, 128), (3, 3, 128), (1, 1, 64)]


@pytest.mark.parametrize("act", ["f16", "bf16"])
@pytest.mark.parametrize("H,Hk,hd", HEADS)
def test_prompt_attention_of_short_and_uneven_sequences(H, Hk, hd, act):
    lengths = [1, 0, 2, 15, 16, 17, 0, 0, 63, 64, 65, 127, 128, 129, 1, 255, 256, 257, 300, 0]
    Prompt(1, lengths, H, Hk, hd, act).check()


@pytest.mark.parametrize("act", ["f16", "bf16"])
@pytest.mark.parametrize("n", [1, 2, 5, 31, 80, 128, 130, 384, 511, 640, 1023, 1500])
def test_prompt_attention_of_one_sequence(n, act):
    Prompt(n, [n], 4, 2, 128, act).check()
    Prompt(n, [n], 3, 1, 64, act, before=3, behind=5, apart=True).check()


@pytest.mark.parametrize("H,Hk,hd", [(28, 4, 128), (12, 12, 128), (16, 4, 64)])
def test_prompt_attention_rows_of_no_sequence_are_zeros(H, Hk, hd):
    p = Prompt(3, [70, 201, 0, 33], H, Hk, hd, "bf16", before=140, behind=300)
    inside = torch.zeros(p.rows, dtype=torch.bool, device="cuda")
    inside[p.start[0]:p.start[-1]] = True
    want = p.forward()
    grad = p.backward(*want)
    for t in (p.q, p.k, p.v, p.d_out):
        t[~inside] = math.nan
    p.check()
    out, lse = p.forward()
    assert bool((out[~inside] == 0).all()) and bool((lse[~inside] == -math.inf).all())
    got = p.backward(out, lse)
    for a, b in zip((out, lse, *got), (*want, *grad)):  # what lies around the sequences changes nothing in them
        assert torch.equal(a, b)
        assert a is lse or bool((a[~inside] == 0).all())


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("what", ["q", "k", "v"])
@pytest.mark.parametrize("act,hd", [("f16", 64), ("bf16", 128)])
def test_prompt_attention_bad_rows_reach_no_row_before_them(bad, what, act, hd):
    p = Prompt(5, [40, 333, 150], 4, 2, hd, act)
    want, w_lse = p.forward()
    at = p.start[1] + 200
    getattr(p, what)[at, 3::7] = bad
    out, lse = p.forward()
    other = [i for i in range(p.rows) if not at <= i < p.start[2]]
    if what == "q":
        other = [i for i in range(p.rows) if i != at]
    # (a row that a bad value of another row spoilt may have been computed again, by other sums)
    _, _, tol, t_lse = R.prompt(*[torch.where(torch.isfinite(t), t, 0) for t in map(p.heads, (p.q, p.k, p.v))], p.start, p.scale, act)
    within(p.heads(out)[other], p.heads(want)[other], 2 * tol[other], "out")
    within(lse[other], w_lse[other], 2 * t_lse[other], "lse")
    if what != "q" and bad != -math.inf:  # the rows that see it show it (a key of -inf may count as weight 0)
        assert not bool(torch.isfinite(p.heads(out)[at:p.start[2]]).all())


@pytest.mark.parametrize("act,hd", [("f16", 64), ("bf16", 128)])
def test_prompt_gradient_bad_rows_stay_in_their_sequence(act, hd):
    p = Prompt(6, [140, 333, 150], 4, 2, hd, act, behind=9)
    out, lse = p.forward()
    want = p.backward(out, lse)
    lo, hi = p.start[1], p.start[2]
    for t in (p.q, p.k, p.v, p.d_out, out, lse):
        t[lo + 1:hi] = math.nan
    got = p.backward(out, lse)
    for a, b in zip(got, want):
        assert torch.equal(a[:lo], b[:lo]) and torch.equal(a[hi:], b[hi:])


@pytest.mark.parametrize("act", ["f16", "bf16"])
@pytest.mark.parametrize("std,scale", [(6.0, None), (1.0, 3.0), (0.01, None), (1.0, 1e-6), (12.0, 1.0)])
def test_prompt_attention_of_large_and_small_scores(act, std, scale):
    Prompt(8, [200, 77], 4, 2, 64, act, std=std, scale=scale).check()


@pytest.mark.parametrize("size", [1e-5, 1e-3, 300.0, 3000.0])
def test_prompt_gradient_of_fp16_of_any_size(size):
    p = Prompt(9, [260, 30], 4, 1, 128, "f16")
    p.d_out *= size
    p.check()


def test_prompt_attention_rows_that_grow():
    # maxima that move far at every key: references of the running softmax follow
    p = Prompt(10, [900], 2, 2, 64, "bf16")
    p.k[:] = p.q[-1] * torch.linspace(-30, 30, p.rows, device="cuda", dtype=torch.bfloat16)[:, None]
    p.q[:] = p.q[-1]
    p.check()
    p.k[:] = p.k.flip(0)
    p.check()


@pytest.mark.parametrize("H,Hk,hd", [(8, 8, 128), (8, 2, 64)])
def test_prompt_attention_of_many_sequences(H, Hk, hd):
    g = torch.Generator().manual_seed(4)
    Prompt(11, torch.randint(0, 9, (700,), generator=g).tolist(), H, Hk, hd, "bf16").check()


def test_prompt_attention_equal_calls_give_equal_bits_and_graphs_replay():
    p = Prompt(12, [300, 5, 644, 129], 8, 2, 128, "bf16", behind=3)
    out, lse = p.forward()
    d = p.backward(out, lse)
    ws = torch.empty(V.vla_prompt_attn_grad_workspace_bytes(p.rows, p.H, p.Hk, p.hd), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o2, l2 = p.forward()
        d2 = p.backward(o2, l2, workspace=ws)
    for _ in range(5):
        for t in (o2, l2, *d2):
            t.fill_(3.0)
        graph.replay()
        for a, b in zip((o2, l2, *d2), (out, lse, *d)):
            assert torch.equal(a, b)
    # other lengths in the same rows, by the same graph
    p.start = starts_of([0, 700, 1, 377])
    p.starts.copy_(ints(p.start))
    graph.replay()
    want = p.forward()
    for a, b in zip((o2, l2, *d2), (*want, *p.backward(*want))):
        assert torch.equal(a, b)


def test_prompt_attention_on_two_streams():
    ps = [Prompt(20 + i, [257, 300 + i, 64], 8, 4, 128, "f16") for i in range(2)]
    want = []
    for p in ps:
        out = p.forward()
        want.append((*out, *p.backward(*out)))
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in ps], [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                out = ps[i].forward()
                got[i].append((*out, *ps[i].backward(*out)))
    torch.cuda.synchronize()
    for i in range(2):
        for one in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(one, want[i]))


@pytest.mark.parametrize("starts", [[0, 50, 40, 90], [-3, 50, 90], [0, 50, 91], [0, 1 << 30], [10, -5, 90]])
def test_prompt_attention_bad_starts_are_reported(starts):
    p = Prompt(13, [90], 2, 2, 64, "f16")
    out, lse = p.forward()
    p.start, p.starts = starts, ints(starts)
    guard = torch.full((64, p.H * p.hd), 5.0, dtype=torch.float16, device="cuda")
    p.forward()
    assert status() == V.VLA_STATUS_SEQUENCES
    p.backward(out, lse)
    assert status() == V.VLA_STATUS_SEQUENCES
    assert bool((guard == 5).all())


@pytest.mark.parametrize("act,hd", [("f16", 64), ("bf16", 128)])
def test_prompt_gradient_is_the_functions_slope(act, hd):
    # along a random direction of all inputs, against central differences in 64 bits
    p = Prompt(14, [9, 140], 4, 2, hd, act)
    x = [p.heads(t).to(F64) for t in (p.q, p.k, p.v)]
    g = gen(15)
    direction = [normal(g, *t.shape).to(F64) for t in x]
    weight = p.heads(p.d_out).to(F64)

    def value(step):
        return float((R.prompt(*[a + step * b for a, b in zip(x, direction)], p.start, p.scale, act)[0] * weight).sum())

    out, lse, _, _ = R.prompt(*x, p.start, p.scale, act)
    got = p.backward(out.to(TYPE[act]).reshape(p.rows, -1), lse.float())
    _, tol = R.prompt_grad(*x, p.start, p.scale, out, lse, weight, act)
    slope = (value(1e-4) - value(-1e-4)) / 2e-4
    along = sum(float((p.heads(a).to(F64) * b).sum()) for a, b in zip(got, direction))
    # out itself was rounded before D was taken from it: U of each product, times the weights' share of the direction
    K, Q = x[1].repeat_interleave(2, 1), x[0]
    slack = 2 * R.U[act] * float((weight * out).abs().sum(-1).max() * p.scale * (Q.norm() * direction[1].norm() + K.norm() * direction[0].norm()))
    assert abs(along - slope) <= sum(float((t * b.abs()).sum()) for t, b in zip(tol, direction)) + slack + 1e-6 * abs(slope)


def test_prompt_attention_function_and_its_gradients():
    g = gen(30)
    rows, H, Hk, hd = 333, 6, 2, 64
    start = ints([0, 100, 100, 320])
    x = normal(g, rows, (H + 2 * Hk) * hd, dtype=torch.bfloat16).requires_grad_()
    q, k, v = x.split([H * hd, Hk * hd, Hk * hd], -1)
    out, lse = L.prompt_attention(q, k, v, start, hd, want_lse=True)
    assert out.shape == (rows, H, hd) and not lse.requires_grad
    w = normal(g, rows, H, hd, dtype=torch.bfloat16)
    (out.transpose(0, 1) * w.transpose(0, 1)).sum().backward()  # (a gradient of other strides)
    views = [t.detach().view(rows, -1, hd) for t in (q, k, v)]
    want, tol = R.prompt_grad(*views, start.tolist(), hd ** -0.5, out.detach(), lse, w, "bf16")
    within(x.grad, torch.cat([t.flatten(1) for t in want], -1), torch.cat([t.flatten(1) for t in tol], -1), "d_qkv")
    L.check()
    # without rows; heads as their own dimension
    e = lambda n: torch.empty(0, n, hd, dtype=torch.float16, device="cuda", requires_grad=True)  # noqa: E731
    leaves = e(4), e(2), e(2)
    L.prompt_attention(*leaves, ints([0, 0]), hd).sum().backward()
    assert all(t.grad.shape == t.shape for t in leaves)


def test_prompt_attention_function_refusals():
    g = gen(31)
    q, k = normal(g, 10, 128, dtype=torch.float16), normal(g, 10, 64, dtype=torch.float16)
    start = ints([0, 10])
    with pytest.raises(ValueError):
        L.prompt_attention(q, k.bfloat16(), k, start, 64)
    with pytest.raises(ValueError):
        L.prompt_attention(q, k[:9], k, start, 64)
    with pytest.raises(ValueError):
        L.prompt_attention(q, k, k, start.long(), 64)
    with pytest.raises(ValueError):
        L.prompt_attention(q, k, k, start.cpu(), 64)
    with pytest.raises(ValueError):
        L.prompt_attention(q.cpu(), k.cpu(), k.cpu(), start, 64)
    with pytest.raises(ValueError):
        L.prompt_attention(q.t().contiguous().t(), k, k, start, 64)
    with pytest.raises(V.VlaError):
        L.prompt_attention(q.float(), k.float(), k.float(), start, 64)
    with pytest.raises(V.VlaError):
        L.prompt_attention(q, k, k, start, 32)
    with pytest.raises(V.VlaError):
        L.prompt_attention(q, k, k, start, 64, scale=-1.0)


# ------------------------------------------------------------------------------------------- block norm
class Norm:
    def __init__(self, seed, rows, dim, act, stream_type, post, gate, scale=0.5, first=False, gap=0):
        g = gen(seed)
        self.rows, self.dim, self.act, self.stream, self.scale, self.eps = rows, dim, act, stream_type, scale, 1e-6
        part = lambda dtype, std=1.0: normal(g, rows, dim + gap, dtype=dtype, std=std)[:, gap // 2:gap // 2 + dim]  # noqa: E731
        gain = lambda: (1 + 0.3 * normal(g, dim)).to(torch.bfloat16)  # noqa: E731
        self.y = None if first else part(TYPE[act], 0.7)
        self.h, self.pre = part(TYPE[stream_type], 2.0), gain()
        self.post = gain() if post else None
        self.gate = None if gate == "none" else normal(g, dim, dtype=TYPE[act], std=0.5) if gate == "channel" else part(TYPE[act], 0.5)
        self.d_x, self.d_h_out = part(TYPE[act]), part(TYPE[stream_type])
        self.new = lambda dtype: torch.full((rows, dim + gap), 7.0, dtype=dtype, device="cuda")[:, gap // 2:gap // 2 + dim]

    def ptr(self, t):
        return 0 if t is None else t.data_ptr()

    def ld(self, t):
        return 0 if t is None or t.dim() == 1 else t.stride(0)

    def forward(self, in_place=False):
        h = self.h.clone() if in_place else self.h
        h_out = None if self.y is None else h if in_place else self.new(TYPE[self.stream])
        x, rstd = self.new(TYPE[self.act]), torch.empty(self.rows, 2, device="cuda")
        rc = V.vla_block_norm(self.ptr(self.y), self.ld(self.y), CODE[self.act], h.data_ptr(), h.stride(0), CODE[self.stream], self.rows, self.dim,
                              self.ptr(self.post), self.ptr(self.gate), self.ld(self.gate), self.scale, self.pre.data_ptr(), self.eps,
                              self.ptr(h_out), self.ld(h_out), x.data_ptr(), x.stride(0), rstd.data_ptr(), stream())
        assert rc == 0, V.vla_last_error()
        return h_out, x, rstd

    def backward(self, h, rstd, with_h_out=True, in_place=False):
        f = lambda: torch.full((self.dim,), 7.0, device="cuda")  # noqa: E731
        d_in = self.d_h_out.clone() if in_place else self.d_h_out
        out = {"d_h": d_in if in_place else self.new(TYPE[self.stream]), "d_pre_gain": f()}
        if self.y is not None:
            out["d_y"] = self.new(TYPE[self.act])
        if self.post is not None:
            out["d_post_gain"] = f()
        if self.gate is not None:
            out["d_gate"] = f() if self.gate.dim() == 1 else self.new(TYPE[self.act])
        n = V.vla_block_norm_grad_workspace_bytes(self.rows, self.dim)
        ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
        at = lambda k: self.ptr(out.get(k))  # noqa: E731
        rc = V.vla_block_norm_grad(self.ptr(self.y), self.ld(self.y), CODE[self.act], h.data_ptr(), h.stride(0), CODE[self.stream], self.rows,
                                   self.dim, self.ptr(self.post), self.ptr(self.gate), self.ld(self.gate), self.scale, self.pre.data_ptr(),
                                   rstd.data_ptr(), self.d_x.data_ptr(), self.d_x.stride(0), d_in.data_ptr() if with_h_out else 0, d_in.stride(0),
                                   at("d_h"), out["d_h"].stride(0), at("d_y"), self.ld(out.get("d_y")), at("d_gate"),
                                   self.ld(out.get("d_gate")), at("d_post_gain"), at("d_pre_gain"), ws.data_ptr(), n, stream())
        assert rc == 0, V.vla_last_error()
        return out

    def check(self, **kw):
        h_out, x, rstd = self.forward()
        w_h, w_x, t_h, t_x = R.block_norm(self.y, self.h, self.pre, self.post, self.gate, self.scale, self.eps, self.act, self.stream)
        if self.y is not None:
            within(h_out, w_h, t_h, "h_out")
        within(x, w_x, t_x, "x")
        h = self.h if self.y is None else w_h.to(TYPE[self.stream])
        want, tol = R.block_norm_grad(self.y, h, self.pre, self.post, self.gate, self.scale, rstd, self.d_x,
                                      self.d_h_out if kw.get("with_h_out", True) else None, self.act, self.stream)
        got = self.backward(h, rstd, **kw)
        assert got.keys() == want.keys()
        for k in want:
            within(got[k], want[k], tol[k], k)


TYPES = [("f16", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "f32")]


@pytest.mark.parametrize("act,stream_type", TYPES)
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("gate", ["none", "channel", "row"])
def test_block_norm_forms(act, stream_type, post, gate):
    for rows, dim in ((37, 1155), (5, 1152), (1, 64), (3, 4096)):
        Norm(dim, rows, dim, act, stream_type, post, gate).check()


@pytest.mark.parametrize("rows,dim", [(1, 1), (2, 7), (700, 31), (9, 63), (33, 255), (40, 256), (11, 2047), (11, 2048), (11, 2056), (12, 4097),
                                      (6, 8191), (6, 8192), (4, 8200), (3, 12345), (3, 16384), (1500, 96), (611, 2560)])
def test_block_norm_sizes(rows, dim):
    Norm(dim, rows, dim, "bf16", "f32", True, "channel").check()
    Norm(dim + 1, rows, dim, "bf16", "bf16", True, "row", scale=-0.7).check(with_h_out=False)
    Norm(dim + 2, rows, dim, "f16", "f32", False, "none").check(in_place=True)
    Norm(dim + 3, rows, dim, "f16", "f32", False, "none", first=True).check()


@pytest.mark.parametrize("gap", [1, 2, 8, 16, 24])
def test_block_norm_rows_apart(gap):
    Norm(gap, 21, 520, "bf16", "f32", True, "row", gap=gap).check()
    Norm(gap, 21, 520, "f16", "f16", True, "channel", gap=gap).check(with_h_out=False)


def test_block_norm_in_place_and_equal_bits():
    n = Norm(3, 50, 1024, "bf16", "f32", True, "row")
    h, x, rstd = n.forward()
    h2, x2, rstd2 = n.forward(in_place=True)
    assert torch.equal(h, h2) and torch.equal(x, x2) and torch.equal(rstd, rstd2)
    want = n.backward(h, rstd)
    for _ in range(3):
        got = n.backward(h, rstd, in_place=True)
        assert all(torch.equal(got[k], want[k]) for k in want)


def test_block_norm_bad_rows_stay_where_they_are():
    n = Norm(4, 40, 513, "bf16", "f32", True, "none")
    h, x, rstd = n.forward()
    want = n.backward(h, rstd)
    n.y[7, 5], n.h[9, 0] = math.nan, math.inf
    h2, x2, rstd2 = n.forward()
    keep = [i for i in range(40) if i not in (7, 9)]
    assert torch.equal(h2[keep], h[keep]) and torch.equal(x2[keep], x[keep]) and bool(torch.isnan(x2[7]).all())
    got = n.backward(h2, rstd2)
    assert torch.equal(got["d_h"][keep], want["d_h"][keep]) and torch.equal(got["d_y"][keep], want["d_y"][keep])


def test_block_norm_captured_and_replayed():
    n = Norm(5, 600, 2000, "bf16", "f32", True, "channel")
    h, x, rstd = n.forward()
    want = n.backward(h, rstd)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h2, x2, rstd2 = n.forward()
        got = n.backward(h2, rstd2)
    for _ in range(3):
        for t in (h2, x2, rstd2, *got.values()):
            t.fill_(9.0)
        graph.replay()
        assert torch.equal(h2, h) and torch.equal(x2, x) and all(torch.equal(got[k], want[k]) for k in want)


def test_block_norm_gradient_is_the_functions_slope():
    g = gen(16)
    n = Norm(16, 8, 192, "f32", "f32", True, "row")
    x = [t.to(F64) for t in (n.y, n.h, n.gate)]
    pre, post = n.pre.to(F64), n.post.to(F64)
    d = [normal(g, *t.shape).to(F64) for t in (*x, pre, post)]

    def value(step):
        y, h, gate, w, v = [a + step * b for a, b in zip((*x, pre, post), d)]
        h_out, x_out, _, _ = R.block_norm(y, h, w, v, gate, n.scale, n.eps, "f32", "f32")
        return float((h_out * n.d_h_out.to(F64) + x_out * n.d_x.to(F64)).sum())

    h_out, _, rstd = n.forward()
    got = n.backward(h_out, rstd)
    slope = (value(1e-5) - value(-1e-5)) / 2e-5
    terms = [got[k].to(F64) * b for k, b in zip(("d_y", "d_h", "d_gate", "d_pre_gain", "d_post_gain"), d)]
    size = sum(float(t.abs().sum()) for t in terms)
    # 32-bit gradients of rows of 192 (about 64 roundings each, of sizes that cancel by less than 16), and the differences' own error
    assert abs(sum(float(t.sum()) for t in terms) - slope) <= 1024 * R.E * size + 1e-7 * size


def test_block_norm_functions_and_their_gradients():
    g = gen(32)
    rows, dim = 45, 264
    leaf = lambda t: t.requires_grad_()  # noqa: E731
    h, y = leaf(normal(g, rows, dim)), leaf(normal(g, rows, dim, dtype=torch.float16))
    pre, post = leaf((1 + 0.2 * normal(g, dim)).bfloat16()), leaf((1 + 0.2 * normal(g, dim)).bfloat16())
    gate = leaf(normal(g, dim, dtype=torch.float16))
    x, h_out = L.block_norm(y, h, pre, post, gate, residual_scale=0.3)
    wx, wh = normal(g, rows, dim, dtype=torch.float16), normal(g, rows, dim)
    ((x * wx).float().sum() + (h_out * wh).sum()).backward()
    with torch.no_grad():
        rstd = torch.stack([torch.rsqrt(t.double().square().mean(-1) + 1e-6).float() for t in (y, h_out)], -1)
        want, tol = R.block_norm_grad(y, h_out, pre, post, gate, 0.3, rstd, wx, wh, "f16", "f32")
    for name, t in (("d_y", y), ("d_h", h), ("d_pre_gain", pre), ("d_post_gain", post), ("d_gate", gate)):
        u = {torch.float32: 0.0, torch.float16: R.U["f16"], torch.bfloat16: R.U["bf16"]}[t.dtype]
        # rstd was rounded apart from the kernel's: 16 more 32-bit roundings of it, and of what it was taken times
        within(t.grad, want[name], 2 * tol[name] + 1.01 * u * want[name].abs() + 64 * R.E * want[name].abs(), name)
    # only one of the two results used
    for pick in (0, 1):
        a, b = leaf(normal(g, 3, 8)), leaf(normal(g, 3, 8))
        one = torch.ones(8, dtype=torch.bfloat16, device="cuda")
        L.block_norm(a, b, one)[pick].sum().backward()
        assert bool(torch.isfinite(a.grad).all()) and bool(torch.isfinite(b.grad).all())
        assert pick == 0 or (torch.equal(a.grad, torch.ones_like(a)) and torch.equal(b.grad, torch.ones_like(b)))
    s = leaf(normal(g, rows, dim))
    z = L.first_norm(s, pre.detach(), dtype=torch.bfloat16)
    assert z.dtype == torch.bfloat16
    z.float().sum().backward()
    assert bool(torch.isfinite(s.grad).all())
    # no rows: gains get zeros
    w = leaf(torch.ones(8, dtype=torch.bfloat16, device="cuda"))
    L.first_norm(torch.empty(0, 8, device="cuda"), w).sum().backward()
    assert bool((w.grad == 0).all())


def test_block_norm_function_refusals():
    g = gen(33)
    h, y, gain = normal(g, 4, 16), normal(g, 4, 16, dtype=torch.float16), torch.ones(16, dtype=torch.bfloat16, device="cuda")
    for call in (lambda: L.block_norm(None, h, gain), lambda: L.block_norm(y, h, gain.float()), lambda: L.block_norm(y, h, gain[:8]),
                 lambda: L.block_norm(y[:3], h, gain), lambda: L.block_norm(y, h, gain, gate=gain), lambda: L.block_norm(y, h, gain, gate=y[0, :8]),
                 lambda: L.block_norm(y.cpu(), h, gain), lambda: L.block_norm(y, h, gain.cpu()), lambda: L.block_norm(y.t(), h.t(), gain[:4]),
                 lambda: L.block_norm(y.double(), h, gain)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(V.VlaError):
        L.block_norm(y, h.bfloat16(), gain)
    with pytest.raises(V.VlaError):
        L.block_norm(y, h, gain, eps=-1.0)


def test_a_layer_of_both():
    # first norm, projections, attention, block norm with its gain and gate, and back: every leaf against 64-bit autograd
    g = gen(40)
    rows, d, H, Hk, hd = 150, 256, 4, 2, 64
    start = ints([0, 61, 150])
    leaf = lambda *s, std=1.0: normal(g, *s, std=std).bfloat16().requires_grad_()  # noqa: E731
    h = normal(g, rows, d).requires_grad_()
    w_qkv, w_o = leaf((H + 2 * Hk) * hd, d, std=d ** -0.5), leaf(d, H * hd, std=(H * hd) ** -0.5)
    gains = [(1 + 0.2 * normal(g, d)).bfloat16().requires_grad_() for _ in range(3)]
    wx, wh = normal(g, rows, d), normal(g, rows, d)
    x = L.first_norm(h, gains[0], dtype=torch.bfloat16)
    q, k, v = (x @ w_qkv.t()).split([H * hd, Hk * hd, Hk * hd], -1)
    y = L.prompt_attention(q, k, v, start, hd).flatten(1) @ w_o.t()
    z, h_out = L.block_norm(y, h, gains[1], gains[2], residual_scale=0.7)
    leaves = [h, w_qkv, w_o, *gains]
    got = torch.autograd.grad((z.float() * wx).sum() + (h_out * wh).sum(), leaves)
    copies = [t.detach().to(F64).requires_grad_() for t in leaves]
    h6, qkv6, o6, g0, g1, g2 = copies
    norm = lambda t, w: t / (t.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt() * w  # noqa: E731
    q6, k6, v6 = [t.view(rows, -1, hd) for t in (norm(h6, g0) @ qkv6.t()).split([H * hd, Hk * hd, Hk * hd], -1)]
    parts = []
    for a, b in ((0, 61), (61, 150)):
        s = torch.einsum("nhd,mhd->hnm", q6[a:b], k6[a:b].repeat_interleave(2, 1)) * hd ** -0.5
        s = s.masked_fill(torch.ones(b - a, b - a, dtype=torch.bool, device="cuda").triu(1), -math.inf)
        parts.append(torch.einsum("hnm,mhd->nhd", torch.softmax(s, -1), v6[a:b].repeat_interleave(2, 1)))
    y6 = torch.cat(parts).flatten(1) @ o6.t()
    out6 = h6 + 0.7 * norm(y6, g2)
    want = torch.autograd.grad((norm(out6, g1) * wx).sum() + (out6 * wh).sum(), copies)
    # at most about 24 bf16 roundings lie on any path from a leaf to the sum, of random sign: 8 half-steps of the whole
    for a, b in zip(got, want):
        assert float((a.to(F64) - b).norm()) <= 8 * R.U["bf16"] * float(b.norm())
