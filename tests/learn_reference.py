"""The learning pass's operators (include/vla_learn.h) in 64 bits, straight from their formulas, and how far 32-bit sums of
16-bit products may be from them.

`U` is the half-step of a type's own rounding, `E` = 2^-24 that of a 32-bit operation.  A product on the tensor cores may be cut
(not rounded) at 2^-23 of the running sum for every 16 terms, so a sum of n products is off by at most (n / 16 + 8) 2^-23 times the sum
of their sizes."""
import math

import torch

F64 = torch.float64
TYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
CODE = {"f32": 0, "f16": 1, "bf16": 2}
U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -126, "f16": 2.0 ** -25, "bf16": 2.0 ** -126}  # half the spacing of the smallest numbers
E = 2.0 ** -24


def sum_error(n):
    return (n / 16.0 + 8.0) * 2.0 * E


def _mask(n, device):
    return torch.ones(n, n, dtype=torch.bool, device=device).tril()


def prompt(q, k, v, start, scale, act):
    """q [rows, H, hd], k and v [rows, Hk, hd]; start: a list.  (out, lse, tolerance of out, tolerance of lse)."""
    rows, H, hd = q.shape
    group = H // k.shape[1]
    dev = q.device
    out, t_out = torch.zeros(rows, H, hd, dtype=F64, device=dev), torch.zeros(rows, H, hd, dtype=F64, device=dev)
    lse, t_lse = torch.full((rows, H), -math.inf, dtype=F64, device=dev), torch.zeros(rows, H, dtype=F64, device=dev)
    for a, b in zip(start[:-1], start[1:]):
        n = b - a
        for h in range(H if n else 0):
            Q, K, W = q[a:b, h].to(F64), k[a:b, h // group].to(F64), v[a:b, h // group].to(F64)
            seen = _mask(n, dev)
            s = torch.where(seen, scale * Q @ K.T, -math.inf)
            # a score: its products, its scale and the difference from the row's reference, in steps of its size
            e_s = scale * (Q.abs() @ K.abs().T) * (sum_error(hd) + 4 * E)
            e_s = torch.where(seen, e_s, 0.0).amax(-1, keepdim=True) + 4 * E
            top = s.amax(-1, keepdim=True)
            w = torch.exp(s - top)
            total = w.sum(-1, keepdim=True)
            p = w / total
            out[a:b, h] = p @ W
            lse[a:b, h] = (top + torch.log(total)).squeeze(-1)
            # each weight: its score twice (in the sum too), the exponential, its rounding; then the sums and the result's rounding
            size = p @ W.abs()
            t_out[a:b, h] = U[act] * out[a:b, h].abs() + (1.01 * U[act] + 2 * e_s + sum_error(n) + 8 * E) * size + TINY[act] * (
                1 + torch.where(seen, 1.0, 0.0).to(F64) @ W.abs())
            t_lse[a:b, h] = (e_s.squeeze(-1) + (8 + n ** 0.5) * E + 4 * E * lse[a:b, h].abs())
    return out, lse, t_out, t_lse


def prompt_grad(q, k, v, start, scale, out, lse, d_out, act):
    """Gradients from the given out and lse, and their tolerances."""
    rows, H, hd = q.shape
    Hk = k.shape[1]
    group = H // Hk
    dev = q.device
    z = lambda n: torch.zeros(rows, n, hd, dtype=F64, device=dev)  # noqa: E731
    dq, tq, dk, tk, dv, tv = z(H), z(H), z(Hk), z(Hk), z(Hk), z(Hk)
    u = 1.01 * U[act]
    finite = lambda t: torch.where(torch.isfinite(t), t, 0).to(F64)  # noqa: E731
    most = finite(d_out).norm(dim=-1).max() * finite(v).norm(dim=-1).max()
    for a, b in zip(start[:-1], start[1:]):
        n = b - a
        if not n:
            continue
        seen = _mask(n, dev)
        for h in range(H):
            g = h // group
            Q, K, W = q[a:b, h].to(F64), k[a:b, g].to(F64), v[a:b, g].to(F64)
            G, O, L = d_out[a:b, h].to(F64), out[a:b, h].to(F64), lse[a:b, h].to(F64)[:, None]  # noqa: E741
            p = torch.where(seen, torch.exp(torch.where(seen, scale * Q @ K.T - L, 0.0)), 0.0)
            # a weight's relative error: its score's, that of lse in units of log 2, the exponential
            e_p = torch.where(seen, scale * (Q.abs() @ K.abs().T) * (sum_error(hd) + 4 * E), 0.0) + 4 * E * L.abs() + 8 * E
            delta = (G * O).sum(-1, keepdim=True)
            dp = G @ W.T
            e_d = (G.abs() @ W.abs().T + (G * O).abs().sum(-1, keepdim=True)) * sum_error(hd)
            ds = p * (dp - delta)
            e_ds = (u + e_p) * ds.abs() + p * e_d
            if act == "f16":  # dS counts relative to the largest that it can be (38 bits below), P to 1 (14 bits of scale)
                e_ds = e_ds + torch.where(seen, most * 2.0 ** -38, 0.0)
                floor = torch.where(seen, 2.0 ** -38, 0.0).to(F64)
            else:  # a weight below the smallest normal number, 2^-126, may count as 0: its terms are lost whole
                floor = torch.where(seen, 2.0 ** -126, 0.0).to(F64)
                e_ds = e_ds + floor * (dp.abs() + delta.abs())
            e_w = (u + e_p) * p + floor
            s_n = sum_error(n * group)
            dq[a:b, h] = scale * ds @ K
            tq[a:b, h] = scale * (e_ds + s_n * ds.abs()) @ K.abs()
            dk[a:b, g] += scale * ds.T @ Q
            tk[a:b, g] += scale * (e_ds + s_n * ds.abs()).T @ Q.abs()
            dv[a:b, g] += p.T @ G
            tv[a:b, g] += (e_w + s_n * p).T @ G.abs()
    end = lambda x, t: t + U[act] * (x.abs() + t) + TINY[act]  # noqa: E731
    return (dq, dk, dv), (end(dq, tq), end(dk, tk), end(dv, tv))


def block_norm(y, h, pre, post, gate, scale, eps, act, stream):
    """(h_out, x, tolerances): 32-bit arithmetic with one rounding; e counts the roundings of a factor."""
    Y, Hh = (None if y is None else y.to(F64)), h.to(F64)
    dim = h.shape[1]
    e_r = (8 + dim ** 0.5) * E  # a mean of squares under the root, its root, products
    if Y is None:
        h_out, t_h = Hh, torch.zeros_like(Hh)
    else:
        u, e_u = Y, 0.0
        if post is not None:
            u, e_u = Y / (Y.pow(2).mean(-1, keepdim=True) + eps).sqrt() * post.to(F64), e_r
        if gate is not None:
            u = u * gate.to(F64)
        h_out = Hh + scale * u
        t_h = (e_u + 4 * E) * (scale * u).abs() + 2 * E * h_out.abs()
    r = 1 / (h_out.pow(2).mean(-1, keepdim=True) + eps).sqrt()
    x = h_out * r * pre.to(F64)
    e_mean = t_h.pow(2).mean(-1, keepdim=True).sqrt() * r  # what the stream's own errors do to the root, relative
    t_x = (t_h * r * pre.to(F64).abs()) + x.abs() * (e_r + e_mean) + U[act] * x.abs() * 1.01 + TINY[act]
    return h_out, x, t_h + U[stream] * h_out.abs() + TINY[stream], t_x


def block_norm_grad(y, h, pre, post, gate, scale, rstd, d_x, d_h_out, act, stream):
    """Gradients at the stream h behind the sum from the given rstd, by name, with their tolerances."""
    n_rows, dim = h.shape
    Hh, X = h.to(F64), d_x.to(F64)
    r_y, r_h = rstd[:, :1].to(F64), rstd[:, 1:].to(F64)
    W = pre.to(F64)
    mean = lambda t: t.mean(-1, keepdim=True)  # noqa: E731
    n, g = Hh * r_h, X * W
    e_m = (8 + dim ** 0.5) * E
    c1, t_c1 = mean(g * n), mean((g * n).abs()) * e_m
    D = torch.zeros_like(Hh) if d_h_out is None else d_h_out.to(F64)
    d_h = D + r_h * (g - n * c1)
    size = D.abs() + r_h * (g.abs() + n.abs() * c1.abs())
    t_h = 6 * E * size + r_h * n.abs() * t_c1
    col = lambda t, e: (t.sum(0), ((8 + n_rows ** 0.5) * E * t.abs() + e).sum(0) + TINY["f32"])  # noqa: E731
    res, tol = {"d_h": d_h}, {"d_h": t_h + U[stream] * d_h.abs() + TINY[stream]}
    res["d_pre_gain"], tol["d_pre_gain"] = col(X * n, 0.0)
    if y is None:
        return res, tol
    Y = y.to(F64)
    m = Y * r_y if post is not None else Y
    u = m * post.to(F64) if post is not None else Y
    d_u, t_u = scale * d_h, abs(scale) * t_h + 2 * E * (scale * d_h).abs()
    if gate is not None:
        t = d_u * u
        e = t_u * u.abs() + 4 * E * t.abs()
        if gate.dim() == 2:
            res["d_gate"], tol["d_gate"] = t, e + U[act] * t.abs() + TINY[act]
        else:
            res["d_gate"], tol["d_gate"] = col(t, e)
        d_u, t_u = d_u * gate.to(F64), t_u * gate.to(F64).abs() + 2 * E * (d_u * gate.to(F64)).abs()
    if post is not None:
        P = post.to(F64)
        t = d_u * m
        res["d_post_gain"], tol["d_post_gain"] = col(t, t_u * m.abs() + 4 * E * t.abs())
        d_m = d_u * P
        c2 = mean(d_m * m)
        # c2 comes from sums over q (d_h_out + r_h g) and q r_h n, taken together
        q = (scale * P * m if gate is None else scale * P * m * gate.to(F64)).abs()
        t_c2 = (mean(q * (D.abs() + r_h * g.abs())) + c1.abs() * mean(q * r_h * n.abs())) * 2 * e_m + t_c1 * mean(q * r_h * n.abs())
        t_u = r_y * (t_u * P.abs() + 4 * E * d_m.abs() + m.abs() * (t_c2 + 4 * E * c2.abs()))
        d_u = r_y * (d_m - m * c2)
    res["d_y"], tol["d_y"] = d_u, t_u + (U[act] + 4 * E) * d_u.abs() + TINY[act]
    return res, tol
