"""The paged cache's operators and the token log-probs (include/vla_lm.h) against plain 64-bit forms, at the
sizes, lengths and masks where they can go wrong.

Tolerances follow from the number formats: `U` is the half-ulp of a type's own rounding, 2^-24 that of every
32-bit operation; a sum of n terms is allowed 4 sqrt(n) of them (rounding errors of random sign) and, on the
tensor cores, one truncation of 2^-23 per 16 terms."""
import math

import pytest
import torch

from paper_2505_18719_gb300 import vla as V

pytestmark = pytest.mark.gpu

F64 = torch.float64
TYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
CODE = {"f32": V.VLA_F32, "f16": V.VLA_F16, "bf16": V.VLA_BF16}
U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 0.0, "f16": 2.0 ** -25, "bf16": 0.0}  # half the spacing of the smallest numbers
E = 2.0 ** -24


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def status():
    rc, bits = V.vla_op_read_status(torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    return bits


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape, dtype=torch.float32, std=1.0):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def within(got, want, tol, what=""):
    got, want = got.detach().cpu().to(F64), want.detach().cpu().to(F64)
    tol = tol.detach().cpu() if torch.is_tensor(tol) else torch.full_like(want, tol)
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    ok = same | ((got - want).abs() <= tol)
    if not bool(ok.all()):
        i = int((~ok).reshape(-1).nonzero()[0])
        raise AssertionError(f"{what}: {int((~ok).sum())} of {ok.numel()} off, first at {i}: got {got.reshape(-1)[i]}, "
                             f"want {want.reshape(-1)[i]}, tolerance {tol.expand_as(want).reshape(-1)[i]}")


# -------------------------------------------------------------------------------------- page plan
def plan_reference(ctx, new, release, ps, table, pool, n_free, max_rows):
    """The plan one environment after the other, on lists; None where it does not fit."""
    table, pool = [list(r) for r in table], list(pool[:n_free])
    ctx = list(ctx)
    for e in range(len(ctx)):
        if release and release[e]:
            pool += table[e][:-(-ctx[e] // ps)]
            ctx[e] = 0
    rows, start = [], [0]
    for e, (c, n) in enumerate(zip(ctx, new)):
        for col in range(-(-c // ps), -(-(c + n) // ps)):
            if not pool or col >= len(table[e]):
                return None
            table[e][col] = pool.pop()
        rows += [(e, c + i, table[e][(c + i) // ps] * ps + (c + i) % ps) for i in range(n)]
        start.append(len(rows))
    if len(rows) > max_rows:
        return None
    rows += [(-1, -1, -1)] * (max_rows - len(rows))
    return {"table": table, "ctx": [c + n for c, n in zip(ctx, new)], "n_free": len(pool), "start": start, "rows": rows}


def plan_call(ctx, new, release, ps, table, pool, n_pages, n_free, max_rows, in_place=False):
    t = {"ctx": ints(ctx), "new": ints(new), "table": ints(table), "pool": ints(pool), "n_free": ints([n_free])}
    rel = ints(release) if release else None
    out = {"ctx": t["ctx"] if in_place else torch.full_like(t["ctx"], -9), "n_free": t["n_free"] if in_place else ints([-9]),
           "start": torch.full((len(ctx) + 1,), -9, dtype=torch.int32, device="cuda")}
    rows = torch.full((3, max(1, max_rows)), -9, dtype=torch.int32, device="cuda")
    rc = V.vla_page_plan(t["ctx"].data_ptr(), t["new"].data_ptr(), rel.data_ptr() if release else 0, len(ctx), ps, t["table"].data_ptr(),
                         t["table"].shape[1], t["pool"].data_ptr(), n_pages, t["n_free"].data_ptr(), out["ctx"].data_ptr(),
                         out["n_free"].data_ptr(), out["start"].data_ptr(), rows[0].data_ptr() if max_rows else 0,
                         rows[1].data_ptr() if max_rows else 0, rows[2].data_ptr() if max_rows else 0, max_rows)
    assert rc == 0, V.vla_last_error()
    bits = status()
    return {"table": t["table"].tolist(), "pool": t["pool"].tolist(), "ctx": out["ctx"].tolist(), "n_free": out["n_free"].item(),
            "start": out["start"].tolist(), "rows": [tuple(r) for r in rows.t().tolist()][:max_rows], "bits": bits}


def plan_state(seed, B, ps, ctx_most, new_most, spare=3, some_empty=True):
    g = torch.Generator().manual_seed(seed)
    draw = lambda most: torch.randint(0, most + 1, (B,), generator=g).tolist()  # noqa: E731
    ctx, new = draw(ctx_most), draw(new_most)
    if some_empty:
        ctx[0], new[-1] = 0, 0
    width = max(-(-(c + n) // ps) for c, n in zip(ctx, new)) + 1
    used = [-(-c // ps) for c in ctx]
    need = sum(-(-(c + n) // ps) for c, n in zip(ctx, new))
    n_pages = need + spare
    order = torch.randperm(n_pages, generator=g).tolist()
    table, at = [], 0
    for u in used:
        table.append(order[at:at + u] + [-7] * (width - u))
        at += u
    free = order[at:]
    return ctx, new, table, free + [-5] * (n_pages - len(free)), n_pages, len(free)


@pytest.mark.parametrize("B,ps,ctx_most,new_most", [(1, 16, 0, 1), (1, 16, 40, 5000), (3, 1, 7, 4), (5, 12, 50, 30), (16, 16, 300, 1),
                                                    (256, 16, 0, 320), (257, 64, 1000, 3), (1000, 8, 20, 20), (1025, 16, 64, 17),
                                                    (4096, 16, 100, 2)])
@pytest.mark.parametrize("releases", [False, True])
def test_page_plan(B, ps, ctx_most, new_most, releases):
    ctx, new, table, pool, n_pages, n_free = plan_state(B + ps, B, ps, ctx_most, new_most)
    release = [int(e % 3 == 1) for e in range(B)] if releases else None
    for max_rows, in_place in ((max(1, sum(new)), False), (sum(new) + 37, True)):
        want = plan_reference(ctx, new, release, ps, table, pool, n_free, max_rows)
        got = plan_call(ctx, new, release, ps, table, pool, n_pages, n_free, max_rows, in_place)
        assert got["bits"] == 0
        for k in ("ctx", "n_free", "start", "rows", "table"):
            assert got[k] == want[k], (k, max_rows)


def test_page_plan_without_rows_only_releases():
    ctx, new, table, pool, n_pages, n_free = plan_state(5, 6, 4, 30, 0, some_empty=False)
    got = plan_call(ctx, new, [1] * 6, 4, table, pool, n_pages, n_free, 0)
    assert got["bits"] == 0 and got["ctx"] == [0] * 6 and got["n_free"] == n_pages and got["start"] == [0] * 7
    assert sorted(got["pool"]) == list(range(n_pages))


@pytest.mark.parametrize("fault", ["pages", "rows", "columns", "negative_new", "negative_ctx", "n_free", "overflow"])
def test_a_plan_that_does_not_fit_changes_nothing(fault):
    B, ps = 9, 16
    ctx, new, table, pool, n_pages, n_free = plan_state(3, B, ps, 60, 40)
    max_rows, release = sum(new), [1] + [0] * (B - 1)
    if fault == "pages":
        n_free = 2
        new = [40] * B
        max_rows = 40 * B
        table = [r + [-7] * 4 for r in table]
    elif fault == "rows":
        max_rows -= 1
    elif fault == "columns":
        new[4] = 16 * len(table[0]) - ctx[4] + 1
        max_rows = sum(new)
    elif fault == "negative_new":
        new[3] = -1
    elif fault == "negative_ctx":
        ctx[3] = -16
    elif fault == "n_free":
        n_free = n_pages + 1
    else:
        new = [2 ** 31 - 1] * B
    got = plan_call(ctx, new, release, ps, table, pool, n_pages, n_free, max_rows)
    assert got["bits"] == V.VLA_STATUS_PAGES
    assert got["ctx"] == ctx and got["n_free"] == n_free and got["table"] == table and got["pool"] == pool
    assert got["start"] == [0] * (B + 1) and got["rows"] == [(-1, -1, -1)] * max_rows


def test_a_page_outside_the_pool_gives_no_slot():
    got = plan_call([0, 3], [2, 2], None, 4, [[-1, -1], [9, -1]], [1, 99, 0], 3, 2, 4)
    assert got["bits"] == V.VLA_STATUS_PAGES
    assert got["rows"] == [(0, 0, -1), (0, 1, -1), (1, 3, -1), (1, 4, 4)]


# ------------------------------------------------------------------------------------ rotary table
@pytest.mark.parametrize("n_pos,dim,theta", [(1, 16, 1e4), (300, 64, 1e4), (1000, 128, 5e5), (131072, 32, 1e4)])
@pytest.mark.parametrize("kind", [V.VLA_ROPE_PLAIN, V.VLA_ROPE_LINEAR, V.VLA_ROPE_TURNS, V.VLA_ROPE_LOG_TURNS])
def test_rope_table(n_pos, dim, theta, kind):
    factor, length, low, high, amp = 8.0, 4096.0, 1.0, 32.0, 1.25
    t = torch.full((n_pos, dim // 2, 2), float("nan"), device="cuda")
    assert V.vla_rope_table(t.data_ptr(), n_pos, dim, theta, kind, factor, length, low, high, amp) == 0
    f = theta ** (-torch.arange(0, dim, 2, dtype=F64) / dim)
    if kind == V.VLA_ROPE_LINEAR:
        f = f / factor
    elif kind != V.VLA_ROPE_PLAIN:
        turns = length * f / (2 * math.pi)
        s = (turns - low) / (high - low) if kind == V.VLA_ROPE_TURNS else torch.log(turns / low) / math.log(high / low)
        s = s.clamp(0, 1)
        f = f * s + (1 - s) * f / factor
    a = torch.arange(n_pos, dtype=F64)[:, None] * f
    want = amp * torch.stack([torch.cos(a), torch.sin(a)], -1)
    # the 64-bit angle is off by a few 2^-53 of itself, the result rounded to 32 bits
    within(t, want, n_pos * 2.0 ** -50 + 2 * amp * E, "table")


# ------------------------------------------------------------------------------------ rope append
def make_cache(g, n_pages, ps, Hk, hd, cache, order, fill=None):
    shape = {"head": (n_pages, Hk, ps, hd), "slot": (n_pages, ps, Hk, hd), "both": (n_pages, 2, Hk, ps, hd)}[order]
    if order == "both":  # keys and values of a page side by side in one buffer
        x = normal(g, *shape, dtype=TYPE[cache])
        k, v = x[:, 0], x[:, 1]
    else:
        k, v = (normal(g, *shape, dtype=TYPE[cache]) for _ in range(2))
        if order == "slot":
            k, v = k.permute(0, 2, 1, 3), v.permute(0, 2, 1, 3)
    if fill is not None:
        k.fill_(fill)
        v.fill_(fill)
    return k, v


def describe(k, v, cache):
    n_pages, Hk, ps, hd = k.shape
    return V.VlaPagedKv(k.data_ptr(), v.data_ptr(), CODE[cache], n_pages, ps, Hk, hd, k.stride(0), k.stride(1), k.stride(2))


def turned(x, gain, eps, rope, pos, dim, interleaved):
    """(norm and rotation in 64 bits, the magnitude that its rounding errors scale with)"""
    x = x.to(F64)
    size = x.abs()
    if gain is not None:
        r = gain.to(F64) / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
        x, size = x * r, size * r.abs()
    if rope is not None:
        c, s = (rope.to(F64)[pos][:, None, :, i] for i in (0, 1))
        i = torch.arange(0, dim, 2, device=x.device) if interleaved else torch.arange(dim // 2, device=x.device)
        j = i + 1 if interleaved else i + dim // 2
        y, t = x.clone(), size.clone()
        y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
        t[..., i] = t[..., j] = (size[..., i] + size[..., j]) * torch.maximum(c.abs(), s.abs())
        x, size = y, t
    return x, size


def append_case(seed, rows, H, Hk, hd, act, cache, norm, dim, interleaved, ps, order, in_place=False, pad=0, holes=()):
    g = gen(seed)
    n_pages, n_pos = -(-rows // ps) + 3, rows + 50
    k_cache, v_cache = make_cache(g, n_pages, ps, Hk, hd, cache, order)
    width = (H + 2 * Hk) * hd + pad
    qkv = normal(g, rows, width, dtype=TYPE[act], std=1.3)
    q, k, v = (qkv[:, a * hd:b * hd] for a, b in ((0, H), (H, H + Hk), (H + Hk, H + 2 * Hk)))
    pos = torch.randint(0, n_pos, (rows,), generator=g, device="cuda").to(torch.int32)
    slot = torch.randperm(n_pages * ps, generator=g, device="cuda")[:rows].to(torch.int32)
    for r, which in holes:
        (pos if which == "pos" else slot)[r] = -1
    gains = [(1 + 0.3 * normal(g, hd)).to(torch.bfloat16) for _ in range(2)] if norm else [None, None]
    rope = torch.empty(n_pos, max(dim, 16) // 2, 2, device="cuda")
    if dim:
        assert V.vla_rope_table(rope.data_ptr(), n_pos, dim, 1e4) == 0
    before = [t.clone() for t in (qkv, k_cache, v_cache)]
    q_out = q if in_place else torch.full((rows, H * hd + 8), float("nan"), dtype=TYPE[act], device="cuda")[:, :H * hd]
    kv = describe(k_cache, v_cache, cache)
    ptr = lambda t: t.data_ptr() if t is not None else 0  # noqa: E731
    rc = V.vla_rope_append(q.data_ptr(), width, k.data_ptr(), width, v.data_ptr(), width, CODE[act], rows, H, kv, ptr(gains[0]),
                           ptr(gains[1]), 1e-6, rope.data_ptr() if dim else 0, n_pos, dim, interleaved, pos.data_ptr(),
                           slot.data_ptr(), q_out.data_ptr(), q_out.stride(0))
    assert rc == 0, V.vla_last_error()
    x0 = before[0].to(F64)
    heads = lambda a, b: x0[:, a * hd:b * hd].reshape(rows, b - a, hd)  # noqa: E731
    at = pos.long().clamp(min=0)
    args = (1e-6, rope if dim else None, at, dim, interleaved)
    want_q, size_q = turned(heads(0, H), gains[0], *args)
    want_k, size_k = turned(heads(H, H + Hk), gains[1], *args)
    empty = (pos < 0)[:, None, None]
    # a sum of hd squares, rsqrt, two products, then two products and a sum
    fuzz = (8 + (4 * hd ** 0.5 if norm else 0)) * E
    within(q_out.reshape(rows, H, hd) if in_place is False else q.reshape(rows, H, hd), torch.where(empty, 0.0, want_q),
           fuzz * size_q + U[act] * want_q.abs() + TINY[act], "q")
    keep = (pos >= 0) & (slot >= 0)
    page, off = slot.long()[keep] // ps, slot.long()[keep] % ps
    for name, buf, old, want, size in (("k", k_cache, before[1], want_k, size_k),
                                       ("v", v_cache, before[2], heads(H + Hk, H + 2 * Hk), heads(H + Hk, H + 2 * Hk).abs())):
        full, tol = old.to(F64), torch.zeros(old.shape, dtype=F64, device="cuda")
        full[page, :, off] = want[keep]
        tol[page, :, off] = (fuzz * size + U[cache] * want.abs() + TINY[cache])[keep]
        within(buf, full, tol, name)  # and every other slot as it was
    if not in_place:
        assert torch.equal(qkv, before[0])
    else:
        assert torch.equal(qkv[:, H * hd:], before[0][:, H * hd:])


@pytest.mark.parametrize("act,cache", [("f32", "f16"), ("f16", "f16"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f16")])
@pytest.mark.parametrize("H,Hk,hd,dim,interleaved", [(4, 4, 64, 64, False), (5, 1, 64, 32, True), (8, 2, 128, 128, False),
                                                     (7, 7, 128, 48, False), (6, 3, 128, 128, True), (2, 2, 64, 16, False), (3, 1, 128, 0, False)])
@pytest.mark.parametrize("norm", [False, True])
def test_rope_append(act, cache, H, Hk, hd, dim, interleaved, norm):
    append_case(H * hd + dim, 37, H, Hk, hd, act, cache, norm, dim, interleaved, 12, "head", holes=((3, "pos"), (20, "slot")))
    assert status() == 0


@pytest.mark.parametrize("rows", [1, 2, 15, 700, 5001])
@pytest.mark.parametrize("ps,order", [(1, "slot"), (16, "both"), (48, "slot"), (64, "head")])
def test_rope_append_rows_pages_and_orders(rows, ps, order):
    append_case(rows + ps, rows, 8, 2, 128, "bf16", "bf16", True, 128, False, ps, order, in_place=rows % 2 == 0, pad=24)
    append_case(rows + ps, rows, 3, 3, 64, "f32", "f16", False, 64, True, ps, order, in_place=rows % 2 == 1, pad=8)
    assert status() == 0


@pytest.mark.parametrize("act,cache", [("f32", "f16"), ("f16", "f16"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f16")])
@pytest.mark.parametrize("H,Hk,hd,dim,interleaved", [(5, 2, 64, 64, False), (9, 1, 64, 32, True), (6, 2, 128, 128, False), (4, 4, 128, 64, True),
                                                     (3, 1, 64, 0, False), (2, 2, 128, 0, False)])
@pytest.mark.parametrize("norm", [False, True])
def test_rope_append_whole_rows(act, cache, H, Hk, hd, dim, interleaved, norm):
    # more rows than are cut over several warps
    append_case(H * hd + dim, 5003, H, Hk, hd, act, cache, norm, dim, interleaved, 16, "slot", pad=8, holes=((3, "pos"), (4999, "slot"), (5002, "pos")))
    assert status() == 0


def test_rope_append_status_and_saturation():
    g = gen(1)
    k_cache, v_cache = make_cache(g, 2, 4, 1, 64, "f16", "head", fill=5.0)
    kv = describe(k_cache, v_cache, "f16")
    x = normal(g, 4, 3 * 64)
    x[1, 64] = 1e6       # a key beyond fp16
    x[1, 129] = -1e9     # a value beyond fp16
    x[1, 130] = float("inf")
    q_out = torch.full((4, 64), 3.0, device="cuda")

    def call(pos, slot):
        p, s = ints(pos), ints(slot)
        assert V.vla_rope_append(x.data_ptr(), 192, x.data_ptr() + 256, 192, x.data_ptr() + 512, 192, V.VLA_F32, 4, 1, kv, 0, 0, 1e-6,
                                 0, 0, 0, 0, p.data_ptr(), s.data_ptr(), q_out.data_ptr(), 64) == 0
        return status()

    assert call([0, 1, 2, 3], [0, 1, 2, 7]) == V.VLA_STATUS_SATURATED
    assert k_cache[0, 0, 1, 0] == 65504 and v_cache[0, 0, 1, 1] == -65504 and torch.isinf(v_cache[0, 0, 1, 2])
    k_cache.fill_(5.0)
    assert call([0, -2, 2, 3], [0, 1, 8, -2]) == V.VLA_STATUS_PAGES
    assert bool((k_cache[0, 0, 1:] == 5.0).all()) and bool((k_cache[1] == 5.0).all())  # only slot 0 was filed
    assert bool((q_out[1] == 0).all()) and torch.equal(q_out[2], x[2, :64])


# --------------------------------------------------------------------------------- paged attention
def attend_reference(q, k, v, table, ps, env, pos, scale):
    """Outputs and log-sums in 64 bits, with what their errors scale with: sum p |v| and the largest
    sum |q| |k| of a score."""
    rows, H, hd = q.shape
    Hk = k.shape[1]
    out = torch.zeros(rows, H, hd, dtype=F64, device="cuda")
    lse = torch.full((rows, H), -math.inf, dtype=F64, device="cuda")
    size, dot = torch.zeros_like(out), torch.zeros(rows, H, dtype=F64, device="cuda")
    for r in range(rows):
        n = int(pos[r]) + 1
        if n <= 0:
            continue
        t = torch.arange(n, device="cuda")
        page = table[int(env[r])].long()[t // ps]
        kk, vv = k[page, :, t % ps].to(F64), v[page, :, t % ps].to(F64)
        qq = q[r].to(F64).view(Hk, H // Hk, hd)
        s = torch.einsum("hgd,nhd->hgn", qq, kk) * scale
        p = torch.softmax(s, -1)
        out[r] = torch.einsum("hgn,nhd->hgd", p, vv).reshape(H, hd)
        size[r] = torch.einsum("hgn,nhd->hgd", p, vv.abs()).reshape(H, hd)
        lse[r] = torch.logsumexp(s, -1).view(H)
        dot[r] = (torch.einsum("hgd,nhd->hgn", qq.abs(), kk.abs()) * abs(scale)).amax(-1).view(H)
    return out, lse, size, dot


def attend_check(q, k, v, table, ps, env, pos, act, cache, out, lse, scale):
    want, want_lse, size, dot = attend_reference(q, k, v, table, ps, env, pos, scale)
    hd = q.shape[-1]
    n = (pos.to(F64) + 1).clamp(min=1).to("cuda")[:, None]
    weight = 2.0 ** -22 if cache == "f16" else 2.0 ** -16
    # a score's error moves its weight by as much; sums of n weights and products
    score = dot * (2.0 ** -22 + (16 + 4 * hd ** 0.5 + hd / 8) * E)
    c = 2 * score + weight + (16 + 4 * n.sqrt() + n / 8) * E
    within(out.view_as(want), want, c[..., None] * size + U[act] * want.abs() + TINY[act], "out")
    within(lse, want_lse, c + 4 * E * want_lse.abs().nan_to_num(0, 0, 0), "lse")


def attend_call(q, k, v, table, env, pos, act, cache, scale, ws, n_env=None, stream=0, ldo_pad=0):
    rows, H, hd = q.shape
    out = torch.full((rows, H * hd + ldo_pad), float("nan"), dtype=TYPE[act], device="cuda")
    lse = torch.full((rows, H), float("nan"), device="cuda")
    rc = V.vla_paged_attn(q.data_ptr(), q.stride(0), CODE[act], rows, H, describe(k, v, cache), table.data_ptr(), table.shape[1],
                          n_env if n_env is not None else table.shape[0], env.data_ptr(), pos.data_ptr(), scale, out.data_ptr(),
                          out.stride(0), lse.data_ptr(), ws.data_ptr(), ws.numel(), stream)
    assert rc == 0, V.vla_last_error()
    return out[:, :H * hd].reshape(rows, H, hd), lse


def workspace(hd):
    return torch.zeros(V.vla_paged_attn_workspace_bytes(hd), dtype=torch.uint8, device="cuda")


def attend_state(seed, lengths, H, Hk, hd, act, cache, ps, order, q_std=1.5, extra_cols=2):
    """Pages in random order; what no row may read (slots past each end, pages that nobody has) is NaN."""
    g = gen(seed)
    used = [-(-n // ps) for n in lengths]
    n_pages = sum(used) + 3
    k, v = make_cache(g, n_pages, ps, Hk, hd, cache, order)
    perm = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lengths), max(used + [1]) + extra_cols), 2 ** 30, dtype=torch.int32, device="cuda")
    at = 0
    for e, n in enumerate(lengths):
        table[e, :used[e]] = perm[at:at + used[e]]
        at += used[e]
        if n % ps:
            k[int(table[e, used[e] - 1]), :, n % ps:] = float("nan")
            v[int(table[e, used[e] - 1]), :, n % ps:] = float("nan")
    k[perm[at:].long()] = float("nan")
    v[perm[at:].long()] = float("nan")
    env = ints(range(len(lengths)))
    pos = ints([n - 1 for n in lengths])
    q = normal(g, len(lengths), H, hd, dtype=TYPE[act], std=q_std)
    return q, k, v, table, env, pos


TYPES = [("f32", "f16"), ("f16", "f16"), ("bf16", "bf16")]


@pytest.mark.parametrize("act,cache", TYPES)
@pytest.mark.parametrize("H,Hk,hd", [(4, 4, 64), (1, 1, 128), (8, 2, 128), (14, 2, 64), (8, 1, 128), (32, 2, 64), (10, 1, 128), (20, 20, 128)])
def test_paged_attn_heads_and_types(act, cache, H, Hk, hd):
    lengths = [1, 0, 2, 15, 16, 17, 63, 64, 65, 300, 129, 31]
    s = attend_state(H * hd, lengths, H, Hk, hd, act, cache, 16, "head")
    out, lse = attend_call(*s, act, cache, hd ** -0.5, workspace(hd))
    attend_check(*s[:4], 16, s[4], s[5], act, cache, out, lse, hd ** -0.5)
    assert status() == 0


@pytest.mark.parametrize("ps", [1, 5, 12, 16, 32, 64, 200, 256])
@pytest.mark.parametrize("order", ["head", "slot", "both"])
def test_paged_attn_pages_and_orders(ps, order):
    lengths = [70, 1, 257, 640, 33, 200, 199, 201]
    s = attend_state(ps, lengths, 8, 2, 128, "bf16", "bf16", ps, order)
    out, lse = attend_call(*s, "bf16", "bf16", 0.1, workspace(128), ldo_pad=8)
    attend_check(*s[:4], ps, s[4], s[5], "bf16", "bf16", out, lse, 0.1)
    s = attend_state(ps, lengths, 3, 3, 64, "f32", "f16", ps, order)
    out, lse = attend_call(*s, "f32", "f16", 0.125, workspace(64))
    attend_check(*s[:4], ps, s[4], s[5], "f32", "f16", out, lse, 0.125)
    assert status() == 0


@pytest.mark.parametrize("act,cache", TYPES)
@pytest.mark.parametrize("lengths,H,Hk,hd", [([20000], 4, 4, 128), ([70000], 8, 1, 128), ([5000, 0, 1, 37, 9000, 128], 8, 2, 64),
                                             ([1500] * 40, 4, 4, 64), ([300] * 200, 4, 2, 128), ([17] * 3000, 2, 1, 64)])
def test_paged_attn_lengths(act, cache, lengths, H, Hk, hd):
    s = attend_state(len(lengths), lengths, H, Hk, hd, act, cache, 16, "head")
    ws = workspace(hd)
    out, lse = attend_call(*s, act, cache, hd ** -0.5, ws)
    attend_check(*s[:4], 16, s[4], s[5], act, cache, out, lse, hd ** -0.5)
    again, lse2 = attend_call(*s, act, cache, hd ** -0.5, ws)
    assert torch.equal(again, out) and torch.equal(lse2, lse)  # equal calls give equal bits
    assert status() == 0


@pytest.mark.parametrize("act,cache", TYPES)
@pytest.mark.parametrize("ps,H,Hk,hd", [(16, 12, 12, 128), (24, 12, 12, 128), (5, 12, 12, 128), (32, 10, 10, 64), (12, 10, 10, 64), (16, 28, 4, 128),
                                        (40, 16, 4, 64), (8, 16, 1, 64)])
def test_paged_attn_many_short_items(act, cache, ps, H, Hk, hd):
    # single warps take whole items, one to three each, some of no position; then a few longer ones, which all warps share
    lengths = [(7 * e) % 41 for e in range(110 * 12 // Hk)]
    for n in (0, 900):
        s = attend_state(ps + n, lengths + [n], H, Hk, hd, act, cache, ps, "head")
        out, lse = attend_call(*s, act, cache, hd ** -0.5, workspace(hd))
        attend_check(*s[:4], ps, s[4], s[5], act, cache, out, lse, hd ** -0.5)
    assert status() == 0


@pytest.mark.parametrize("act,cache", TYPES)
def test_paged_attn_peaked_weights_over_a_flat_tail(act, cache):
    # one position holds half of the weight, 30000 others share the rest: each of their weights is 1e-5
    n, hd = 30001, 64
    q, k, v, table, env, pos = attend_state(8, [n], 2, 1, hd, act, cache, 16, "head")
    k.mul_(0.05)
    first = table[0, 0].long()
    q[:] = 1.0
    k[first, :, 0] = math.log(n) / hd / 0.125
    out, lse = attend_call(q, k, v, table, env, pos, act, cache, 0.125, workspace(hd))
    attend_check(q, k, v, table, 16, env, pos, act, cache, out, lse, 0.125)


def test_paged_attn_rising_scores():
    # the maximum moves at every step
    n, hd = 3000, 128
    q, k, v, table, env, pos = attend_state(9, [n, n - 700], 4, 4, hd, "f32", "f16", 16, "head")
    t = torch.arange(n, device="cuda")
    for e in range(2):
        m = n - 700 * e
        k[table[e].long()[t[:m] // 16], :, t[:m] % 16] += (t[:m] / 400.0)[:, None, None]
    q[:] = q.abs() * 0.3
    out, lse = attend_call(q, k, v, table, env, pos, "f32", "f16", hd ** -0.5, workspace(hd))
    attend_check(q, k, v, table, 16, env, pos, "f32", "f16", out, lse, hd ** -0.5)


def test_paged_attn_rows_share_and_skip_environments():
    # six rows of one environment (re-scored actions), rows in no order, padding rows
    q, k, v, table, _, _ = attend_state(4, [90, 50, 400], 8, 4, 64, "f16", "f16", 16, "head")
    env = ints([2, 0, 0, -1, 0, 1, 2, 2, -1, 0])
    pos = ints([399, 84, 85, -1, 86, 0, 12, 398, -1, 89])
    g = gen(3)
    q = normal(g, 10, 8, 64, dtype=torch.float16)
    out, lse = attend_call(q, k, v, table, env, pos, "f16", "f16", 0.2, workspace(64))
    attend_check(q, k, v, table, 16, env, pos, "f16", "f16", out, lse, 0.2)
    assert status() == 0


def test_paged_attn_workspace_serves_calls_of_any_size():
    ws = workspace(128)
    small = attend_state(1, [5000], 8, 1, 128, "bf16", "bf16", 16, "head")
    large = attend_state(2, [700, 20, 1] * 60, 8, 8, 128, "bf16", "bf16", 16, "slot")
    first = attend_call(*small, "bf16", "bf16", 0.09, ws)
    for _ in range(3):
        out, lse = attend_call(*large, "bf16", "bf16", 0.09, ws)
        attend_check(*large[:4], 16, large[4], large[5], "bf16", "bf16", out, lse, 0.09)
        again = attend_call(*small, "bf16", "bf16", 0.09, ws)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_paged_attn_status():
    q, k, v, table, env, pos = attend_state(6, [40, 40, 40, 40, 40], 2, 2, 64, "f16", "f16", 16, "head")
    want = attend_call(q, k, v, table, env, pos, "f16", "f16", 0.1, workspace(64))
    assert status() == 0
    bad_env, bad_pos, bad_table = env.clone(), pos.clone(), table.clone()
    bad_env[1] = 5
    bad_pos[2] = 16 * table.shape[1]
    bad_pos[3] = -2
    bad_table[4, 1] = k.shape[0]  # its 16 positions are left out
    out, lse = attend_call(q, k, v, bad_table, bad_env, bad_pos, "f16", "f16", 0.1, workspace(64))
    assert status() == V.VLA_STATUS_PAGES
    assert torch.equal(out[0], want[0][0]) and torch.equal(lse[0], want[1][0])
    assert bool((out[1:4] == 0).all()) and bool((lse[1:4] == -math.inf).all())
    assert bool(torch.isfinite(out[4].float()).all())


def test_paged_attn_positions_at_the_end_of_32_bits():
    ps = 1 << 20
    k, v = (torch.zeros(1, 1, ps, 64, dtype=torch.float16, device="cuda") for _ in range(2))
    q = torch.ones(3, 1, 64, dtype=torch.float16, device="cuda")
    table = torch.zeros(1, 2048, dtype=torch.int32, device="cuda")
    env, pos = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.tensor([2**31 - 1, 5, -1], dtype=torch.int32, device="cuda")
    v[0, 0, :6] = 1.0
    out, lse = attend_call(q, k, v, table, env, pos, "f16", "f16", 0.1, workspace(64))
    assert status() == V.VLA_STATUS_PAGES
    assert bool((out[::2] == 0).all()) and bool((lse[::2] == -math.inf).all()) and bool((out[1] == 1).all())


def test_paged_attn_offsets_beyond_32_bits():
    # one buffer of 2^31 + elements; its last pages lie past the 32-bit element offsets
    hd, ps, n_pages = 64, 16, 1040
    stride = 2 ** 21
    buf = torch.empty(n_pages * stride, dtype=torch.float16, device="cuda")
    view = lambda at: buf.as_strided((n_pages, 1, ps, hd), (stride, ps * hd, hd, 1), at)  # noqa: E731
    k, v = view(0), view(stride // 2)
    g = gen(2)
    pages = [1039, 0, 1027, 1023, 1024]
    for p in pages:
        k[p] = normal(g, 1, ps, hd, dtype=torch.float16)
        v[p] = normal(g, 1, ps, hd, dtype=torch.float16)
    table, env, pos = ints([pages]), ints([0]), ints([70])
    q = normal(g, 1, 4, hd, dtype=torch.float16)
    out, lse = attend_call(q, k, v, table, env, pos, "f16", "f16", 0.3, workspace(hd))
    attend_check(q, k, v, table, ps, env, pos, "f16", "f16", out, lse, 0.3)
    x = normal(g, 2, 3 * hd, dtype=torch.float16)
    slot, where = ints([1039 * ps + 7, 1030 * ps + 15]), ints([0, 1])
    q_out = torch.empty(2, hd, dtype=torch.float16, device="cuda")
    assert V.vla_rope_append(x.data_ptr(), 192, x.data_ptr() + 128, 192, x.data_ptr() + 256, 192, V.VLA_F16, 2, 1,
                             describe(k, v, "f16"), 0, 0, 1e-6, 0, 0, 0, 0, where.data_ptr(), slot.data_ptr(), q_out.data_ptr(), hd) == 0
    assert torch.equal(k[1039, 0, 7], x[0, 64:128]) and torch.equal(v[1030, 0, 15], x[1, 128:])
    assert status() == 0


def test_calls_on_another_stream_follow_its_order():
    side = torch.cuda.Stream()
    q, k, v, table, env, pos = attend_state(6, [400, 1000], 4, 4, 128, "f16", "f16", 16, "head")
    q2 = torch.empty_like(q)
    ws = workspace(128)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        q2.copy_(q)
        out, lse = attend_call(q2, k, v, table, env, pos, "f16", "f16", 0.1, ws, stream=side.cuda_stream)
    side.synchronize()
    attend_check(q, k, v, table, 16, env, pos, "f16", "f16", out, lse, 0.1)


# ---------------------------------------------------------------------------------- token log-probs
def logprob_call(x, tokens, T, top, act, want=("logprob", "entropy", "lse")):
    n, vocab = x.shape
    o = {k: torch.full((n,), 777.0, device="cuda") for k in want}
    ids = torch.full((n, top), -9, dtype=torch.int32, device="cuda")
    lps = torch.full((n, top), 777.0, device="cuda")
    ptr = lambda k: o[k].data_ptr() if k in o else 0  # noqa: E731
    rc = V.vla_token_logprobs(x.data_ptr(), x.stride(0), CODE[act], n, vocab, tokens.data_ptr() if tokens is not None else 0, T, top,
                              ptr("logprob"), ptr("entropy"), ptr("lse"), ids.data_ptr() if top else 0, lps.data_ptr() if top else 0)
    assert rc == 0, V.vla_last_error()
    return {**o, "ids": ids, "lps": lps}


def logprob_reference(x, tokens, T, top):
    z = x.to(F64) / T
    lse = torch.logsumexp(z, -1)
    none = lse == -math.inf
    lp = torch.where(z == -math.inf, z, z - torch.where(none, 0.0, lse)[:, None])
    p = lp.exp()
    h = torch.where(p > 0, -p * lp, 0.0).sum(-1)
    ids = torch.sort(x.to(F64) + 0.0, dim=-1, descending=True, stable=True).indices[:, :top]
    chosen = torch.zeros_like(lse) if tokens is None else torch.where(
        tokens >= 0, lp.gather(1, tokens.long().clamp(min=0)[:, None])[:, 0], 0.0)
    return {"logprob": chosen, "entropy": h, "lse": lse, "ids": ids, "lps": lp.gather(1, ids), "lp": lp, "p": p}


def logprob_check(x, tokens, T, top, got):
    want = logprob_reference(x, tokens, T, top)
    vocab = x.shape[1]
    finite = torch.where(torch.isfinite(x), x.to(F64), 0.0).abs().amax(-1) / T
    total = (32 + 4 * vocab ** 0.5) * E
    tol = 8 * E * finite + total + 8 * E * math.log(vocab + 1)
    within(got["lse"], want["lse"], tol, "lse")
    within(got["logprob"], want["logprob"], 2 * tol, "logprob")
    within(got["entropy"], want["entropy"], tol * (2 + math.log(vocab)), "entropy")
    if top:
        assert torch.equal(got["ids"].long(), want["ids"]), "ids"
        within(got["lps"], want["lps"], 2 * tol[:, None], "top log-probs")


@pytest.mark.parametrize("act", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,vocab,pad", [(1, 1, 0), (3, 2, 1), (5, 31, 0), (2, 255, 2), (7, 257, 0), (9, 1000, 0), (4, 4099, 5), (1, 32064, 0),
                                            (64, 32064, 0), (300, 8200, 3), (3, 151937, 0), (700, 256, 0)])
@pytest.mark.parametrize("T,top", [(1.0, 0), (1.5, 1), (0.7, 8), (0.0, 32)])
def test_token_logprobs(act, rows, vocab, pad, T, top):
    g = gen(rows + vocab)
    x = normal(g, rows, vocab + pad, dtype=TYPE[act], std=2.5)
    x[:, vocab:] = float("nan")
    x = x[:, :vocab]
    tokens = torch.randint(-1, vocab, (rows,), generator=g, device="cuda").to(torch.int32)
    top = min(top, vocab)
    got = logprob_call(x, tokens, T, top, act)
    assert status() == 0
    logprob_check(x, tokens, T or 1.0, top, got)


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [40, 1000, 32064])
def test_token_logprobs_ties_and_masks(act, vocab):
    g = gen(vocab)
    x = normal(g, 10, vocab, dtype=TYPE[act])
    x[0] = 0.0                                     # all equal: the lowest ids
    x[1] = -math.inf
    x[1, vocab // 2] = 1.0                         # one id only
    x[2] = -math.inf                               # none
    x[3, :vocab - 3] = -math.inf                   # fewer ids than alternatives
    x[4] = (torch.arange(vocab, device="cuda") % 3).to(x.dtype)  # a third of the ids tie for the first place
    x[5] = torch.finfo(x.dtype).min                # masks of the type's lowest value
    x[5, 7] = 0.0
    x[6] = torch.finfo(x.dtype).min                # and nothing else
    x[7] = torch.where(torch.arange(vocab, device="cuda") % 2 == 0, 0.0, -0.0).to(x.dtype)  # zeros of both signs tie
    x[8] = x[8] - 1e4                              # far from zero
    tokens = ints([0, vocab // 2, 3, vocab - 1, 2, 7, 5, 1, 9, 0])
    for T in (1.0, 0.5):
        x[6] = torch.finfo(x.dtype).min if T == 1.0 else torch.finfo(x.dtype).min * 0.25
        x[5] = torch.where(x[5] < 0, x[6], x[5])
        got = logprob_call(x, tokens, T, min(20, vocab), act)
        assert status() == 0
        logprob_check(x, tokens, T, min(20, vocab), got)


def test_token_logprobs_nonfinite_and_bad_tokens():
    g = gen(0)
    x = normal(g, 5, 500)
    x[1, 30] = float("nan")
    x[3, 400] = float("inf")
    clean = logprob_call(x[::2].contiguous(), ints([1, 2, 3]), 1.0, 3, "f32")
    assert status() == 0
    got = logprob_call(x, ints([1, 1, 2, 1, 3]), 1.0, 3, "f32")
    assert status() == V.VLA_STATUS_NONFINITE
    for k in ("logprob", "entropy", "lse", "ids", "lps"):
        assert torch.equal(got[k][::2], clean[k])
        if k != "ids":
            assert bool(torch.isnan(got[k][1::2]).all()), k
    for bad in (500, -2):
        got = logprob_call(x[::2].contiguous(), ints([1, bad, 3]), 1.0, 3, "f32")
        assert status() == V.VLA_STATUS_BAD_TOKEN
        assert got["logprob"][1] == 0 and got["logprob"][0] == clean["logprob"][0]
        assert torch.equal(got["entropy"], clean["entropy"])
    # outputs that are not asked for
    only = logprob_call(x[::2].contiguous(), None, 1.0, 0, "f32", want=("entropy",))
    assert torch.equal(only["entropy"], clean["entropy"])


# 32, 64 and 128 threads a row; rows cut over 2, 4 and 8 CTAs (16-bit rows of 41111 ids stay whole)
@pytest.mark.parametrize("act", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,vocab,pad", [(4000, 300, 3), (2000, 700, 1), (2100, 1290, 0), (1000, 2999, 2), (200, 41111, 1), (130, 90001, 3),
                                            (20, 90001, 5)])
@pytest.mark.parametrize("T,top", [(1.0, 0), (1.5, 2), (0.7, 32)])
def test_token_logprobs_threads_and_cuts(act, rows, vocab, pad, T, top):
    test_token_logprobs(act, rows, vocab, pad, T, top)


@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_token_logprobs_ties_and_masks_of_cut_rows(act):
    test_token_logprobs_ties_and_masks(act, 100003)


@pytest.mark.parametrize("act", ["f32", "f16"])
def test_token_logprobs_nonfinite_in_a_slice(act):
    g = gen(9)
    x = normal(g, 6, 100001, dtype=TYPE[act])
    x[1, 99999] = float("nan")
    x[3, 40000] = float("inf")
    x[5, 0] = float("nan")
    tokens = ints([1, 99999, 2, 50000, 100000, 7])
    clean = logprob_call(x[::2].contiguous(), tokens[::2].contiguous(), 1.0, 5, act)
    assert status() == 0
    got = logprob_call(x, tokens, 1.0, 5, act)
    assert status() == V.VLA_STATUS_NONFINITE
    for k in ("logprob", "entropy", "lse", "lps"):
        assert torch.equal(got[k][::2], clean[k]) and bool(torch.isnan(got[k][1::2]).all()), k
    assert torch.equal(got["ids"][::2], clean["ids"])


# ------------------------------------------------------------------------------------------ gradient
def grad_call(x, tokens, T, lse, entropy, g, h, act, out=None):
    n, vocab = x.shape
    d = torch.full((n, vocab + 3), 777.0, dtype=TYPE[act], device="cuda")[:, :vocab] if out is None else out
    rc = V.vla_token_logprobs_grad(x.data_ptr(), x.stride(0), CODE[act], n, vocab, tokens.data_ptr(), T, lse.data_ptr(),
                                   entropy.data_ptr(), g.data_ptr(), h.data_ptr() if h is not None else 0, d.data_ptr(), d.stride(0))
    assert rc == 0, V.vla_last_error()
    return d


@pytest.mark.parametrize("act", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,vocab,pad", [(1, 1, 0), (3, 7, 1), (5, 256, 0), (6, 1001, 0), (4, 8192, 8), (700, 256, 0), (40, 32064, 0), (2, 151937, 2)])
@pytest.mark.parametrize("T,bonus", [(1.0, True), (1.5, False), (0.0, True)])
def test_token_logprobs_grad(act, rows, vocab, pad, T, bonus):
    gn = gen(rows * 3 + vocab)
    x = normal(gn, rows, vocab + pad, dtype=TYPE[act], std=2.0)[:, :vocab]
    if vocab > 300:
        x[::2, :vocab - 256] = -math.inf
    tokens = torch.randint(0, vocab, (rows,), generator=gn, device="cuda").to(torch.int32)
    if vocab > 300:
        tokens[::2] = vocab - 1 - tokens[::2] % 256
    if rows > 2:
        tokens[2] = -1
    g, h = normal(gn, rows), normal(gn, rows, std=0.3) if bonus else None
    fwd = logprob_call(x, tokens, T, 0, act)
    d = grad_call(x, tokens, T, fwd["lse"], fwd["entropy"], g, h, act)
    t = T or 1.0
    want = logprob_reference(x, tokens, t, 0)
    lp, p, H = want["lp"], want["p"], want["entropy"][:, None]
    gg, hh = g.to(F64)[:, None], (h.to(F64) if bonus else torch.zeros(rows, dtype=F64, device="cuda"))[:, None]
    lp0 = torch.where(p > 0, lp, 0.0)
    exact = -gg * p - hh * p * (lp0 + H)
    exact.scatter_add_(1, tokens.long().clamp(min=0)[:, None], gg)
    kept = (tokens >= 0)[:, None]
    exact = torch.where(kept, exact / t, 0.0)
    finite = torch.where(torch.isfinite(x), x.to(F64), 0.0).abs().amax(-1, keepdim=True) / t
    # the weight's exponent and the sums it comes from, then its products
    eps = 16 * E * (finite + H + 2) + 2 * (32 + 4 * vocab ** 0.5) * E
    tol = eps * p * (gg.abs() + hh.abs() * (lp0.abs() + H + 1) * (2 + math.log(vocab))) / t
    tol.scatter_add_(1, tokens.long().clamp(min=0)[:, None], 4 * E * gg.abs() / t)
    within(d, exact, torch.where(kept, tol + U[act] * exact.abs() + TINY[act], 0.0), "gradient")
    # in place
    own = x.clone() if pad == 0 else x
    assert torch.equal(grad_call(own, tokens, T, fwd["lse"], fwd["entropy"], g, h, act, out=own), d)
    assert status() == 0


def test_token_logprobs_grad_against_differences():
    # the 64-bit objective's central differences: their own error is step^2 / 6 of its third derivative
    # (at most 10 here) plus 2^-52 / step
    gn = gen(5)
    rows, vocab, T, step = 6, 37, 1.3, 1e-4
    x = normal(gn, rows, vocab, std=1.5)
    tokens = ints([3, 36, 0, -1, 12, 3])
    g, h = normal(gn, rows), normal(gn, rows)
    fwd = logprob_call(x, tokens, T, 0, "f32")
    d = grad_call(x, tokens, T, fwd["lse"], fwd["entropy"], g, h, "f32")

    def objective(z):
        r = logprob_reference(z, tokens, T, 0)
        return torch.where(tokens >= 0, g.to(F64) * r["logprob"] + h.to(F64) * r["entropy"], 0.0)

    z = x.to(F64)
    for j in range(vocab):
        up, down = z.clone(), z.clone()
        up[:, j] += step
        down[:, j] -= step
        slope = (objective(up) - objective(down)) / (2 * step)
        within(d[:, j], slope, 2e-6 * (1.0 + g.abs() + h.abs()).to(F64), f"id {j}")
