"""The operators of a token policy over a paged key-value cache, as cases to time and to compare.

A rollout that serves many environments from one pool of cache pages does four things besides its
matrix products: it takes pages for the tokens of the step and maps rows to cache slots ("plan"), it
normalises and rotates queries and keys and files keys and values into their slots ("append"), each
new token attends to its environment's whole paged context ("attend"), and it reads the log
probability of the chosen token, the entropy and the best alternatives off the logits ("logprobs"); the
learning phase sends a gradient back through that last step ("grad").  The sizes are those of this
repository's workloads (1 to 256 environments, prefixes of 16 to 320 rows, contexts of about 80, 300
and 1100 positions, heads of 64 and 128, 32064 ids) and generic ones where the workloads have none
(shared key-value heads, long contexts, wider vocabularies).

Where `own` is false, `run` computes the operators from elementary torch operations in 32 bits;
where it is true, it makes the framework's calls on the same state.
"""
import math

import torch

own = False

DEV = "cuda"
F64 = torch.float64
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
CODE = {"f32": 0, "f16": 1, "bf16": 2}
EPS = 1e-6
THETA = 1e4
MOST_KV = 4.7e9  # bytes of keys and values of the largest context set


# ------------------------------------------------------------------------------------- cases
def _plan(name, envs, ctx, new_min, new_max, page):
    return {"name": name, "kind": "plan", "envs": envs, "ctx": ctx, "new_min": new_min, "new_max": new_max, "page": page}


def _append(name, envs, ctx, new_min, new_max, q_heads, kv_heads, head, act, cache, norm, layout, rope, page, order):
    return {"name": name, "kind": "append", "envs": envs, "ctx": ctx, "new_min": new_min, "new_max": new_max,
            "q_heads": q_heads, "kv_heads": kv_heads, "head": head, "act": act, "cache": cache, "norm": norm,
            "layout": layout, "rope": rope, "page": page, "order": order}


def _attend(name, envs, ctx_min, ctx_max, q_heads, kv_heads, head, act, cache, page, order):
    return {"name": name, "kind": "attend", "envs": envs, "ctx_min": ctx_min, "ctx_max": ctx_max, "q_heads": q_heads,
            "kv_heads": kv_heads, "head": head, "act": act, "cache": cache, "page": page, "order": order}


def _logits(name, kind, rows, vocab, pad, act, temperature, top, narrow):
    return {"name": name, "kind": kind, "rows": rows, "vocab": vocab, "pad": pad, "act": act, "temperature": temperature,
            "top": top, "narrow": narrow}


def listed():
    return [
        # one decode step of 16 environments: one row each, a new page for a few of them
        _plan("plan_b16_step", 16, 290, 1, 1, 16),
        # the prefill of 256 ragged prefixes: about 76000 rows and 4900 pages in one call
        _plan("plan_b256_prefill", 256, 0, 272, 320, 16),
        # one decode step of the smallest shape: 4 rows of 4 heads of 64
        _append("append_b4_step", 4, 80, 1, 1, 4, 4, 64, "f32", "f16", False, "half", 64, 16, "head"),
        # one decode step of 64 environments on the 7B shape, the framework's 32-bit queries
        _append("append_b64_step", 64, 290, 1, 1, 32, 32, 128, "f32", "f16", False, "half", 128, 16, "head"),
        # the prefill of 64 prefixes, four queries to a key head, with norms of queries and keys,
        # interleaved pairs over half of the head, pages laid out slot by slot
        _append("append_b64_prefill", 64, 0, 272, 304, 32, 8, 128, "bf16", "bf16", True, "interleaved", 64, 16, "slot"),
        # one token of the smallest shape over a short context: latency
        _attend("attend_b4_short", 4, 80, 87, 4, 4, 64, "f32", "f16", 16, "head"),
        # one decode step of the 7B shape: 64 environments over ragged contexts of about 290
        _attend("attend_b64", 64, 273, 311, 32, 32, 128, "f32", "f16", 16, "head"),
        # the last turn of 256 environments over long multi-turn contexts
        _attend("attend_b256_turns", 256, 1031, 1097, 32, 32, 128, "f16", "f16", 32, "slot"),
        # few long documents with shared key-value heads, lengths far apart
        _attend("attend_b8_long", 8, 1000, 131072, 32, 8, 128, "bf16", "bf16", 16, "head"),
        # the tokens of one decode step of 64 environments, with the 8 best alternatives
        _logits("logprobs_b64_step", "logprobs", 64, 32064, 0, "f32", 1.5, 8, 0),
        # the learning phase's pass over 512 samples of 7 tokens, some rows held to the action bins
        _logits("logprobs_3584", "logprobs", 3584, 32064, 0, "bf16", 1.0, 4, 256),
        # its gradient, with an entropy bonus
        _logits("grad_3584", "grad", 3584, 32064, 0, "bf16", 1.0, 0, 256),
    ]


def _log_int(rng, lo, hi):
    n = max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    return n + 1 if n == 3072 else n


def draw(rng):
    kind = rng.choice(["plan", "append", "attend", "attend", "logprobs", "grad"])
    page = rng.choice([8, 12, 16, 16, 32, 64])
    if kind == "plan":
        envs = _log_int(rng, 1, 1024)
        new = _log_int(rng, 1, max(1, min(2048, 80000 // envs)))
        c = _plan("", envs, rng.choice([0, _log_int(rng, 1, 4096)]), rng.choice([new, 1, 0]), new, page)
    elif kind in ("append", "attend"):
        q_heads, kv_heads, head = rng.choice([(4, 4, 64), (10, 10, 64), (16, 4, 64), (12, 12, 128), (20, 20, 128), (32, 32, 128),
                                              (32, 8, 128), (64, 8, 128), (8, 1, 128), (28, 4, 128), (16, 1, 64)])
        act, cache = rng.choice([("f32", "f16"), ("f16", "f16"), ("bf16", "bf16")])
        order = rng.choice(["head", "slot"])
        envs = _log_int(rng, 1, 256)
        if kind == "append":
            row = (q_heads + 2 * kv_heads) * head * 4.0
            new = _log_int(rng, 1, max(1, min(2048, int(4e8 / row / envs))))
            c = _append("", envs, rng.choice([0, _log_int(rng, 1, 1024)]), rng.choice([new, 1]), new, q_heads, kv_heads, head,
                        act, cache, rng.random() < 0.5, rng.choice(["half", "interleaved"]),
                        rng.choice([head, head, head // 2, head // 4]), page, order)
        else:
            most = max(1, min(131072, int(MOST_KV / (envs * kv_heads * head * 4.0))))
            ctx = _log_int(rng, 1, most)
            c = _attend("", envs, rng.choice([ctx, max(1, ctx * 3 // 4), 0]), ctx, q_heads, kv_heads, head, act, cache, page, order)
    else:
        vocab = _log_int(rng, 256, 160000)
        rows = _log_int(rng, 1, max(1, min(8192, int(1.1e8 / vocab))))
        c = _logits("", kind, rows, vocab, rng.choice([0, 0, rng.randint(1, 64)]), rng.choice(["f32", "f16", "bf16"]),
                    rng.choice([0.7, 1.0, 1.5]), 0 if kind == "grad" else rng.choice([0, 1, rng.randint(2, 16)]),
                    rng.choice([0, 256]) if vocab > 1024 else 0)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------ inputs
def _spread(n, lo, hi):
    """n lengths over [lo, hi], the same ones for the same arguments; the first is hi, the second lo."""
    return [hi if b == 0 else lo if b == 1 else lo + int((hi - lo + 1) * ((b * 0.6180339887 + 0.31) % 1.0)) for b in range(n)]


def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _normal(g, shape, dtype, std=1.0):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=g)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _ceil(a, b):
    return (a + b - 1) // b


def _pages(g, lengths, page, width):
    """(pages in the pool, a shuffled order of them, table [envs, width] whose first columns hold each
    environment's pages and whose other columns hold -1, pages in use)."""
    used = [_ceil(n, page) for n in lengths]
    total = sum(used)
    n_pages = total + max(4, total // 8)
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    col = torch.arange(width, device=DEV)
    count = torch.tensor(used, device=DEV)
    first = torch.cumsum(count, 0) - count
    table = torch.where(col < count[:, None], order[(first[:, None] + col).clamp(max=n_pages - 1)], -1).to(torch.int32)
    return n_pages, order, table.contiguous(), total


def _rope_table(n_pos, dim):
    """(cos, sin) of each position and pair of a rotation over `dim` channels, 32 bits: [n_pos, dim / 2, 2]."""
    inv = THETA ** (-2.0 * torch.arange(dim // 2, dtype=F64, device=DEV) / dim)
    a = torch.arange(n_pos, dtype=F64, device=DEV)[:, None] * inv
    return torch.stack([torch.cos(a), torch.sin(a)], -1).to(torch.float32).contiguous()


def _plan_inputs(case, seed):
    g = _generator(seed)
    B, ps = case["envs"], case["page"]
    ctx = [case["ctx"] + (b * 7 + int(seed)) % 23 if case["ctx"] else 0 for b in range(B)]
    new = _spread(B, case["new_min"], case["new_max"])
    width = max(_ceil(c + n, ps) for c, n in zip(ctx, new)) + 3
    # the pool has pages for both; those of the present contexts are in the table, the rest is free
    n_pages, order, table, _ = _pages(g, [ps * (_ceil(c + n, ps) + 1) for c, n in zip(ctx, new)], ps, 1)
    used = torch.tensor([_ceil(c, ps) for c in ctx], device=DEV)
    col = torch.arange(width, device=DEV)
    first = torch.cumsum(used, 0) - used
    table = torch.where(col < used[:, None], order[(first[:, None] + col).clamp(max=n_pages - 1)], -1).to(torch.int32).contiguous()
    held = sum(_ceil(c, ps) for c in ctx)
    pool = torch.full((n_pages,), -1, dtype=torch.int32, device=DEV)
    pool[:n_pages - held] = order[held:]
    rows = max(1, sum(new))
    empty = lambda n: torch.empty(n, dtype=torch.int32, device=DEV)  # noqa: E731
    return {"ctx": _ints(ctx), "new": _ints(new), "table": table, "pool": pool, "n_free": _ints([n_pages - held]), "width": width,
            "n_pages": n_pages, "rows": rows, "ctx_out": empty(B), "n_free_out": empty(1), "row_start": empty(B + 1),
            "row_env": empty(rows), "row_pos": empty(rows), "row_slot": empty(rows)}


def _cache(g, case, n_pages):
    """Keys and values as [page, head, slot, channel] views of the order that the case names."""
    ps, H, hd = case["page"], case["kv_heads"], case["head"]
    shape = (n_pages, H, ps, hd) if case["order"] == "head" else (n_pages, ps, H, hd)
    kv = [_normal(g, shape, DTYPE[case["cache"]]) for _ in range(2)]
    return [x if case["order"] == "head" else x.permute(0, 2, 1, 3) for x in kv]


def _append_inputs(case, seed):
    g = _generator(seed)
    B, ps, H, Hk, hd = case["envs"], case["page"], case["q_heads"], case["kv_heads"], case["head"]
    ctx = [case["ctx"] + (b * 7 + int(seed)) % 23 if case["ctx"] else 0 for b in range(B)]
    new = _spread(B, case["new_min"], case["new_max"])
    end = [c + n for c, n in zip(ctx, new)]
    n_pages, _, table, _ = _pages(g, end, ps, max(_ceil(n, ps) for n in end))
    rows = sum(new)
    env = torch.repeat_interleave(torch.arange(B, device=DEV), torch.tensor(new, device=DEV))
    start = torch.tensor([sum(new[:b]) - ctx[b] for b in range(B)], device=DEV)
    pos = torch.arange(rows, device=DEV) - start[env]
    slot = table.long()[env, pos // ps] * ps + pos % ps
    k, v = _cache(g, case, n_pages)
    # the rows of one q|k|v projection
    qkv = _normal(g, (rows, (H + 2 * Hk) * hd), DTYPE[case["act"]], 1.3)
    gain = lambda: (1.0 + 0.2 * _normal(g, (hd,), torch.float32)).to(torch.bfloat16)  # noqa: E731
    s = {"qkv": qkv, "k_cache": k, "v_cache": v, "n_pages": n_pages, "pos": pos.to(torch.int32), "slot": slot.to(torch.int32),
         "rope": _rope_table(max(end), case["rope"]), "n_pos": max(end), "rows": rows,
         "q_gain": gain() if case["norm"] else None, "k_gain": gain() if case["norm"] else None}
    s["q_out"] = torch.empty(rows, H, hd, dtype=DTYPE[case["act"]], device=DEV)
    return s


def _attend_inputs(case, seed):
    g = _generator(seed)
    B, ps, H, hd = case["envs"], case["page"], case["q_heads"], case["head"]
    lengths = _spread(B, case["ctx_min"], case["ctx_max"])
    width = max(1, _ceil(case["ctx_max"], ps))
    n_pages, _, table, _ = _pages(g, lengths, ps, width)
    k, v = _cache(g, case, n_pages)
    q = _normal(g, (B, H, hd), DTYPE[case["act"]], 1.5)
    return {"q": q, "k_cache": k, "v_cache": v, "n_pages": n_pages, "table": table, "width": width,
            "env": torch.arange(B, dtype=torch.int32, device=DEV), "pos": _ints([n - 1 for n in lengths]), "lengths": lengths,
            "out": torch.empty_like(q), "lse": torch.empty(B, H, dtype=torch.float32, device=DEV)}


def _logits_inputs(case, seed):
    g = _generator(seed)
    n, V = case["rows"], case["vocab"]
    x = _normal(g, (n, V + case["pad"]), DTYPE[case["act"]], 2.5)[:, :V]
    token = torch.randint(0, V, (n,), generator=g, device=DEV)
    if case["narrow"]:  # every second row is held to the last `narrow` ids
        x[::2, :V - case["narrow"]] = -math.inf
        token[::2] = V - 1 - token[::2] % case["narrow"]
    if n > 4:
        token[3::11] = -1  # padding: no token to score
    f = lambda *sh: torch.empty(*sh, dtype=torch.float32, device=DEV)  # noqa: E731
    s = {"logits": x, "token": token.to(torch.int32)}
    if case["kind"] == "grad":
        z = x.float() / case["temperature"]
        m = z.amax(-1)
        s["lse"] = m + torch.log(torch.exp(z - m[:, None]).sum(-1))
        p = torch.exp(z - s["lse"][:, None])
        s["entropy"] = -torch.where(p > 0, p * (z - s["lse"][:, None]), 0.0).sum(-1)
        s["g_logprob"] = torch.randn(n, generator=g, device=DEV)
        s["g_entropy"] = torch.full((n,), 0.01, device=DEV)
        s["d_logits"] = torch.empty(n, V, dtype=x.dtype, device=DEV)
    else:
        k = case["top"]
        s.update(logprob=f(n), entropy=f(n), lse=f(n), top_id=torch.empty(n, k, dtype=torch.int32, device=DEV), top_logprob=f(n, k))
    return s


def prepare(case, seed):
    s = {"plan": _plan_inputs, "append": _append_inputs, "attend": _attend_inputs, "logprobs": _logits_inputs,
         "grad": _logits_inputs}[case["kind"]](case, seed)
    s["case"] = case
    s["stream"] = torch.cuda.current_stream().cuda_stream
    if own and "k_cache" in s:  # the descriptor and the workspace that a serving program keeps
        from paper_2505_18719_gb300 import vla as V
        k, v = s["k_cache"], s["v_cache"]
        s["kv"] = V.VlaPagedKv(k.data_ptr(), v.data_ptr(), CODE[case["cache"]], s["n_pages"], case["page"], case["kv_heads"],
                               case["head"], k.stride(0), k.stride(1), k.stride(2))
        if case["kind"] == "attend":
            s["workspace"] = torch.zeros(V.vla_paged_attn_workspace_bytes(case["head"]), dtype=torch.uint8, device=DEV)
    return s


# --------------------------------------------------------------------------------------- run
def run(state):
    return (_own if own else _plain)[state["case"]["kind"]](state)


def _ptr(t):
    return t.data_ptr() if t is not None else 0


def _own_plan(s):
    from paper_2505_18719_gb300 import vla as V
    c = s["case"]
    _ok(V, V.vla_page_plan(_ptr(s["ctx"]), _ptr(s["new"]), 0, c["envs"], c["page"], _ptr(s["table"]), s["width"], _ptr(s["pool"]),
                           s["n_pages"], _ptr(s["n_free"]), _ptr(s["ctx_out"]), _ptr(s["n_free_out"]), _ptr(s["row_start"]),
                           _ptr(s["row_env"]), _ptr(s["row_pos"]), _ptr(s["row_slot"]), s["rows"], s["stream"]))
    return {n: s[n] for n in ("table", "ctx_out", "n_free_out", "row_start", "row_env", "row_pos", "row_slot")}


def _own_append(s):
    from paper_2505_18719_gb300 import vla as V
    c, qkv = s["case"], s["qkv"]
    at, size, ld = qkv.data_ptr(), qkv.element_size(), qkv.stride(0)
    _ok(V, V.vla_rope_append(at, ld, at + c["q_heads"] * c["head"] * size, ld, at + (c["q_heads"] + c["kv_heads"]) * c["head"] * size,
                             ld, CODE[c["act"]], s["rows"], c["q_heads"], s["kv"], _ptr(s["q_gain"]), _ptr(s["k_gain"]), EPS,
                             _ptr(s["rope"]), s["n_pos"], c["rope"], c["layout"] == "interleaved", _ptr(s["pos"]), _ptr(s["slot"]),
                             _ptr(s["q_out"]), c["q_heads"] * c["head"], s["stream"]))
    return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _own_attend(s):
    from paper_2505_18719_gb300 import vla as V
    c = s["case"]
    ld = c["q_heads"] * c["head"]
    _ok(V, V.vla_paged_attn(_ptr(s["q"]), ld, CODE[c["act"]], c["envs"], c["q_heads"], s["kv"], _ptr(s["table"]), s["width"],
                            c["envs"], _ptr(s["env"]), _ptr(s["pos"]), 1.0 / math.sqrt(c["head"]), _ptr(s["out"]), ld,
                            _ptr(s["lse"]), _ptr(s["workspace"]), s["workspace"].numel(), s["stream"]))
    return {"out": s["out"], "lse": s["lse"]}


def _own_logprobs(s):
    from paper_2505_18719_gb300 import vla as V
    c, x = s["case"], s["logits"]
    _ok(V, V.vla_token_logprobs(_ptr(x), x.stride(0), CODE[c["act"]], c["rows"], c["vocab"], _ptr(s["token"]), c["temperature"],
                                c["top"], _ptr(s["logprob"]), _ptr(s["entropy"]), _ptr(s["lse"]), _ptr(s["top_id"]),
                                _ptr(s["top_logprob"]), s["stream"]))
    return {n: s[n] for n in ("logprob", "entropy", "lse", "top_id", "top_logprob")}


def _own_grad(s):
    from paper_2505_18719_gb300 import vla as V
    c, x, d = s["case"], s["logits"], s["d_logits"]
    _ok(V, V.vla_token_logprobs_grad(_ptr(x), x.stride(0), CODE[c["act"]], c["rows"], c["vocab"], _ptr(s["token"]), c["temperature"],
                                     _ptr(s["lse"]), _ptr(s["entropy"]), _ptr(s["g_logprob"]), _ptr(s["g_entropy"]), _ptr(d),
                                     d.stride(0), s["stream"]))
    return {"d_logits": d}


def _ok(V, rc):
    if rc != V.VLA_OK:
        raise V.VlaError(rc, V.vla_last_error())


def _plain_plan(s):
    ps, width, n_pages = s["case"]["page"], s["width"], s["n_pages"]
    ctx, new, table, n_free = s["ctx"].long(), s["new"].long(), s["table"].long(), s["n_free"].long()
    end = ctx + new
    have, want = (ctx + ps - 1) // ps, (end + ps - 1) // ps
    need = want - have
    first = torch.cumsum(need, 0) - need
    col = torch.arange(width, device=DEV)
    at = n_free - 1 - (first[:, None] + col - have[:, None])
    fresh = (col >= have[:, None]) & (col < want[:, None])
    table = torch.where(fresh, s["pool"].long()[at.clamp(0, n_pages - 1)], table)
    row_start = torch.cat([torch.zeros(1, dtype=torch.long, device=DEV), torch.cumsum(new, 0)])
    r = torch.arange(s["rows"], device=DEV)
    live = r < row_start[-1]
    env = torch.searchsorted(row_start[1:], r, right=True).clamp(max=ctx.numel() - 1)
    pos = ctx[env] + r - row_start[env]
    slot = table[env, (pos // ps).clamp(max=width - 1)] * ps + pos % ps
    i32 = lambda t: t.to(torch.int32)  # noqa: E731
    return {"table": i32(table), "ctx_out": i32(end), "n_free_out": i32(n_free - need.sum()), "row_start": i32(row_start),
            "row_env": i32(torch.where(live, env, -1)), "row_pos": i32(torch.where(live, pos, -1)),
            "row_slot": i32(torch.where(live, slot, -1))}


def _normed(x, gain):
    return x if gain is None else x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain.float()


def _rotated(x, cs, layout):
    half = cs.shape[1]
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    if layout == "half":
        a, b = x[..., :half], x[..., half:2 * half]
        return torch.cat([a * c - b * s, b * c + a * s, x[..., 2 * half:]], -1)
    a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
    return torch.cat([torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2), x[..., 2 * half:]], -1)


def _plain_append(s):
    c = s["case"]
    H, Hk, hd = c["q_heads"], c["kv_heads"], c["head"]
    x = s["qkv"].float().view(s["rows"], H + 2 * Hk, hd)
    q, k, v = x[:, :H], x[:, H:H + Hk], x[:, H + Hk:]
    cs = s["rope"][s["pos"].long()]
    q, k = _rotated(_normed(q, s["q_gain"]), cs, c["layout"]), _rotated(_normed(k, s["k_gain"]), cs, c["layout"])
    page, off = s["slot"].long() // c["page"], s["slot"].long() % c["page"]
    s["k_cache"][page, :, off] = k.to(DTYPE[c["cache"]])
    s["v_cache"][page, :, off] = v.to(DTYPE[c["cache"]])
    return {"q": q.to(DTYPE[c["act"]]), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_attend(s):
    c = s["case"]
    B, H, Hk, hd = c["envs"], c["q_heads"], c["kv_heads"], c["head"]
    pages = s["table"].long().clamp(min=0)[s["env"].long()]

    def context(cache):  # [B, Hk, positions, hd]
        return cache[pages].permute(0, 2, 1, 3, 4).reshape(B, Hk, -1, hd).float()

    score = s["q"].float().view(B, Hk, H // Hk, hd) @ context(s["k_cache"]).transpose(2, 3) * (1.0 / math.sqrt(hd))
    seen = torch.arange(score.shape[-1], device=DEV) <= s["pos"].long()[:, None]
    score = torch.where(seen[:, None, None], score, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.where(seen[:, None, None], torch.exp(score - top), 0.0)
    total = p.sum(-1, keepdim=True)
    out = (p @ context(s["v_cache"])) / total
    some = (s["pos"] >= 0)[:, None, None, None]
    lse = torch.where(some, top + torch.log(total), -math.inf)  # an empty context: zeros, and a sum of nothing
    return {"out": torch.where(some, out, 0.0).view(B, H, hd).to(DTYPE[c["act"]]), "lse": lse.view(B, H)}


def _plain_logprobs(s):
    c = s["case"]
    z = s["logits"].float() / c["temperature"]
    m = z.amax(-1, keepdim=True)
    lse = m + torch.log(torch.exp(z - m).sum(-1, keepdim=True))
    lp = z - lse
    p = torch.exp(lp)
    entropy = -torch.where(p > 0, p * lp, 0.0).sum(-1)
    token = s["token"].long()
    chosen = torch.where(token >= 0, lp.gather(1, token.clamp(min=0)[:, None])[:, 0], 0.0)
    # the k largest by value, the lower id first among equals: one whole number per entry orders both
    bits = (s["logits"].float() + 0.0).view(torch.int32)
    key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * (1 << 32) + (c["vocab"] - torch.arange(c["vocab"], device=DEV))
    best = c["vocab"] - (torch.topk(key, c["top"], dim=-1).values & 0xFFFFFFFF)
    return {"logprob": chosen, "entropy": entropy, "lse": lse[:, 0], "top_id": best.to(torch.int32), "top_logprob": lp.gather(1, best)}


def _plain_grad(s):
    c, x = s["case"], s["logits"]
    token, T = s["token"].long(), c["temperature"]
    lp = x.float() / T - s["lse"][:, None]
    p = torch.exp(lp)
    g, h = s["g_logprob"][:, None], s["g_entropy"][:, None]
    d = -g * p - h * torch.where(p > 0, p * (lp + s["entropy"][:, None]), 0.0)
    d = d.scatter_add(1, token.clamp(min=0)[:, None], g) / T
    return {"d_logits": torch.where(token[:, None] >= 0, d, 0.0).to(x.dtype)}


_own = {"plan": _own_plan, "append": _own_append, "attend": _own_attend, "logprobs": _own_logprobs, "grad": _own_grad}
_plain = {"plan": _plain_plan, "append": _plain_append, "attend": _plain_attend, "logprobs": _plain_logprobs, "grad": _plain_grad}


# -------------------------------------------------------------------------------------- work
def work(case):
    size = {"f32": 4.0, "f16": 2.0, "bf16": 2.0}
    if case["kind"] == "plan":
        rows = sum(_spread(case["envs"], case["new_min"], case["new_max"]))
        fresh = rows / case["page"]
        return {"bytes": 4.0 * (4 * case["envs"] + 3 * rows + 2 * fresh), "flops": 8.0 * rows}
    if case["kind"] == "append":
        rows = sum(_spread(case["envs"], case["new_min"], case["new_max"]))
        H, Hk, hd = case["q_heads"], case["kv_heads"], case["head"]
        end = (case["ctx"] + 22 if case["ctx"] else 0) + case["new_max"]
        moved = (2 * H + 2 * Hk) * hd * size[case["act"]] + 2 * Hk * hd * size[case["cache"]] + 8
        turn = 8.0 * case["rope"] / 2 * min(end, rows)  # the rotations of the positions that occur
        return {"bytes": rows * moved + turn, "flops": rows * (H + Hk) * hd * (7.0 if case["norm"] else 3.0)}
    if case["kind"] == "attend":
        n = float(sum(_spread(case["envs"], case["ctx_min"], case["ctx_max"])))
        H, hd = case["q_heads"], case["head"]
        rows = case["envs"] * H * (2.0 * hd * size[case["act"]] + 4)
        return {"bytes": 2.0 * n * case["kv_heads"] * hd * size[case["cache"]] + rows + 4.0 * n / case["page"], "flops": 4.0 * n * H * hd}
    n = float(case["rows"]) * case["vocab"]
    if case["kind"] == "grad":
        return {"bytes": 2.0 * n * size[case["act"]] + 20.0 * case["rows"], "flops": 10.0 * n}
    return {"bytes": n * size[case["act"]] + case["rows"] * (16.0 + 8 * case["top"]), "flops": 8.0 * n}


# ------------------------------------------------------------------------------------- exact
def exact(case, seed):
    if case["kind"] == "plan":
        return None  # whole numbers only
    if case["kind"] == "append":
        s = _append_inputs(case, seed)
        H, Hk, hd, half = case["q_heads"], case["kv_heads"], case["head"], case["rope"] // 2
        x = s["qkv"].to(F64).view(s["rows"], H + 2 * Hk, hd)
        cs = s["rope"].to(F64)[s["pos"].long()]
        turn = torch.complex(cs[..., 0], cs[..., 1])[:, None]

        def turned(y, gain):
            if gain is not None:
                y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + EPS) * gain.to(F64)
            pairs = y[..., :2 * half]
            pairs = pairs.unflatten(-1, (2, half)).transpose(-1, -2) if case["layout"] == "half" else pairs.unflatten(-1, (half, 2))
            pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
            pairs = pairs.transpose(-1, -2).flatten(-2) if case["layout"] == "half" else pairs.flatten(-2)
            return torch.cat([pairs, y[..., 2 * half:]], -1)

        page, off = s["slot"].long() // case["page"], s["slot"].long() % case["page"]
        k, v = s["k_cache"].to(F64), s["v_cache"].to(F64)
        k[page, :, off] = turned(x[:, H:H + Hk], s["k_gain"])
        v[page, :, off] = x[:, H + Hk:].clone()
        return {"q": turned(x[:, :H], s["q_gain"]), "k_cache": k, "v_cache": v}
    if case["kind"] == "attend":
        s = _attend_inputs(case, seed)
        H, Hk, hd, ps = case["q_heads"], case["kv_heads"], case["head"], case["page"]
        out = torch.zeros(case["envs"], H, hd, dtype=F64, device=DEV)
        lse = torch.full((case["envs"], H), -math.inf, dtype=F64, device=DEV)
        for b, n in enumerate(s["lengths"]):
            if n == 0:
                continue
            t = torch.arange(n, device=DEV)
            page = s["table"][b].long()[t // ps]
            k, v = (x[page, :, t % ps].to(F64) for x in (s["k_cache"], s["v_cache"]))  # [n, Hk, hd]
            score = torch.einsum("hgd,nhd->hgn", s["q"][b].to(F64).view(Hk, H // Hk, hd), k) / math.sqrt(hd)
            lse[b] = torch.logsumexp(score, -1).view(H)
            out[b] = torch.einsum("hgn,nhd->hgd", torch.softmax(score, -1), v).reshape(H, hd)
        return {"out": out, "lse": lse}
    s = _logits_inputs(case, seed)
    T = case["temperature"]
    parts = []
    for x, token, *g in zip(*(t.split(512) for t in [s["logits"], s["token"].long()] +
                              ([s["g_logprob"], s["g_entropy"]] if case["kind"] == "grad" else []))):
        lp = torch.log_softmax(x.to(F64) / T, -1)
        h = torch.special.entr(lp.exp()).sum(-1)
        rows = torch.arange(len(token), device=DEV)
        kept = token >= 0
        if case["kind"] == "grad":
            p = lp.exp()
            d = -(g[0].to(F64)[:, None] + g[1].to(F64)[:, None] * (torch.where(p > 0, lp, 0.0) + h[:, None])) * p
            d[rows, token.clamp(min=0)] += g[0].to(F64)
            parts.append([torch.where(kept[:, None], d / T, 0.0)])
            continue
        best = torch.sort(x.to(F64) + 0.0, dim=-1, descending=True, stable=True).indices[:, :case["top"]]
        parts.append([torch.where(kept, lp[rows, token.clamp(min=0)], 0.0), h, torch.logsumexp(x.to(F64) / T, -1), lp.gather(1, best)])
    parts = [torch.cat(p) for p in zip(*parts)]
    if case["kind"] == "grad":
        return {"d_logits": parts[0]}
    return {"logprob": parts[0], "entropy": parts[1], "lse": parts[2], "top_id": None, "top_logprob": parts[3]}
