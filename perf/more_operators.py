"""The operators of a policy's learning pass over whole sequences, as cases to time and to compare.

A rollout reads its contexts one token at a time; the learning phase sends whole sequences of different
lengths through the same layers at once, packed one behind the other, and the gradient back.  Two parts
of a layer are no plain matrix products there: the causal attention of the packed sequences, with grouped
heads ("prompt", and "prompt_grad" for its gradient), and what lies between two blocks: the norm of a block's
output, its gate and scale, the sum with the residual stream and the norm before the next block ("norm", and
"norm_grad").  The sizes are those of this repository's workloads (4 to 64 environments, prefixes of about 80
and 300 rows, 448 rows of action tokens, heads of 64 and 128, a stream of 4096 channels) and generic ones where the
workloads have none (shared key-value heads, uneven and long sequences, odd widths, gates of each row).

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


# ------------------------------------------------------------------------------------- cases
def _prompt(name, kind, seqs, len_min, len_max, q_heads, kv_heads, head, act, pad):
    """`seqs` sequences of len_min to len_max rows, `pad` rows behind the last that belong to none."""
    return {"name": name, "kind": kind, "seqs": seqs, "len_min": len_min, "len_max": len_max, "q_heads": q_heads,
            "kv_heads": kv_heads, "head": head, "act": act, "pad": pad}


def _norm(name, kind, rows, dim, act, stream, post, gate, scale):
    """gate: "none", "channel" (one for all rows) or "row" (one for each)."""
    return {"name": name, "kind": kind, "rows": rows, "dim": dim, "act": act, "stream": stream, "post": post, "gate": gate,
            "scale": scale}


def listed():
    return [
        # the prefixes of the smallest shape: 4 environments, 4 heads of 64; latency
        _prompt("prompt_b4", "prompt", 4, 70, 80, 4, 4, 64, "f16", 0),
        # the prefixes of 64 environments on the 7B shape
        _prompt("prompt_b64", "prompt", 64, 272, 304, 32, 32, 128, "f16", 0),
        # trajectories of very different lengths with shared key-value heads, in a batch of fixed size
        _prompt("prompt_ragged", "prompt", 16, 1, 2048, 32, 8, 128, "bf16", 37),
        # one long document
        _prompt("prompt_long", "prompt", 1, 16384, 16384, 32, 8, 128, "bf16", 0),
        # the gradient of the smallest shape, with shared key-value heads; latency
        _prompt("prompt_grad_b4", "prompt_grad", 4, 70, 80, 4, 2, 64, "bf16", 0),
        # the gradient of one learning step over 64 samples of the 7B shape
        _prompt("prompt_grad_b64", "prompt_grad", 64, 272, 304, 32, 32, 128, "bf16", 0),
        # the gradient of a long document with shared key-value heads
        _prompt("prompt_grad_long", "prompt_grad", 1, 8192, 8192, 32, 8, 128, "bf16", 0),
        # between two blocks of a small batch: one token of each of 64 environments; latency
        _norm("norm_b64_step", "norm", 64, 4096, "f16", "f32", False, "none", 1.0),
        # between two blocks of the 64 prefixes, with a norm and a learned gate behind each block
        _norm("norm_b64", "norm", 18385, 4096, "bf16", "f32", True, "channel", 0.5),
        # the gradient over the 448 action tokens of 64 samples
        _norm("norm_grad_448", "norm_grad", 448, 4096, "bf16", "f32", False, "none", 1.0),
        # the gradient over 64 whole samples, with a norm and a learned gate behind each block
        _norm("norm_grad_b64", "norm_grad", 18385, 4096, "bf16", "f32", True, "channel", 0.5),
        # the gradient of an odd width with a gate of each row, stream and blocks in 16 bits
        _norm("norm_grad_odd", "norm_grad", 2311, 1155, "bf16", "bf16", True, "row", 1.0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "prompt_grad", "prompt_grad", "norm", "norm_grad"])
    if kind in ("prompt", "prompt_grad"):
        q_heads, kv_heads, head = rng.choice([(4, 4, 64), (4, 2, 64), (10, 10, 64), (16, 4, 64), (12, 12, 128), (20, 20, 128), (32, 32, 128),
                                              (32, 8, 128), (28, 4, 128), (8, 1, 128), (6, 2, 64)])
        seqs = _log_int(rng, 1, 128)
        # scores of all sequences, padded to the longest: at most those of the longest listed case
        most = 32.0 * (16384 if kind == "prompt" else 8192) ** 2
        # (a lone row attends to itself alone: its queries and keys have no gradient but noise)
        longest = _log_int(rng, 1 if kind == "prompt" else 2, max(2, min(16384, int(math.sqrt(most / (seqs * q_heads))), 40000 // seqs)))
        shortest = rng.choice([longest, max(1, longest * 3 // 4), 1, 0])
        c = _prompt("", kind, seqs, shortest, longest, q_heads, kv_heads, head, rng.choice(["f16", "bf16"]), rng.choice([0, 0, rng.randint(1, 200)]))
    else:
        dim = rng.choice([_log_int(rng, 64, 8192), 8 * _log_int(rng, 8, 1024)])
        act, stream = rng.choice([("f16", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "f32")])
        c = _norm("", kind, _log_int(rng, 1, max(1, min(30000, int(5e7 / dim)))), dim, act, stream, rng.random() < 0.5,
                  rng.choice(["none", "channel", "row"]), rng.choice([1.0, 0.5, 0.22]))
    del c["name"]
    return c


# ------------------------------------------------------------------------------------ inputs
def _lengths(case):
    """The lengths of a case's sequences, spread over their range; the first is the longest, the second the shortest."""
    lo, hi = case["len_min"], case["len_max"]
    return [hi if b == 0 else lo if b == 1 else lo + int((hi - lo + 1) * ((b * 0.6180339887 + 0.31) % 1.0)) for b in range(case["seqs"])]


def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _normal(g, shape, dtype, std=1.0):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=g)


def _prompt_inputs(case, seed):
    g = _generator(seed)
    H, Hk, hd, dt = case["q_heads"], case["kv_heads"], case["head"], DTYPE[case["act"]]
    lengths = _lengths(case)
    rows = sum(lengths) + case["pad"]
    start = [0]
    for n in lengths:
        start.append(start[-1] + n)
    qkv = _normal(g, (rows, (H + 2 * Hk) * hd), dt)  # the rows of one q|k|v projection
    s = {"qkv": qkv, "start": torch.tensor(start, dtype=torch.int32, device=DEV), "rows": rows, "longest": max(1, max(lengths)),
         "lengths": lengths, "scale": 1.0 / math.sqrt(hd), "out": torch.empty(rows, H, hd, dtype=dt, device=DEV),
         "lse": torch.empty(rows, H, dtype=torch.float32, device=DEV)}
    if case["kind"] == "prompt_grad":  # what the pass before left, and the gradient that comes in
        s["case"] = case
        kept = _plain_prompt(s)
        s["out"], s["lse"] = kept["out"].contiguous(), kept["lse"].contiguous()
        s["d_out"] = _normal(g, (rows, H, hd), dt)
        s["d_qkv"] = torch.empty_like(qkv)
    return s


def _norm_inputs(case, seed):
    g = _generator(seed)
    n, d, act, stream = case["rows"], case["dim"], DTYPE[case["act"]], DTYPE[case["stream"]]
    gain = lambda: (1.0 + 0.2 * _normal(g, (d,), torch.float32)).to(torch.bfloat16)  # noqa: E731
    s = {"y": _normal(g, (n, d), act, 0.7), "h": _normal(g, (n, d), stream, 2.0), "pre_gain": gain(),
         "post_gain": gain() if case["post"] else None,
         "gate": None if case["gate"] == "none" else _normal(g, (n, d) if case["gate"] == "row" else (d,), act, 0.5)}
    if case["kind"] == "norm":
        s.update(h_out=torch.empty_like(s["h"]), x=torch.empty_like(s["y"]), rstd=torch.empty(n, 2, dtype=torch.float32, device=DEV))
    else:  # `h` is the stream behind the sum, as the pass before left it
        rstd = [torch.rsqrt(t.float().square().mean(-1) + EPS) for t in (s["y"], s["h"])]
        s["rstd"] = torch.stack(rstd, -1).contiguous()
        s.update(d_x=_normal(g, (n, d), act), d_h_out=_normal(g, (n, d), stream), d_h=torch.empty_like(s["h"]), d_y=torch.empty_like(s["y"]))
        f = lambda: torch.empty(d, dtype=torch.float32, device=DEV)  # noqa: E731
        s["d_pre_gain"], s["d_post_gain"] = f(), f() if case["post"] else None
        s["d_gate"] = None if case["gate"] == "none" else torch.empty_like(s["gate"]) if case["gate"] == "row" else f()
    return s


def prepare(case, seed):
    s = (_prompt_inputs if case["kind"] in ("prompt", "prompt_grad") else _norm_inputs)(case, seed)
    s["case"] = case
    s["stream"] = torch.cuda.current_stream().cuda_stream
    if own and case["kind"] in ("prompt_grad", "norm_grad"):  # the workspace that a learning program keeps
        from paper_2505_18719_gb300 import vla as V
        if case["kind"] == "prompt_grad":
            size = V.vla_prompt_attn_grad_workspace_bytes(s["rows"], case["q_heads"], case["kv_heads"], case["head"])
        else:
            size = V.vla_block_norm_grad_workspace_bytes(case["rows"], case["dim"])
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device=DEV)
    return s


# --------------------------------------------------------------------------------------- run
def run(state):
    return (_own if own else _plain)[state["case"]["kind"]](state)


def _ptr(t):
    return t.data_ptr() if t is not None else 0


def _ok(V, rc):
    if rc != V.VLA_OK:
        raise V.VlaError(rc, V.vla_last_error())


def _own_prompt(s):
    from paper_2505_18719_gb300 import vla as V
    c, qkv = s["case"], s["qkv"]
    H, Hk, hd = c["q_heads"], c["kv_heads"], c["head"]
    at, size, ld = qkv.data_ptr(), qkv.element_size(), qkv.stride(0)
    _ok(V, V.vla_prompt_attn(at, ld, at + H * hd * size, ld, at + (H + Hk) * hd * size, ld, CODE[c["act"]], s["rows"], H, Hk, hd,
                             _ptr(s["start"]), c["seqs"], s["scale"], _ptr(s["out"]), H * hd, _ptr(s["lse"]), s["stream"]))
    return {"out": s["out"], "lse": s["lse"]}


def _own_prompt_grad(s):
    from paper_2505_18719_gb300 import vla as V
    c, qkv, d = s["case"], s["qkv"], s["d_qkv"]
    H, Hk, hd = c["q_heads"], c["kv_heads"], c["head"]
    size, ld = qkv.element_size(), qkv.stride(0)
    k, v = H * hd * size, (H + Hk) * hd * size
    _ok(V, V.vla_prompt_attn_grad(_ptr(qkv), ld, _ptr(qkv) + k, ld, _ptr(qkv) + v, ld, CODE[c["act"]], s["rows"], H, Hk, hd,
                                  _ptr(s["start"]), c["seqs"], s["scale"], _ptr(s["out"]), H * hd, _ptr(s["lse"]), _ptr(s["d_out"]), H * hd,
                                  _ptr(d), ld, _ptr(d) + k, ld, _ptr(d) + v, ld, _ptr(s["workspace"]), s["workspace"].numel(), s["stream"]))
    return {"dq": d[:, :H * hd], "dk": d[:, H * hd:(H + Hk) * hd], "dv": d[:, (H + Hk) * hd:]}


def _own_norm(s):
    from paper_2505_18719_gb300 import vla as V
    c, d = s["case"], s["case"]["dim"]
    _ok(V, V.vla_block_norm(_ptr(s["y"]), d, CODE[c["act"]], _ptr(s["h"]), d, CODE[c["stream"]], c["rows"], d, _ptr(s["post_gain"]),
                            _ptr(s["gate"]), d if c["gate"] == "row" else 0, c["scale"], _ptr(s["pre_gain"]), EPS, _ptr(s["h_out"]), d,
                            _ptr(s["x"]), d, _ptr(s["rstd"]), s["stream"]))
    return {"h": s["h_out"], "x": s["x"]}


def _own_norm_grad(s):
    from paper_2505_18719_gb300 import vla as V
    c, d = s["case"], s["case"]["dim"]
    ldg = d if c["gate"] == "row" else 0
    _ok(V, V.vla_block_norm_grad(_ptr(s["y"]), d, CODE[c["act"]], _ptr(s["h"]), d, CODE[c["stream"]], c["rows"], d, _ptr(s["post_gain"]),
                                 _ptr(s["gate"]), ldg, c["scale"], _ptr(s["pre_gain"]), _ptr(s["rstd"]), _ptr(s["d_x"]), d,
                                 _ptr(s["d_h_out"]), d, _ptr(s["d_h"]), d, _ptr(s["d_y"]), d, _ptr(s["d_gate"]), ldg,
                                 _ptr(s["d_post_gain"]), _ptr(s["d_pre_gain"]), _ptr(s["workspace"]), s["workspace"].numel(), s["stream"]))
    return {n: s[n] for n in ("d_h", "d_y", "d_pre_gain", "d_post_gain", "d_gate") if s[n] is not None}


def _places(s):
    """(packed row of each sequence and position, whether there is one; sequence and position of each packed row, whether it has one)."""
    start = s["start"].long()
    t = torch.arange(s["longest"], device=DEV)
    row = start[:-1, None] + t
    r = torch.arange(s["rows"], device=DEV)
    seq = torch.searchsorted(start[1:], r, right=True).clamp(max=start.numel() - 2)
    return row.clamp(max=max(0, s["rows"] - 1)), row < start[1:, None], seq, (r - start[seq]).clamp(max=s["longest"] - 1), r < start[-1]


def _heads(s):
    """Queries [sequence, key head, query head of it x position, channel], keys and values [sequence, key head, position, channel] in
    32 bits, sequences padded to the longest; what each position sees [sequence, 1, 1, position, position]; the places of the rows."""
    c = s["case"]
    H, Hk, hd, L = c["q_heads"], c["kv_heads"], c["head"], s["longest"]
    places = _places(s)
    x = s["qkv"].view(s["rows"], H + 2 * Hk, hd)[places[0]]
    q, k, v = x[:, :, :H], x[:, :, H:H + Hk], x[:, :, H + Hk:]
    t = torch.arange(L, device=DEV)
    seen = ((t <= t[:, None]) & places[1][:, None, :] & places[1][:, :, None])[:, None, None]
    return _grouped(s, q), k.transpose(1, 2).float(), v.transpose(1, 2).float(), seen, places


def _grouped(s, x):
    """[sequence, position, query head, channel] -> [sequence, key head, query head of it x position, channel] in 32 bits."""
    c = s["case"]
    return x.transpose(1, 2).float().reshape(x.shape[0], c["kv_heads"], -1, c["head"])


def _plain_prompt(s):
    c = s["case"]
    H, Hk, hd, L = c["q_heads"], c["kv_heads"], c["head"], s["longest"]
    if s["rows"] == 0:
        return {"out": s["out"], "lse": s["lse"]}
    q, k, v, seen, (_, _, seq, pos, live) = _heads(s)
    score = (q @ k.transpose(2, 3) * s["scale"]).view(c["seqs"], Hk, H // Hk, L, L)
    score = torch.where(seen, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    out = (p.view(c["seqs"], Hk, -1, L) @ v).view(c["seqs"], H, L, hd) / total.clamp(min=1e-30).view(c["seqs"], H, L, 1)
    lse = (top + torch.log(total)).view(c["seqs"], H, L)
    return {"out": torch.where(live[:, None, None], out[seq, :, pos], 0.0).to(DTYPE[c["act"]]),
            "lse": torch.where(live[:, None], lse[seq, :, pos], -math.inf)}


def _plain_prompt_grad(s):
    c = s["case"]
    H, Hk, hd, L = c["q_heads"], c["kv_heads"], c["head"], s["longest"]
    if s["rows"] == 0:
        return {"dq": s["d_qkv"][:, :H * hd], "dk": s["d_qkv"][:, H * hd:(H + Hk) * hd], "dv": s["d_qkv"][:, (H + Hk) * hd:]}
    q, k, v, seen, (row, _, seq, pos, live) = _heads(s)
    d_out = _grouped(s, s["d_out"][row])
    delta = (s["d_out"].float() * s["out"].float()).sum(-1)[row].transpose(1, 2).reshape(c["seqs"], Hk, H // Hk, L, 1)
    lse = s["lse"][row].transpose(1, 2).reshape(c["seqs"], Hk, H // Hk, L, 1)
    score = (q @ k.transpose(2, 3) * s["scale"]).view(c["seqs"], Hk, H // Hk, L, L)
    p = torch.where(seen, torch.exp(score - lse), 0.0)
    del score
    ds = (d_out @ v.transpose(2, 3)).view(c["seqs"], Hk, H // Hk, L, L)
    ds = torch.where(seen, p * (ds - delta), 0.0).view(c["seqs"], Hk, -1, L)
    p = p.view(c["seqs"], Hk, -1, L)
    dq = (ds @ k).view(c["seqs"], H, L, hd) * s["scale"]
    dk = ds.transpose(2, 3) @ q * s["scale"]
    dv = p.transpose(2, 3) @ d_out
    packed = lambda x: torch.where(live[:, None, None], x[seq, :, pos], 0.0).to(DTYPE[c["act"]]).flatten(1)  # noqa: E731
    return {"dq": packed(dq), "dk": packed(dk), "dv": packed(dv)}


def _plain_norm(s):
    c = s["case"]
    u = s["y"].float()
    if c["post"]:
        u = u * torch.rsqrt((u * u).mean(-1, keepdim=True) + EPS) * s["post_gain"].float()
    if s["gate"] is not None:
        u = u * s["gate"].float()
    h = s["h"].float() + c["scale"] * u
    x = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * s["pre_gain"].float()
    return {"h": h.to(s["h"].dtype), "x": x.to(s["y"].dtype)}


def _plain_norm_grad(s):
    c = s["case"]
    r_y, r_h = s["rstd"][:, :1], s["rstd"][:, 1:]
    n, d_x = s["h"].float() * r_h, s["d_x"].float()
    g = d_x * s["pre_gain"].float()
    d_h = s["d_h_out"].float() + r_h * (g - n * (g * n).mean(-1, keepdim=True))
    out = {"d_h": d_h.to(s["h"].dtype), "d_pre_gain": (d_x * n).sum(0)}
    u = m = s["y"].float()
    if c["post"]:
        m = m * r_y
        u = m * s["post_gain"].float()
    d_u = c["scale"] * d_h
    if s["gate"] is not None:
        d_gate = d_u * u
        out["d_gate"] = d_gate.to(s["gate"].dtype) if c["gate"] == "row" else d_gate.sum(0)
        d_u = d_u * s["gate"].float()
    if c["post"]:
        out["d_post_gain"] = (d_u * m).sum(0)
        d_m = d_u * s["post_gain"].float()
        d_u = r_y * (d_m - m * (d_m * m).mean(-1, keepdim=True))
    out["d_y"] = d_u.to(s["y"].dtype)
    return {k: out[k] for k in ("d_h", "d_y", "d_pre_gain", "d_post_gain", "d_gate") if k in out}


_own = {"prompt": _own_prompt, "prompt_grad": _own_prompt_grad, "norm": _own_norm, "norm_grad": _own_norm_grad}
_plain = {"prompt": _plain_prompt, "prompt_grad": _plain_prompt_grad, "norm": _plain_norm, "norm_grad": _plain_norm_grad}


# -------------------------------------------------------------------------------------- work
def work(case):
    size = {"f32": 4.0, "f16": 2.0, "bf16": 2.0}
    if case["kind"] in ("prompt", "prompt_grad"):
        lengths = _lengths(case)
        rows = float(sum(lengths))
        pairs = sum(n * (n + 1) / 2.0 for n in lengths) * case["q_heads"] * case["head"]
        q = rows * case["q_heads"] * case["head"] * size[case["act"]]
        kv = 2.0 * rows * case["kv_heads"] * case["head"] * size[case["act"]]
        lse = 4.0 * rows * case["q_heads"]
        if case["kind"] == "prompt":
            return {"bytes": 2 * q + kv + lse, "flops": 4.0 * pairs}
        return {"bytes": 4 * q + 2 * kv + lse, "flops": 10.0 * pairs}
    n, act, stream = float(case["rows"]) * case["dim"], size[case["act"]], size[case["stream"]]
    gate = n * act if case["gate"] == "row" else 0.0
    if case["kind"] == "norm":
        return {"bytes": n * (2 * act + 2 * stream) + gate, "flops": 8.0 * n}
    return {"bytes": n * (3 * act + 3 * stream) + 2 * gate, "flops": 20.0 * n}


# ------------------------------------------------------------------------------------- exact
def _exact_heads(case, s, fn):
    """fn(q, k, v, rows, query heads, key head) for each sequence and key head, all in 64 bits."""
    H, Hk, hd = case["q_heads"], case["kv_heads"], case["head"]
    x = s["qkv"].view(s["rows"], H + 2 * Hk, hd)
    at = 0
    for n in s["lengths"]:
        if n:
            for j in range(Hk):
                heads = slice(j * (H // Hk), (j + 1) * (H // Hk))
                fn(x[at:at + n, heads].to(F64), x[at:at + n, H + j].to(F64), x[at:at + n, H + Hk + j].to(F64), slice(at, at + n), heads, j)
        at += n


def _exact_prompt(case, seed):
    s = _prompt_inputs(case, seed)
    out = torch.zeros(s["rows"], case["q_heads"], case["head"], dtype=F64, device=DEV)
    lse = torch.full((s["rows"], case["q_heads"]), -math.inf, dtype=F64, device=DEV)

    def one(q, k, v, rows, heads, _):
        score = torch.einsum("nhd,md->hnm", q, k).div_(math.sqrt(case["head"]))
        score.masked_fill_(torch.ones(score.shape[1:], dtype=torch.bool, device=DEV).triu_(1), -math.inf)
        lse[rows, heads] = torch.logsumexp(score, -1).T
        out[rows, heads] = torch.einsum("hnm,md->nhd", torch.softmax(score, -1), v)

    _exact_heads(case, s, one)
    return {"out": out, "lse": lse}


def _exact_prompt_grad(case, seed):
    s = _prompt_inputs(case, seed)
    H, Hk, hd = case["q_heads"], case["kv_heads"], case["head"]
    dq = torch.zeros(s["rows"], H, hd, dtype=F64, device=DEV)
    dk, dv = (torch.zeros(s["rows"], Hk, hd, dtype=F64, device=DEV) for _ in range(2))

    def one(q, k, v, rows, heads, j):
        d_out = s["d_out"][rows, heads].to(F64)
        score = torch.einsum("nhd,md->hnm", q, k).div_(math.sqrt(hd))
        score.masked_fill_(torch.ones(score.shape[1:], dtype=torch.bool, device=DEV).triu_(1), -math.inf)
        p = torch.softmax(score, -1)
        del score
        dv[rows, j] = torch.einsum("hnm,nhd->md", p, d_out)
        d = torch.einsum("nhd,md->hnm", d_out, v)
        d = p * (d - (p * d).sum(-1, keepdim=True)) / math.sqrt(hd)
        dq[rows, heads] = torch.einsum("hnm,md->nhd", d, k)
        dk[rows, j] = torch.einsum("hnm,nhd->md", d, q)

    _exact_heads(case, s, one)
    return {"dq": dq.flatten(1), "dk": dk.flatten(1), "dv": dv.flatten(1)}


def _exact_norm(case, seed):
    s = _norm_inputs(case, seed)
    y, h = s["y"].to(F64), s["h"].to(F64)
    if case["post"]:
        y = y / (y.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * s["post_gain"].to(F64)
    h = h + case["scale"] * (y if s["gate"] is None else y * s["gate"].to(F64))
    return {"h": h, "x": h / (h.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * s["pre_gain"].to(F64)}


def _exact_norm_grad(case, seed):
    """By torch's differentiation of the definition in 64 bits: the block's output through the sum, and the stream behind it."""
    s = _norm_inputs(case, seed)
    leaf = lambda t: None if t is None else t.to(F64).requires_grad_()  # noqa: E731
    h, y, pre, post, gate = leaf(s["h"]), leaf(s["y"]), leaf(s["pre_gain"]), leaf(s["post_gain"]), leaf(s["gate"])
    with torch.enable_grad():
        x = h / (h.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * pre
        d_h, d_pre = torch.autograd.grad(x, [h, pre], s["d_x"].to(F64))
        d_h = d_h + s["d_h_out"].to(F64)
        u = y if post is None else y / (y.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * post
        u = case["scale"] * (u if gate is None else u * gate)
        names = [n for n, t in (("d_y", y), ("d_post_gain", post), ("d_gate", gate)) if t is not None]
        found = dict(zip(names, torch.autograd.grad(u, [t for t in (y, post, gate) if t is not None], d_h)))
    found.update(d_h=d_h, d_pre_gain=d_pre)
    return {k: found[k] for k in ("d_h", "d_y", "d_pre_gain", "d_post_gain", "d_gate") if k in found}


def exact(case, seed):
    return {"prompt": _exact_prompt, "prompt_grad": _exact_prompt_grad, "norm": _exact_norm, "norm_grad": _exact_norm_grad}[case["kind"]](case, seed)
