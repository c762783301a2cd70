"""The torch wrappers over the paged operators, and a rollout that uses them together, against the same decoder over
dense contexts in 64 bits."""
import pytest
import torch

from examples import paged_rollout as X
from paper_2505_18719_gb300 import paged as P
from paper_2505_18719_gb300 import vla as V

pytestmark = pytest.mark.gpu

F64 = torch.float64


def norm64(x, gain):
    return x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * gain.to(F64)


def dense_logits(policy, rows):
    """Logits after each of one context's rows ([n, d], embeddings), in 64 bits."""
    h, hd = rows.to(F64), policy.hd
    n = h.shape[0]
    cs = policy.rope[:n].to(F64)
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]

    def turned(x):
        a, b = x.chunk(2, -1)
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    for w in policy.layers:
        qkv = (norm64(h, w["norm"]) @ w["qkv"].to(F64).T).view(n, -1, hd)
        q, k, v = qkv.split([policy.heads, policy.kv_heads, policy.kv_heads], 1)
        q, k = turned(norm64(q, w["q_gain"])), turned(norm64(k, w["k_gain"]))
        k, v = (x.repeat_interleave(policy.heads // policy.kv_heads, 1) for x in (k, v))
        score = torch.einsum("qhd,khd->hqk", q, k) * hd ** -0.5
        score = score.masked_fill(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), float("-inf"))
        out = torch.einsum("hqk,khd->qhd", torch.softmax(score, -1), v).reshape(n, -1)
        h = h + out @ w["o"].to(F64).T
        gate, up = (norm64(h, w["ffn_norm"]) @ w["gate_up"].to(F64).T).chunk(2, -1)
        h = h + (torch.nn.functional.silu(gate) * up) @ w["down"].to(F64).T
    return norm64(h, policy.final_norm) @ policy.head.to(F64).T


def test_a_paged_rollout_equals_the_dense_decoder():
    policy = X.PagedDecoder(n_pages=56)  # fewer than all contexts would need without the pages given back
    record = X.rollout(policy)
    context = [[] for _ in range(policy.cache.n_env)]
    # the cache's 11 significant bits: keys and values off by 2^-11 of about 1 move a logit of about 1 (unit
    # variance) by as much, twice a layer; 32 times that for the largest of 2.3 million of them
    tol = 32 * 4 * 2.0 ** -12
    for r in record:
        for e in range(policy.cache.n_env):
            if r["release"][e]:
                context[e] = []
            start = len(context[e]) + len(r["ids"][e])
            context[e] += r["ids"][e].tolist() + r["tokens"][e].tolist()[:-1]
            z = dense_logits(policy, policy.embed[torch.tensor(context[e], device="cuda")])[start - 1:]
            assert float((r["logits"][e] - z).abs().max()) < tol, e
            lp = torch.log_softmax(r["logits"][e].to(F64), -1)
            assert torch.equal(r["logits"][e].argmax(-1).int(), r["tokens"][e])
            assert float((lp.gather(1, r["tokens"][e].long()[:, None])[:, 0] - r["logprobs"][e]).abs().max()) < 1e-5
    held = sum(-(-len(c) // policy.cache.page_size) for c in context)
    assert policy.cache.free_pages() == policy.cache.n_pages - held
    assert policy.cache.ctx.tolist() == [len(c) for c in context]


def test_learning_step_gradient_is_autograds():
    policy = X.PagedDecoder(vocab=1000)
    record = X.rollout(policy, turns=2)
    samples = sum(len(r["tokens"]) for r in record)
    adv = torch.linspace(-1, 1, samples, device="cuda")
    for r in record:  # an older policy's log-probs: some ratios are clipped
        r["logprobs"] = r["logprobs"] - 0.1 * torch.linspace(-1, 1, r["logprobs"].numel(), device="cuda").view_as(r["logprobs"])
    objective, grad = X.learning_step(record, adv)
    z = torch.cat([r["logits"] for r in record]).to(F64).requires_grad_()
    lp = torch.log_softmax(z, -1)
    old = torch.cat([r["logprobs"] for r in record]).to(F64)
    chosen = lp.gather(-1, torch.cat([r["tokens"] for r in record]).long()[..., None])[..., 0]
    ratio = torch.exp(chosen.sum(1) - old.sum(1))
    want = torch.minimum(ratio * adv, ratio.clamp(0.8, 1.2) * adv).mean() + 0.01 * -(lp.exp() * lp).sum(-1).mean()
    want.backward()
    assert abs(float(objective - want.detach())) < 1e-5
    # each weight's relative error is that of its exponent, about 20 of 2^-24, times the row's gradient
    assert float((grad - z.grad).abs().max()) < 64 * 2.0 ** -24 * float(z.grad.abs().max() + 1.0 / samples)


def test_a_captured_step_serves_growing_contexts():
    # the plan, the append and the attention of a decode step in one graph: replays extend the contexts, with padding rows
    g = torch.Generator(device="cuda").manual_seed(0)
    n_env, heads, hd = 5, 4, 64
    cache = P.PagedCache(n_env, 40, 16, 1, heads, hd, 128)
    rope = P.rope_table(128, hd)
    new_len = torch.ones(n_env, dtype=torch.int32, device="cuda")
    qkv = torch.empty(n_env + 2, 3 * heads * hd, device="cuda")
    q, k, v = qkv.split(heads * hd, 1)

    def step():
        rows = cache.plan(new_len, n_env + 2)
        return rows, cache.attend(0, cache.append(0, q, k, v, rows, rope), rows)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        qkv.normal_(generator=g)
        step()
        cache.ctx.zero_()
        cache.n_free.fill_(40)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rows, out = step()
    fed = []
    for t in range(40):
        qkv.normal_(generator=g)
        new_len.fill_(1)
        new_len[3] = t % 2  # grows every other step
        fed.append((qkv.clone(), new_len.tolist()))
        graph.replay()
    torch.cuda.synchronize()
    assert V.vla_op_read_status(0) == (0, 0)
    assert cache.ctx.tolist() == [40, 40, 40, 20, 40]
    # the last step's rows over everything fed, in 64 bits
    cs = rope.to(F64)
    order = [e for e in range(n_env) for _ in range(fed[-1][1][e])]
    assert rows.env.tolist() == order + [-1] * (n_env + 2 - len(order))
    for r, e in enumerate(order):
        keys, values = [], []
        for x, n in fed:
            at = sum(n[:e])
            if n[e]:
                row = x[at].to(F64).view(3, heads, hd)
                c, s = cs[len(keys), :, 0], cs[len(keys), :, 1]
                a, b = row[1].chunk(2, -1)
                keys.append(torch.cat([a * c - b * s, b * c + a * s], -1))
                values.append(row[2])
        a, b = fed[-1][0][r].to(F64).view(3, heads, hd)[0].chunk(2, -1)
        query = torch.cat([a * c - b * s, b * c + a * s], -1)
        p = torch.softmax(torch.einsum("hd,nhd->hn", query, torch.stack(keys)) * hd ** -0.5, -1)
        want = torch.einsum("hn,nhd->hd", p, torch.stack(values))
        # keys and values of 11 significant bits, scores of up to about 4
        assert float((out[r] - want).abs().max()) < 16 * 2.0 ** -11
    assert bool((out[len(order):] == 0).all())


def test_wrappers_refuse_what_does_not_fit():
    cache = P.PagedCache(2, 4, 16, 1, 2, 64, 64)
    good = torch.ones(2, dtype=torch.int32, device="cuda")
    for bad in (good.long(), good[:1], torch.ones(2, 2, dtype=torch.int32, device="cuda")[:, 0]):
        with pytest.raises(ValueError):
            cache.plan(bad, 2)
    rows = cache.plan(good, 2)
    x = torch.zeros(2, 3, 2, 64, device="cuda")
    q, k, v = x.unbind(1)
    with pytest.raises(ValueError):
        cache.append(0, q[..., ::2], k, v, rows)
    with pytest.raises(ValueError):
        cache.append(0, q, k.half(), v, rows)
    with pytest.raises(ValueError):
        cache.append(0, q[:1], k[:1], v[:1], rows)
    with pytest.raises(ValueError):
        cache.append(0, q, k, v, rows, q_gain=torch.ones(64, device="cuda"))
    with pytest.raises(ValueError):
        cache.attend(0, q[:1], rows)
    with pytest.raises(V.VlaError):
        cache.attend(0, q.to(torch.bfloat16), rows)  # bf16 queries over an fp16 cache
    with pytest.raises(ValueError):
        P.token_logprobs(torch.zeros(2, 8, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(V.VlaError):
        P.PagedCache(2, 4, 16, 1, 2, 96, 64)
    cache.plan(torch.full((2,), 60, dtype=torch.int32, device="cuda"), 200)  # more than the pool holds
    with pytest.raises(V.VlaError):
        cache.check()
    cache.check()  # the status was cleared


def test_logprob_gradients_of_rows_without_tokens_and_unused_outputs():
    g = torch.Generator(device="cuda").manual_seed(3)
    z = torch.randn(6, 50, generator=g, device="cuda").requires_grad_()
    tokens = torch.tensor([3, -1, 49, 0, -1, 7], dtype=torch.int32, device="cuda")
    out = P.token_logprobs(z, tokens, temperature=1.5, top_k=3)
    out.logprob.sum().backward()
    want = torch.zeros(6, 50, dtype=F64, device="cuda")
    p = torch.softmax(z.detach().to(F64) / 1.5, -1)
    for r, t in enumerate(tokens.tolist()):
        if t >= 0:
            want[r] = -p[r]
            want[r, t] += 1
    assert float((z.grad - want / 1.5).abs().max()) < 64 * 2.0 ** -24
    assert torch.equal(out.top_ids.long(), torch.topk(z, 3).indices)
    z.grad = None
    P.token_logprobs(z, tokens).entropy[0].backward()
    lp = torch.log_softmax(z.detach().to(F64), -1)
    h = -(lp.exp() * lp).sum(-1, keepdim=True)
    assert float((z.grad[0] + (lp.exp() * (lp + h))[0]).abs().max()) < 64 * 2.0 ** -24
    assert bool((z.grad[1:] == 0).all())


def test_logprob_and_entropy_gradients_together():
    # both gradients arrive as broadcast scalars; a lone row's stride is arbitrary; no second derivatives
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(7, 90, generator=g, device="cuda")
    tokens = torch.arange(7, dtype=torch.int32, device="cuda") * 11
    for rows in (slice(None), slice(2, 3)):
        z = x[rows].clone().as_strided(x[rows].shape, (90 if rows == slice(None) else 1, 1)).requires_grad_()
        out = P.token_logprobs(z, tokens[rows])
        (2.0 * out.logprob.sum() - 0.25 * out.entropy.sum()).backward()
        z64 = x[rows].to(F64).requires_grad_()
        lp = torch.log_softmax(z64, -1)
        (2.0 * lp.gather(1, tokens[rows].long()[:, None]).sum() + 0.25 * (lp.exp() * lp).sum()).backward()
        assert float((z.grad - z64.grad).abs().max()) < 64 * 2.0 ** -24 * 2
    z = x.clone().requires_grad_()
    first, = torch.autograd.grad(P.token_logprobs(z, tokens).logprob.sum(), z, create_graph=True)
    with pytest.raises(RuntimeError):
        first.square().sum().backward()


def test_wrappers_refuse_tensors_elsewhere_and_other_types():
    cache = P.PagedCache(2, 4, 16, 1, 2, 64, 64)
    new_len = torch.ones(2, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        cache.plan(new_len.cpu(), 2)
    rows = cache.plan(new_len, 2)
    q, k, v = torch.zeros(2, 3, 2, 64, device="cuda").unbind(1)
    for bad in (q.cpu(), q.double()):
        with pytest.raises(ValueError):
            cache.append(0, bad, k.to(bad.dtype), v.to(bad.dtype), rows)
        with pytest.raises(ValueError):
            cache.attend(0, bad, rows)
    for rope in (torch.zeros(64, 32, 2), torch.zeros(64, 64, device="cuda"), torch.zeros(64, 32, 2, device="cuda", dtype=F64)):
        with pytest.raises(ValueError):
            cache.append(0, q, k, v, rows, rope)
    with pytest.raises(ValueError):
        P.rope_table(8, 64, device="cpu")
    tokens = torch.zeros(2, dtype=torch.int32, device="cuda")
    for z, t in ((torch.zeros(2, 8), tokens.cpu()), (torch.zeros(2, 8, device="cuda"), tokens.cpu()), (torch.zeros(2, 8, device="cuda", dtype=F64), tokens)):
        with pytest.raises(ValueError):
            P.token_logprobs(z, t)
    # one row, one head: their strides do not count
    one = P.PagedCache(1, 1, 16, 1, 1, 64, 16)
    x = torch.randn(64, device="cuda")
    lone = x.as_strided((1, 1, 64), (3, 5, 1))
    rows = one.plan(torch.ones(1, dtype=torch.int32, device="cuda"), 1)
    out = one.attend(0, one.append(0, lone, lone, lone, rows), rows)
    assert float((out.view(64) - x).abs().max()) <= 2.0 ** -11 * float(x.abs().max()) + 2.0 ** -20
    one.check()


def test_a_launch_that_fails_is_reported_and_leaves_the_next_call_sound():
    out_of_resources = 701
    cache = P.PagedCache(2, 4, 16, 1, 2, 64, 64)
    new_len = torch.ones(2, dtype=torch.int32, device="cuda")
    q, k, v = torch.randn(2, 3, 2, 64, device="cuda").unbind(1)
    z = torch.randn(2, 40, device="cuda", requires_grad=True)
    tokens = torch.zeros(2, dtype=torch.int32, device="cuda")

    def failing(call):
        assert V.vla_test_inject_launch_error(1, out_of_resources) == 0
        try:
            with pytest.raises(V.VlaError) as e:
                call()
            assert e.value.code == V.VLA_ERR_CUDA and "701" in str(e.value)
        finally:
            V.vla_test_inject_launch_error(0, 0)
        return call()

    failing(lambda: P.rope_table(16, 64))
    rows = failing(lambda: cache.plan(new_len, 2))
    turned = failing(lambda: cache.append(0, q, k, v, rows))
    out = failing(lambda: cache.attend(0, turned, rows))
    lp = failing(lambda: P.token_logprobs(z, tokens, top_k=3)).logprob
    failing(lambda: torch.autograd.grad(lp.sum(), z, retain_graph=True))
    assert cache.ctx.tolist() == [1, 1] and cache.free_pages() == 2
    assert float((out - v).abs().max()) <= 2.0 ** -11 * float(v.abs().max()) + 2.0 ** -20  # one position: its values
    cache.check()
