"""A token policy rolled out over paged contexts, and one step of its learning phase.

Environments of uneven prefixes share one pool of cache pages.  Every turn appends a chunk to each context and then
generates a few tokens greedily; one environment's episode ends on the way, and its pages serve the others.
Afterwards the generated tokens' log-probs go through the clipped objective, and its gradient back to the logits.

    python -m examples.paged_rollout

The decoder is the smallest shape of this repository's workloads with shared key-value heads and norms of queries
and keys; its projections run on the library's fp16 tensor-core GEMM, its contexts on the paged operators.
"""
from __future__ import annotations

import torch

from paper_2505_18719_gb300 import paged as P
from paper_2505_18719_gb300 import vla as V


class PagedDecoder:
    """Two layers of a Llama-style decoder: d 256, 4 query heads and 2 key-value heads of 64, 32064 ids."""

    def __init__(self, n_env=6, layers=2, d=256, heads=4, kv_heads=2, hd=64, ffn=688, vocab=32064, n_pages=64, page_size=16,
                 max_positions=512, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        w = lambda *s: torch.empty(*s, dtype=torch.float16, device="cuda").normal_(0, s[-1] ** -0.5, generator=g)  # noqa: E731
        gain = lambda n: (1 + 0.1 * torch.randn(n, generator=g, device="cuda")).to(torch.bfloat16)  # noqa: E731
        self.d, self.heads, self.kv_heads, self.hd, self.vocab = d, heads, kv_heads, hd, vocab
        self.embed = torch.randn(vocab, d, generator=g, device="cuda")
        self.layers = [{"norm": gain(d), "qkv": w((heads + 2 * kv_heads) * hd, d), "q_gain": gain(hd), "k_gain": gain(hd), "o": w(d, heads * hd),
                        "ffn_norm": gain(d), "gate_up": w(2 * ffn, d), "down": w(d, ffn)} for _ in range(layers)]
        self.final_norm, self.head = gain(d), w(vocab, d)
        self.rope = P.rope_table(max_positions, hd)
        self.cache = P.PagedCache(n_env, n_pages, page_size, layers, kv_heads, hd, max_positions)

    def _stream(self):
        return torch.cuda.current_stream().cuda_stream

    def _norm(self, h, gain):
        """RMSNorm as the fp16 pair (high, low) that a projection reads."""
        pair = torch.empty(2, *h.shape, dtype=torch.float16, device="cuda")
        P._ok(V.vla_op_rmsnorm(h.data_ptr(), h.stride(0), h.shape[0], h.shape[1], gain.data_ptr(), 1e-6, pair[0].data_ptr(),
                               pair[1].data_ptr(), True, self._stream()))
        return pair

    def _project(self, pair, weight):
        n, k = weight.shape
        out = torch.empty(pair.shape[1], n, dtype=torch.float32, device="cuda")
        P._ok(V.vla_op_gemm_f16(pair[0].data_ptr(), pair[1].data_ptr(), k, weight.data_ptr(), k, out.data_ptr(), n, out.shape[0], n, k,
                                128, 1, 0, self._stream()))
        return out

    @staticmethod
    def _pair(x):
        hi = x.to(torch.float16)
        return torch.stack([hi, (x - hi.float()).to(torch.float16)])

    def step(self, h, new_len, release=None):
        """Appends the rows h (f32 [rows, d]), new_len of them to each context; returns the final states [rows, d]."""
        rows = self.cache.plan(new_len, h.shape[0], release)
        h = h.clone()
        q_end, k_end = self.heads * self.hd, (self.heads + self.kv_heads) * self.hd
        for i, w in enumerate(self.layers):
            qkv = self._project(self._norm(h, w["norm"]), w["qkv"])
            q = self.cache.append(i, qkv[:, :q_end], qkv[:, q_end:k_end], qkv[:, k_end:], rows, self.rope, q_gain=w["q_gain"],
                                  k_gain=w["k_gain"])
            out = self.cache.attend(i, q, rows)
            h += self._project(self._pair(out.view(h.shape[0], -1)), w["o"])
            gate, up = self._project(self._norm(h, w["ffn_norm"]), w["gate_up"]).chunk(2, -1)
            h += self._project(self._pair(torch.nn.functional.silu(gate) * up), w["down"])
        return h, rows

    def logits(self, h):
        return self._project(self._norm(h.contiguous(), self.final_norm), self.head)


def rollout(policy: PagedDecoder, turns=3, actions=4, ends=((1, 2),), seed=1):
    """Per turn: the ids fed to each environment, the tokens it generated, their log-probs and logits."""
    g = torch.Generator().manual_seed(seed)
    n_env = policy.cache.n_env
    record = []
    for turn in range(turns):
        release = torch.zeros(n_env, dtype=torch.int32)
        for t, env in ends:
            release[env] = int(t == turn)
        lengths = torch.randint(3, 40, (n_env,), generator=g).to(torch.int32)
        ids = [torch.randint(0, policy.vocab, (int(n),), generator=g) for n in lengths]
        h, rows = policy.step(policy.embed[torch.cat(ids).cuda()], lengths.cuda(), release.cuda())
        h = h[rows.start[1:].long() - 1]  # each environment's last row
        tokens, logprobs, logits = [], [], []
        for a in range(actions):
            z = policy.logits(h)
            none = torch.full((n_env,), -1, dtype=torch.int32, device="cuda")
            best = P.token_logprobs(z, none, top_k=1)
            tokens.append(best.top_ids[:, 0].contiguous())
            logprobs.append(best.top_logprobs[:, 0])
            logits.append(z)
            if a + 1 < actions:
                h, _ = policy.step(policy.embed[tokens[-1].long()], torch.ones(n_env, dtype=torch.int32, device="cuda"))
        policy.cache.check()
        record.append({"ids": ids, "release": release, "tokens": torch.stack(tokens, 1), "logprobs": torch.stack(logprobs, 1),
                       "logits": torch.stack(logits, 1)})
    return record


def learning_step(record, advantages, eps=0.2, bonus=0.01):
    """The clipped objective of the generated tokens (with an entropy bonus) and its gradient at their logits."""
    logits = torch.cat([r["logits"] for r in record]).detach().requires_grad_()  # [samples, actions, vocab]
    tokens = torch.cat([r["tokens"] for r in record])
    old = torch.cat([r["logprobs"] for r in record])
    now = P.token_logprobs(logits.view(-1, logits.shape[-1]), tokens.reshape(-1))
    ratio = torch.exp(now.logprob.view_as(old).sum(1) - old.sum(1))
    objective = torch.minimum(ratio * advantages, ratio.clamp(1 - eps, 1 + eps) * advantages).mean() + bonus * now.entropy.mean()
    objective.backward()
    return objective.detach(), logits.grad


if __name__ == "__main__":
    policy = PagedDecoder()
    record = rollout(policy)
    samples = sum(len(r["tokens"]) for r in record)
    objective, grad = learning_step(record, torch.linspace(-1, 1, samples, device="cuda"))
    print(f"{len(record)} turns, {policy.cache.n_env} environments, {policy.cache.free_pages()} of {policy.cache.n_pages} pages free")
    print(f"tokens of the last turn {record[-1]['tokens'].tolist()}")
    print(f"objective {objective.item():.4f}, gradient norm {grad.norm().item():.4f}")
