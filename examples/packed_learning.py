"""One learning step of a small decoder over whole sequences, packed one behind the other.

Sequences of uneven lengths, each a prefix and the tokens that a policy chose after it, go through the decoder at once; the
clipped objective of the chosen tokens' log-probs (with an entropy bonus) sends its gradient back through every layer to all
weights.  A batch of fixed size has rows behind its last sequence: they count for nothing.

    python -m examples.packed_learning

Norms, gates and residual sums between the blocks, the causal attention with shared key-value heads and the log-probs are the
library's operators with their gradients; the projections are torch's.
"""
from __future__ import annotations

import torch

from paper_2505_18719_gb300 import learn as L
from paper_2505_18719_gb300 import paged as P


class Decoder:
    """Two layers: d 256, 4 query heads and 2 key-value heads of 64, norms before and after each block, a learned gate, 997 ids."""

    def __init__(self, layers=2, d=256, heads=4, kv_heads=2, hd=64, ffn=512, vocab=997, max_positions=512, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        w = lambda *s: torch.empty(*s, device="cuda").normal_(0, s[-1] ** -0.5, generator=g).bfloat16().requires_grad_()  # noqa: E731
        gain = lambda: (1 + 0.1 * torch.randn(d, generator=g, device="cuda")).bfloat16().requires_grad_()  # noqa: E731
        self.heads, self.kv_heads, self.hd = heads, kv_heads, hd
        self.embed = torch.randn(vocab, d, generator=g, device="cuda").requires_grad_()
        self.layers = [{"qkv": w((heads + 2 * kv_heads) * hd, d), "o": w(d, heads * hd), "up": w(ffn, d), "down": w(d, ffn), "attn_norm": gain(),
                        "attn_gate": gain(), "ffn_norm": gain(), "ffn_gate": gain(), "next_norm": gain()} for _ in range(layers)]
        self.first_norm, self.head = gain(), w(vocab, d)
        self.rope = P.rope_table(max_positions, hd)

    def leaves(self):
        return [self.embed, self.first_norm, self.head] + [t for w in self.layers for t in w.values()]

    def _rotated(self, x, pos):
        x = x.view(x.shape[0], -1, self.hd)
        cos, sin = self.rope[pos].to(x.dtype).unbind(-1)
        a, b = x.chunk(2, -1)
        return torch.cat([a * cos[:, None] - b * sin[:, None], b * cos[:, None] + a * sin[:, None]], -1)

    def logits(self, ids, start, pos):
        """ids and positions of the packed rows; float32 [rows, vocab]."""
        h = self.embed[ids]
        x = L.first_norm(h, self.first_norm, dtype=torch.bfloat16)
        widths = [self.heads * self.hd, self.kv_heads * self.hd, self.kv_heads * self.hd]
        for w in self.layers:
            q, k, v = (x @ w["qkv"].t()).split(widths, -1)
            y = L.prompt_attention(self._rotated(q, pos), self._rotated(k, pos), v, start, self.hd).flatten(1) @ w["o"].t()
            x, h = L.block_norm(y, h, w["ffn_norm"], w["attn_norm"], w["attn_gate"], residual_scale=0.5)
            y = torch.nn.functional.silu(x @ w["up"].t()) @ w["down"].t()
            x, h = L.block_norm(y, h, w["next_norm"], None, w["ffn_gate"], residual_scale=0.5)
        return (x @ self.head.t()).float()


def batch(lengths=(37, 150, 5, 260), chosen=7, rows=480, vocab=997, seed=1):
    """ids, starts and positions of packed sequences, and the tokens to score (-1: none): the last `chosen` of each, a row earlier."""
    g = torch.Generator().manual_seed(seed)
    start = torch.tensor([0, *lengths]).cumsum(0).to(torch.int32)
    ids, tokens = torch.randint(0, vocab, (rows,), generator=g), torch.full((rows,), -1, dtype=torch.int32)
    pos = torch.zeros(rows, dtype=torch.long)
    for a, b in zip(start[:-1].tolist(), start[1:].tolist()):
        pos[a:b] = torch.arange(b - a)
        first = max(a, b - 1 - chosen)
        tokens[first:b - 1] = ids[first + 1:b].to(torch.int32)
    return ids.cuda(), start.cuda(), pos.cuda(), tokens.cuda()


def objective(logits, tokens, old, advantages, start, eps=0.2, bonus=0.01):
    """The clipped objective of each sequence's chosen tokens, and their mean entropy."""
    now = P.token_logprobs(logits, tokens)
    live = (tokens >= 0).float()
    rows = torch.arange(tokens.shape[0], device="cuda")
    seq = torch.searchsorted(start[1:].long(), rows, right=True).clamp(max=advantages.shape[0] - 1)
    change = torch.zeros_like(advantages).index_add(0, seq, (now.logprob - old) * live)
    ratio = torch.exp(change)
    clipped = torch.minimum(ratio * advantages, ratio.clamp(1 - eps, 1 + eps) * advantages).mean()
    return clipped + bonus * (now.entropy * live).sum() / live.sum()


def learning_step(policy, data, old, advantages):
    """The objective and its gradient at every weight."""
    ids, start, pos, tokens = data
    value = objective(policy.logits(ids, start, pos), tokens, old, advantages, start)
    grads = torch.autograd.grad(value, policy.leaves())
    L.check()
    return value.detach(), grads


if __name__ == "__main__":
    policy, data = Decoder(), batch()
    with torch.no_grad():
        old = P.token_logprobs(policy.logits(*data[:3]), data[3]).logprob
    advantages = torch.tensor([1.0, -0.5, 0.25, 0.8], device="cuda")
    value, grads = learning_step(policy, data, old, advantages)
    print(f"objective {value.item():.4f}, gradient norm {torch.stack([g.float().norm() for g in grads]).norm().item():.4f}")
