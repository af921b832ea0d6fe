"""Rollouts of a few questions decoded with drafted tokens: the decode step's calls as a rollout engine makes them.

One attention layer with random weights stands for the model, a second one that reads 16-bit keys and is a little off for the
drafter.  Per step and for all rollouts at once:
  draft    the drafter proposes `drafts` tokens, one after the other (e3_prefix_attention with one query per row,
           e3_sample_entropy for the token),
  verify   the model takes them all in one pass: their keys and values go into the 8-bit cache (e3_cache_append), drafts + 1 queries
           per row attend to the question's prompt, which its rollouts share, and to the row's own tokens
           (e3_prefix_attention), and e3_verify_drafts keeps the drafts that hold, adds a token of the model's own, and
           reports the log-probs and entropies that GRPO and the temperature scheduler need.
Rejected drafts stay behind the rows' lengths in the cache, where nothing sees them, and are written over by the next step.

  python examples/speculative_rollout.py [steps]
"""
from __future__ import annotations

import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2505_18573_amd as e3  # noqa: E402


class Layer:
    """Token embeddings, one attention layer over a paged cache, and the projection to logits."""

    def __init__(self, V, q_heads, kv_heads, D, pages, page, cache_type, g, dev, embedding=None, noise=0.0):
        width = q_heads * D
        randn = lambda *s: torch.randn(s, generator=g, device=dev)
        self.V, self.q_heads, self.kv_heads, self.D, self.page = V, q_heads, kv_heads, D, page
        self.embedding = randn(V, width) if embedding is None else embedding + noise * randn(V, width)
        self.qkv = randn(width, (q_heads + 2 * kv_heads) * D) * width ** -0.5
        self.cache = e3.new_cache(pages, page, kv_heads, D, cache_type, dev)

    def project(self, ids):
        x = (self.embedding[ids] @ self.qkv).to(torch.bfloat16)
        heads = x.reshape(*ids.shape, self.q_heads + 2 * self.kv_heads, self.D)
        return heads[..., :self.q_heads, :], heads[..., self.q_heads:self.q_heads + self.kv_heads, :], heads[..., self.q_heads + self.kv_heads:, :]

    def write(self, ids, slots):
        _, k, v = self.project(ids.reshape(-1))
        e3.e3_cache_append(self.cache, k, v, slots.reshape(-1))

    def logits(self, ids, group_offsets, prefix, rows):
        """Logits [rows, T, V] after each of the T last tokens `ids` [rows, T] of every row; their keys are written already."""
        q, _, _ = self.project(ids)
        out, _ = e3.e3_prefix_attention(q, self.cache, group_offsets, *prefix, *rows, self.D ** -0.5)
        h = out.reshape(*ids.shape, -1).float() + 0.05 * self.embedding[(ids + 1) % self.V]
        return (0.2 * h @ self.embedding.t()).to(torch.bfloat16)


class Rollouts:
    """The rollouts of some questions: budgets per question, prompts shared in the cache."""

    def __init__(self, budgets, prompt_lens, longest, V=1024, q_heads=8, kv_heads=2, D=64, page=32, drafts=3, tau=1.0, seed=0, dev="cuda"):
        g = torch.Generator(device=dev).manual_seed(seed)
        self.dev, self.drafts, self.seed, self.page, self.tau = dev, drafts, seed, page, tau
        self.rows, G = int(sum(budgets)), len(budgets)
        self.offsets = torch.from_numpy(np.concatenate([[0], np.cumsum(budgets)]).astype(np.int32)).to(dev)
        wide = -(-max(prompt_lens) // page)
        own = -(-(longest + drafts + 1) // page)
        pages = G * wide + self.rows * own
        order = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
        self.prefix_pages = order[:G * wide].reshape(G, wide).contiguous()
        self.row_pages = order[G * wide:].reshape(self.rows, own).contiguous()
        self.prefix_lens = torch.tensor(prompt_lens, dtype=torch.int32, device=dev)
        self.lens = torch.zeros(self.rows, dtype=torch.int32, device=dev)      # own tokens whose keys are in the caches
        self.target = Layer(V, q_heads, kv_heads, D, pages, page, torch.float8_e4m3fn, g, dev)
        self.drafter = Layer(V, q_heads, kv_heads, D, pages, page, torch.bfloat16, g, dev, self.target.embedding, noise=0.1)
        prompts = [torch.randint(0, V, (n,), generator=g, device=dev) for n in prompt_lens]
        at = [torch.arange(n - 1, device=dev) for n in prompt_lens]            # the last token of a prompt is each row's first input
        slots = torch.cat([self.prefix_pages[i][a // page].long() * page + a % page for i, a in enumerate(at)])
        for layer in (self.target, self.drafter):
            layer.write(torch.cat([p[:-1] for p in prompts]), slots)           # once per question, not once per rollout
        self.prefix_lens -= 1
        self.last = torch.cat([p[-1:].expand(b) for p, b in zip(prompts, budgets)]).to(torch.int32)

    def slots(self, first, count):
        """Where tokens first, first + 1, ... of every row go: [rows, count]."""
        at = (first[:, None] + torch.arange(count, device=self.dev)).long()
        return torch.gather(self.row_pages, 1, at // self.page).long() * self.page + at % self.page

    def step(self, i):
        """One draft and one verification; returns (accepted, token, logp, entropy) of e3_verify_drafts."""
        prefix = self.prefix_pages, self.prefix_lens
        token, drafted, drafted_logits = self.last, [], []
        for t in range(self.drafts):
            lens = self.lens + t + 1
            self.drafter.write(token.long()[:, None], self.slots(lens - 1, 1))
            z = self.drafter.logits(token.long()[:, None], self.offsets, prefix, (self.row_pages, lens))
            token, _, _ = e3.e3_sample_entropy(z[:, 0], None, self.tau, seed=self.seed + 1, row_base=(i * self.drafts + t) * self.rows)
            drafted.append(token)
            drafted_logits.append(z)
        drafts = torch.stack(drafted, 1)
        ids = torch.cat([self.last[:, None], drafts], 1).long()                # the last token and the drafts: drafts + 1 queries
        n = self.drafts + 1
        lens = self.lens + n
        self.target.write(ids, self.slots(self.lens, n))
        self.drafter.write(ids[:, -1:], self.slots(lens - 1, 1))               # the last draft's keys, which the drafter has not written
        z = self.target.logits(ids, self.offsets, prefix, (self.row_pages, lens))
        out = e3.e3_verify_drafts(z, drafts, torch.cat(drafted_logits, 1), None, None, self.tau, seed=self.seed + 2, row_base=i * self.rows)
        accepted, token = out[:2]
        self.last = torch.gather(token, 1, accepted.long()[:, None])[:, 0]
        self.lens = self.lens + accepted + 1
        return out


def main(steps=20):
    ranks = (np.random.default_rng(0).permutation(6) + 1) / 6
    budgets, _ = e3.e3_allocate_budgets(ranks, 8, 4, 12)                       # Algorithm 1: more rollouts for harder questions
    r = Rollouts(budgets.tolist(), [37, 120, 64, 5, 200, 90], longest=4 * steps + 4)
    kept = written = 0
    entropy = 0.0
    for i in range(steps):
        accepted, token, logp, h = r.step(i)
        kept += int(accepted.sum())
        written += int((token >= 0).sum())
        entropy += float(h.sum())
    print(f"{r.rows} rollouts of {len(budgets)} questions (budgets {budgets.tolist()}), {steps} steps: {written / (steps * r.rows):.2f} tokens per "
          f"step and rollout, {kept / (steps * r.rows * r.drafts):.0%} of the drafts accepted, mean entropy {entropy / written:.3f}")


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 20)
