"""Beam search over a paged cache with rotary positions and a sliding window: the calls as a decoder makes them.

One attention layer with random weights stands for the model.
  prompt   all sequences' prompts at once: their keys are turned and stored on the way (e3_cache_append_rotated), their queries
           attend with the window and the first tokens (e3_window_attention), e3_beam_select takes the first beams; every beam
           shares its sequence's full pages and gets a copy of the last one (e3_cache_copy),
  step     every beam's new token goes the same way, e3_beam_select takes the best continuations over beams and vocabulary, the
           tables follow the parents (e3_beam_reorder) and the last pages of beams with several children are copied.
Nothing comes to the host between the steps.

  python examples/beam_search.py [steps]
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2505_18573_amd as e3  # noqa: E402


class Layer:
    """Token embeddings, one attention layer over a paged cache, and the projection to logits."""

    def __init__(self, V, q_heads, kv_heads, D, pages, page, cache_type, window, sinks, seed, dev):
        g = torch.Generator(device=dev).manual_seed(seed)
        randn = lambda *s: torch.randn(s, generator=g, device=dev)
        self.V, self.q_heads, self.kv_heads, self.D, self.page, self.window, self.sinks = V, q_heads, kv_heads, D, page, window, sinks
        self.embedding = randn(V, q_heads * D)
        qkv = randn(q_heads * D, (q_heads + 2 * kv_heads) * D) * (q_heads * D) ** -0.5
        # with a single layer queries, keys and values depend on the token alone: one row of each for every token
        self.projected = (self.embedding @ qkv).to(torch.bfloat16).reshape(V, -1, D)
        self.rotary = e3.new_rotary(D, device=dev)
        self.cache = e3.new_cache(pages, page, kv_heads, D, cache_type, dev)

    def project(self, ids):
        x, q, k = self.projected[ids], self.q_heads, self.kv_heads
        return x[:, :q], x[:, q:q + k], x[:, q + k:]

    def attend(self, ids, positions, slots, offsets, table, lens):
        """Stores the tokens' keys and values and returns their attention [tokens, q_heads, D]."""
        q, k, v = self.project(ids)
        q = e3.e3_cache_append_rotated(self.cache, q, k, v, self.rotary, positions, slots)
        out, _ = e3.e3_window_attention(q, self.cache, offsets, table, lens, self.window, self.sinks, self.D ** -0.5)
        return out

    def logits(self, ids, out):
        h = out.reshape(ids.shape[0], -1).float() + 0.2 * self.embedding[(ids + 1) % self.V]
        return (0.1 * h @ self.embedding.t()).to(torch.bfloat16)


class BeamSearch:
    """`beams` beams for each of some prompts of different lengths.  V: a multiple of 8, so that rows of logits start on 16 bytes."""

    def __init__(self, prompts, beams, longest, V=1000, q_heads=8, kv_heads=2, D=64, page=32, cache_type=torch.float8_e4m3fn, window=40, sinks=2,
                 eos=0, tau=1.0, seed=0, dev="cuda"):
        self.beams, self.page, self.eos, self.tau, self.dev = beams, page, eos, tau, dev
        self.seqs, self.rows = len(prompts), len(prompts) * beams
        self.width = (max(len(p) for p in prompts) + longest) // page + 1
        self.layer = Layer(V, q_heads, kv_heads, D, self.rows * self.width, page, cache_type, window, sinks, seed, dev)
        # every row has as many pages as it can need; full ones are shared after the prompt
        self.own = torch.arange(self.rows * self.width, dtype=torch.int32, device=dev).reshape(self.rows, self.width)
        self.table = self.own.clone()
        self.lens = torch.tensor([len(p) for p in prompts], dtype=torch.int32, device=dev).repeat_interleave(beams)
        self.one_each = torch.arange(self.rows + 1, dtype=torch.int32, device=dev)
        self.prompt(prompts)

    def prompt(self, prompts):
        dev, page, first = self.dev, self.page, self.table[::self.beams].contiguous()
        lens = self.lens[::self.beams].contiguous()
        ids = torch.tensor([t for p in prompts for t in p], device=dev)
        row = torch.repeat_interleave(torch.arange(self.seqs, device=dev), lens.long())
        offsets = torch.zeros(self.seqs + 1, dtype=torch.int32, device=dev)
        offsets[1:] = torch.cumsum(lens, 0)
        at = torch.arange(ids.shape[0], device=dev) - offsets[row]
        slots = first[row, at // page].long() * page + at % page
        out = self.layer.attend(ids, at, slots, offsets, first, lens)
        last = offsets[1:].long() - 1
        logits = self.layer.logits(ids[last], out[last]).reshape(self.seqs, 1, -1)
        _, tokens, self.scores = e3.e3_beam_select(logits, torch.zeros((self.seqs, 1), device=dev), self.beams, self.tau)
        self.tokens = tokens.long().reshape(-1)
        self.finished = (tokens == self.eos).to(torch.uint8)
        # the other beams: the first one's full pages, and a copy of the last
        shared = first.repeat_interleave(self.beams, 0)
        full = torch.arange(self.width, device=dev) < (self.lens // page)[:, None]
        self.table = torch.where(full, shared, self.own).contiguous()
        at = (self.lens // page).long()[:, None]
        e3.e3_cache_copy(self.layer.cache, shared.gather(1, at)[:, 0].contiguous(), self.own.gather(1, at)[:, 0].contiguous(), self.lens % page)

    def step(self):
        """One token for every beam.  Returns (logits, scores, finished before the selection; parents, tokens)."""
        at = self.lens.long()
        slots = self.table.gather(1, (at // self.page)[:, None])[:, 0].long() * self.page + at % self.page
        self.lens = self.lens + 1
        out = self.layer.attend(self.tokens, at, slots, self.one_each, self.table, self.lens)
        self.attended = out
        logits = self.layer.logits(self.tokens, out).reshape(self.seqs, self.beams, -1)
        before = (logits, self.scores, self.finished)
        parent, tokens, self.scores = e3.e3_beam_select(logits, self.scores, self.beams, self.tau, self.finished, self.eos)
        # the page of the next token: a row's own where one has been filled
        new = (torch.arange(self.width, device=self.dev) == (self.lens // self.page)[:, None]) & (self.lens % self.page == 0)[:, None]
        table = torch.where(new, self.own, self.table).contiguous()
        self.table, self.lens, src, dst, counts = e3.e3_beam_reorder(parent, table, self.lens, self.page)
        e3.e3_cache_copy(self.layer.cache, src, dst, counts)
        self.tokens = tokens.long().reshape(-1)
        self.finished = (tokens == self.eos).to(torch.uint8)
        return (*before, parent, tokens)


def main(steps=20):
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(1, 1000, (n,), generator=g).tolist() for n in (5, 64, 129, 33)]
    search = BeamSearch(prompts, beams=4, longest=steps)
    history = search.tokens.reshape(4, 4, 1)
    for _ in range(steps):
        *_, parent, tokens = search.step()
        history = torch.cat([history.gather(1, parent.long()[..., None].expand(-1, -1, history.shape[2])), tokens.long()[..., None]], 2)
    for i in range(4):
        print(f"prompt of {len(prompts[i])} tokens, best beam {float(search.scores[i, 0]):.3f}: {history[i, 0].tolist()}")


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 20)
