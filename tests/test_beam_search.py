"""The calls of a beam search together, as a decoder makes them (examples/beam_search.py): what every beam's pages hold, what its
queries get from them and which continuations are taken, each against a plain computation from the beam's tokens alone."""
import importlib.util
import math
import os

import pytest
import torch

import paper_2505_18573_amd as e3
from tests.test_beam import check, reference

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DEV = "cuda:0"


def example():
    spec = importlib.util.spec_from_file_location("beam_search", os.path.join(ROOT, "examples", "beam_search.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.gpu
@pytest.mark.parametrize("cache_type", [torch.float8_e4m3fn, torch.bfloat16])
@pytest.mark.parametrize("beams,window,sinks", [(4, 40, 2), (3, 1000, 0), (8, 7, 1)])
def test_beams_pages_attention_and_selection(cache_type, beams, window, sinks):
    g = torch.Generator().manual_seed(beams)
    prompts = [torch.randint(1, 300, (n,), generator=g).tolist() for n in (5, 64, 31, 97)]
    steps = 45                                                    # over a page's end twice
    s = example().BeamSearch(prompts, beams, steps, V=304, page=32, cache_type=cache_type, window=window, sinks=sinks, dev=DEV)
    layer = s.layer
    tokens = [p + [int(s.tokens[i * beams + b])] for i, p in enumerate(prompts) for b in range(beams)]
    for n in range(steps):
        logits, scores, finished, parent, chosen = s.step()
        want = reference(logits, scores, beams, 1.0, finished.cpu(), s.eos)
        check((parent, chosen, s.scores), want)
        if n % 9 == 0 or n == steps - 1:
            # attention: keys and values of the row's tokens stored once more, in a cache of their own
            for r in range(s.rows):
                ids = torch.tensor(tokens[r], device=DEV)
                L = len(ids)
                q, k, v = layer.project(ids)
                own = e3.new_cache(-(-L // 32), 32, layer.kv_heads, layer.D, cache_type, DEV)
                at = torch.arange(L, device=DEV)
                q = e3.e3_cache_append_rotated(own, q, k, v, layer.rotary, at, at)[-1].double()
                k, v = (x.double() for x in e3.e3_cache_read(own, at, torch.float32))
                seen = (at > L - 1 - window) | (at < sinks)
                R = layer.q_heads // layer.kv_heads
                k, v = (x[seen].repeat_interleave(R, 1).transpose(0, 1) for x in (k, v))
                p = torch.softmax((k @ q[..., None])[..., 0] * layer.D ** -0.5, -1)
                out, size = (p[:, None] @ v)[:, 0], (p[:, None] @ v.abs())[:, 0]
                # bf16's rounding, and 1e-4 for weights and scores in fp32
                assert bool(((s.attended[r].double() - out).abs() <= (2.0 ** -8 + 1e-4) * size).all())
        tokens = [tokens[i * beams + int(p)] + [int(t)] for i in range(s.seqs) for p, t in zip(parent[i], chosen[i])]
    # what the pages hold now: bit for bit the keys and values of the beam's own tokens
    for r in range(s.rows):
        ids = torch.tensor(tokens[r][:-1], device=DEV)            # the last one has not been stored yet
        L = len(ids)
        assert int(s.lens[r]) == L
        _, k, v = layer.project(ids)
        at = torch.arange(L, device=DEV)
        own = e3.new_cache(-(-L // 32), 32, layer.kv_heads, layer.D, cache_type, DEV)
        e3.e3_cache_append_rotated(own, None, k, v, layer.rotary, at, at)
        slots = s.table[r].long()[at // 32] * 32 + at % 32
        for a, b in zip(e3.e3_cache_read(layer.cache, slots, torch.float32), e3.e3_cache_read(own, at, torch.float32)):
            assert torch.equal(a, b)
    assert math.isfinite(float(s.scores.max()))


@pytest.mark.gpu
def test_the_example_runs(capsys):
    example().main(3)
    assert capsys.readouterr().out.count("best beam") == 4


@pytest.mark.gpu
@pytest.mark.parametrize("beams", [1, 3, 8])
def test_tables_that_are_filled_ahead(beams):
    # Every row has all the pages that it can need from the start.  Behind the page of the next token a table is the parent's after a
    # reordering; with the row's own entries set there again no page that is written to has two names, and pages hold the beams' tokens.
    g = torch.Generator().manual_seed(beams)
    seqs, page, width, D = 4, 32, 4, 64
    rows = seqs * beams
    cache = e3.new_cache(rows * width, page, 1, D, torch.bfloat16, DEV)
    table = torch.randperm(rows * width, generator=g).reshape(rows, width).to(torch.int32).to(DEV)
    lens = torch.zeros(rows, dtype=torch.int32, device=DEV)
    held = torch.zeros((rows, 0), dtype=torch.int64)              # the numbers that stand for a row's tokens
    index = torch.arange(width, device=DEV)
    for step in range(width * page - 1):
        new = torch.randint(0, 200, (rows,), generator=g)         # exact in bf16
        held = torch.cat([held, new[:, None]], 1)
        slots = table.gather(1, (lens // page).long()[:, None])[:, 0].long() * page + lens % page
        x = new.to(DEV).to(torch.bfloat16)[:, None, None].expand(rows, 1, D).contiguous()
        e3.e3_cache_append(cache, x, x, slots)
        lens = lens + 1
        parent = torch.randint(0, beams, (seqs, beams), generator=g).to(torch.int32)
        before = table
        table, lens, src, dst, counts = e3.e3_beam_reorder(parent.to(DEV), before, lens, page)
        e3.e3_cache_copy(cache, src, dst, counts)
        of = (torch.arange(seqs)[:, None] * beams + parent).reshape(-1)
        held = held[of]
        behind = index > (lens // page)[:, None]
        assert torch.equal(table[behind], before[of.to(DEV)][behind])
        table = torch.where(behind, before, table)
        written = table[index >= (lens // page)[:, None]]
        assert written.unique().numel() == written.numel()
        if step % 31 == 30 or step == width * page - 2:
            at = torch.arange(step + 1, device=DEV)
            for r in range(rows):
                k, v = e3.e3_cache_read(cache, table[r].long()[at // page] * page + at % page)
                assert torch.equal(k[:, 0, 0].long().cpu(), held[r]) and torch.equal(v[:, 0, D - 1].long().cpu(), held[r])
