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
