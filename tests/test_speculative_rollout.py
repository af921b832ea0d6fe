"""The decode step's calls together, as the example makes them, against the same model computed plainly in 64 bits."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import paper_2505_18573_amd as e3

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DEV = "cuda:0"


def _example():
    spec = importlib.util.spec_from_file_location("speculative_rollout", os.path.join(ROOT, "examples", "speculative_rollout.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_the_example_can_be_imported_without_a_gpu():
    assert callable(_example().main)


@pytest.mark.gpu
def test_kept_tokens_have_the_models_probabilities():
    m = _example()
    budgets, prompts = [3, 1, 2], [33, 5, 70]
    r = m.Rollouts(budgets, prompts, longest=40, V=256, q_heads=4, kv_heads=2, D=64, drafts=3, seed=5)
    layer, group = r.target, np.repeat(np.arange(3), budgets)
    texts = [[int(t)] for t in r.last]                    # input tokens of every row, the prompt's last first
    stored = {}
    for i in range(6):
        before = [len(t) for t in texts]
        accepted, token, logp, entropy = (t.cpu() for t in r.step(i))
        for row, n in enumerate(accepted.tolist()):
            assert 0 <= n <= 3 and (token[row, n + 1:] == -1).all() and (token[row, :n + 1] >= 0).all()
            texts[row] += token[row, :n + 1].tolist()
            stored[row, i] = (before[row], logp[row, :n + 1], entropy[row, :n + 1])
        assert r.lens.cpu().tolist() == [len(t) - 1 for t in texts]
    # every row again, one token after the other, from what the cache holds of its prompt and its own tokens
    emb = layer.embedding.double().cpu()
    for row, text in enumerate(texts):
        g = group[row]

        def read(pages, n):
            at = torch.arange(n, device=DEV)
            slots = pages[at // r.page].long() * r.page + at % r.page
            return [x.double().cpu() for x in e3.e3_cache_read(layer.cache, slots, torch.float32)]

        kp, vp = read(r.prefix_pages[g], prompts[g] - 1)
        kr, vr = read(r.row_pages[row], len(text) - 1)
        ids = torch.tensor(text[:-1], device=DEV)
        q = layer.project(ids)[0].double().cpu()
        ln_p = []
        for t in range(len(text) - 1):
            k, v = torch.cat([kp, kr[:t + 1]]), torch.cat([vp, vr[:t + 1]])
            out = torch.cat([torch.softmax(k[:, h // 2] @ q[t, h] * 64 ** -0.5, 0) @ v[:, h // 2] for h in range(4)])
            ln_p.append(torch.log_softmax(0.2 * (out + 0.05 * emb[(text[t] + 1) % 256]) @ emb.t(), -1))
        for i in range(6):
            at, logp, entropy = stored[row, i]
            for j in range(logp.numel()):
                p = ln_p[at - 1 + j]
                # logits are up to about 10 in size, rounded to bf16 (2^-8 of each, 0.04) from an output that is rounded too (2^-8 of its
                # 256 elements of both signs: 0.2 * 2^-8 * 16): 0.1 in a log-prob with its normaliser
                assert abs(float(logp[j]) - float(p[text[at + j]])) < 0.1
                assert abs(float(entropy[j]) + float((p.exp() * p).sum())) < 0.1


@pytest.mark.gpu
def test_the_example_runs(capsys):
    _example().main(3)
    assert "tokens per step and rollout" in capsys.readouterr().out
