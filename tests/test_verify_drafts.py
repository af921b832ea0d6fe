"""Verification of drafted tokens against a plain restatement in 64 bits.

Whole numbers (accepted drafts, tokens) have to be equal, except on rows whose decision lies within fp32 rounding: |u q / p - 1| <=
1e-5 at a draft up to the first rejection, or the two best scores of either level of the draw within 1e-5 of each other (the
margin the library's samplers use).  Log-probs and entropies: 1e-4 relative with a floor of 1e-6, the library's bar."""
import ctypes as C
import math

import numpy as np
import pytest
import torch
from scipy.stats import chisquare

import paper_2505_18573_amd as e3
from tests.philox_np import noise_words

DEV = "cuda:0"
NEAR = 1e-5


def uniforms(seed, row, stream, index):
    return ((noise_words(seed, row, stream, index) >> np.uint32(9)).astype(np.float64) + 0.5) / 8388608.0


def softmax(z, tau):
    """p, ln p and the entropy of one line in 64 bits; None if it is no distribution."""
    a = np.asarray(z, dtype=np.float64)
    a = np.where(a <= -1e30, -np.inf, a) / float(np.float32(tau))
    if np.isnan(a).any() or not np.isfinite(a.max()):
        return None
    ln = a - a.max()
    ln = ln - np.log(np.exp(ln).sum())
    p = np.exp(ln)
    return p, ln, -np.sum(np.where(p > 0, p * np.where(p > 0, ln, 0.0), 0.0))


def best_of(weight, noise):
    """(lowest index of the best, whether the second is near)."""
    score = np.where(weight > 0, weight / -np.log(noise), -1.0)
    i = int(np.argmax(score))
    rest = np.delete(score, i)
    return i, bool(rest.size and rest.max() > 0 and rest.max() >= score[i] * (1 - NEAR))


def draw(r, seed, row):
    V = r.size
    cols = np.arange(V)
    tile = cols // 4096 * 64 + cols % 512 // 8
    mass = np.bincount(tile, weights=r, minlength=-(-V // 4096) * 64)
    t, near = best_of(mass, uniforms(seed, row, 6, np.arange(mass.size)))
    inside = cols[tile == t]
    i, near2 = best_of(r[inside], uniforms(seed, row, 7, inside))
    return int(inside[i]), near or near2


def verify_row(z, x, d, n, tau, tau_d, seed, row):
    """(accepted, tokens, logp, entropy, near) of one row: z [K + 1, V], x [K], d [K, V] or None, n drafts."""
    near = False
    logp, entropy = [], []
    u = uniforms(seed, row, 5, np.arange(max(n, 1)))
    for t in range(n + 1):
        p = softmax(z[t], tau)
        if p is None:
            return t, list(x[:t]) + [None], logp + [math.nan], entropy + [math.nan], near
        r = p[0]
        if t < n:
            q = softmax(d[t], tau_d) if d is not None else None
            if 0 <= x[t] < r.size and (d is None or q is not None):
                left, right = u[t] * (q[0][x[t]] if d is not None else 1.0), r[x[t]]
                near |= abs(left - right) <= NEAR * max(left, right)
                if left < right:
                    logp.append(p[1][x[t]])
                    entropy.append(p[2])
                    continue
            if d is None:
                r = r.copy()
                if 0 <= x[t] < r.size:
                    r[x[t]] = 0.0
            elif q is not None:
                # what rounding may turn either way is no weight to draw by
                r = np.maximum(r - q[0], 0.0)
            if not (r > 0).any():
                r = p[0]
        tok, close = draw(r, seed, row)
        return t, list(x[:t]) + [tok], logp + [p[1][tok]], entropy + [p[2]], near or close


def test_argument_checks_without_gpu():
    L = e3.lib()
    need = e3.e3_verify_workspace_bytes(4, 2, 64)
    assert need > 0
    for bad in ((-1, 2, 64), (4, -1, 64), (4, 64, 64), (4, 2, 0), (4, 2, 1 << 21), (1 << 31, 2, 64)):
        assert e3.e3_verify_workspace_bytes(*bad) == 0

    def call(z=0x1000, dtype=1, rows=4, K=2, V=64, rs=192, ps=64, x=0x2000, lens=None, d=0x3000, drs=128, dps=64, tau=1.0,
             acc=0x4000, tok=0x5000, ws=0x10000, ws_bytes=need):
        return L.e3_verify_drafts(z, dtype, rows, K, V, rs, ps, x, lens, d, drs, dps, None, tau, None, 1, 0, acc, tok, None, None,
                                  ws, ws_bytes, None)

    assert call(dtype=2) == -3
    assert call(rows=-1) == -2 and call(K=-1) == -2 and call(K=64) == -2 and call(V=0) == -2 and call(ps=63) == -2 and call(dps=56) == -2
    assert call(V=1 << 21, ps=1 << 21, dps=1 << 21) == -2
    assert call(tau=0.0) == -5 and call(tau=float("nan")) == -5
    for name in ("z", "acc", "tok", "x"):
        assert call(**{name: None}) == -1
    assert call(ws=None) == -6 and call(ws_bytes=need - 1) == -6
    assert call(z=0x1008) == -4 and call(d=0x3004) == -4 and call(ws=0x10080) == -4 and call(rs=196) == -4 and call(drs=132) == -4
    assert call(rows=0, z=None, x=None, acc=None, tok=None, ws=None) == 0


def test_shapes_beyond_a_launch_are_refused():
    # 2^23 positions: their workgroups would pass 2^32 threads
    assert e3.e3_verify_workspace_bytes((1 << 21) - 1, 3, 8) > 0
    assert e3.e3_verify_workspace_bytes(1 << 21, 3, 8) == 0 and e3.e3_verify_workspace_bytes(1 << 23, 0, 8) == 0


def test_the_restatement_draws_from_the_target():
    # whatever the drafter, the first token is distributed as p_0, the second (where there is one) as p_1
    rng = np.random.default_rng(0)
    V, n = 6, 6000
    z, d = rng.normal(0, 1.5, (2, V)), rng.normal(0, 1.5, (1, V))
    for drafter in (d, None):
        q = softmax(d[0], 1.0)[0]
        x = rng.choice(V, n, p=q)
        first, second = np.zeros(V), np.zeros(V)
        for r in range(n):
            a, tok, *_ = verify_row(z, x[r:r + 1], drafter, 1, 1.0, 1.0, 11, r)
            if drafter is None and x[r] != 2:
                continue                                 # without a distribution the draft is one token: look at one
            first[tok[0]] += 1
            if a:
                second[tok[1]] += 1
        assert chisquare(first, softmax(z[0], 1.0)[0] * first.sum()).pvalue > 1e-4
        assert chisquare(second, softmax(z[1], 1.0)[0] * second.sum()).pvalue > 1e-4


class Batch:
    def __init__(self, rows, K, V, dtype, drafter=True, ragged=False, seed=0, spread=3.0, tau=True, draft_tau=False):
        g = torch.Generator().manual_seed(seed)
        self.rows, self.K, self.V, self.seed = rows, K, V, seed * 77 + 5
        self.z = (torch.randn((rows, K + 1, V), generator=g) * spread).to(dtype)
        self.d = (self.z[:, :K].float() + torch.randn((rows, K, V), generator=g) * 0.7).to(dtype) if drafter else None
        self.tau = 0.6 + 0.8 * torch.rand(rows, generator=g) if tau else None
        self.tau_d = 0.6 + 0.8 * torch.rand(rows, generator=g) if draft_tau else None
        t = self.tau_d if draft_tau else self.tau
        t = t[:, None, None] if t is not None else 1.0
        src = (self.d if drafter else self.z[:, :K]).float()
        self.x = ((src / t) - torch.log(-torch.log(torch.rand(src.shape, generator=g).clamp_(1e-9, 1 - 1e-7)))).argmax(-1).to(torch.int32) \
            if K else torch.zeros((rows, 0), dtype=torch.int32)
        self.lens = torch.randint(0, K + 1, (rows,), generator=g).to(torch.int32) if ragged else None

    def call(self, pad=8, **more):
        dt = self.z.dtype

        def padded(t):
            if t is None:
                return None
            wide = torch.full((*t.shape[:2], -(-self.V // 8) * 8 + pad), 1e4, dtype=dt, device=DEV)
            wide[..., :self.V] = t.to(DEV)
            return wide[..., :self.V]

        put = lambda t: None if t is None else t.to(DEV)
        return e3.e3_verify_drafts(padded(self.z), put(self.x), padded(self.d), put(self.lens), put(self.tau), 1.0, self.seed, 1000,
                                   put(self.tau_d), **more)

    def check(self, got, most_near=0.02):
        acc, tok, logp, ent = (t.cpu().numpy() for t in got)
        skipped = 0
        for r in range(self.rows):
            tau = float(self.tau[r]) if self.tau is not None else 1.0
            n = self.K if self.lens is None else int(self.lens[r])
            a, t, lp, h, near = verify_row(self.z[r].double().numpy(), self.x[r].tolist(), None if self.d is None else self.d[r].double().numpy(), n,
                                           tau, float(self.tau_d[r]) if self.tau_d is not None else tau, self.seed, 1000 + r)
            if near:
                skipped += 1
                continue
            assert acc[r] == a, (r, acc[r], a)
            assert (tok[r, a + 1:] == -1).all() and (logp[r, a + 1:] == 0).all() and (ent[r, a + 1:] == 0).all()
            assert tok[r, :a].tolist() == t[:a]
            if t[a] is None:
                assert 0 <= tok[r, a] < self.V
            else:
                assert tok[r, a] == t[a], (r, tok[r], t)
            for x, w in ((logp[r, :a + 1], lp), (ent[r, :a + 1], h)):
                w = np.array(w)
                assert (np.isnan(x) == np.isnan(w)).all()
                assert (np.abs(x - w)[~np.isnan(w)] <= 1e-4 * np.maximum(np.abs(w), 1e-6)[~np.isnan(w)]).all(), (r, x, w)
        assert skipped <= max(1, most_near * self.rows)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("drafter", [True, False])
@pytest.mark.parametrize("rows,K,V", [
    (1, 1, 1), (3, 2, 2), (5, 3, 7), (4, 4, 64), (2, 1, 511), (2, 5, 513), (3, 2, 4096), (3, 3, 4097), (2, 2, 33_001),
    (1, 3, 151_936), (6, 63, 100), (7, 0, 1000), (1, 2, 300_000),
    (600, 1, 1), (300, 3, 130), (700, 0, 77), (260, 2, 4099), (128, 7, 2500)])
def test_against_the_restatement(dtype, drafter, rows, K, V):
    # the first lists go through slices, the last (512 positions and more) through pairs
    b = Batch(rows, K, V, dtype, drafter, ragged=rows % 2 == 0, seed=rows + K + V, draft_tau=V % 3 == 0)
    b.check(b.call())


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [4, 400])
def test_peaked_rows(rows):
    b = Batch(rows, 3, 3000, torch.float32, seed=rows, spread=1.0, tau=False)
    b.z[:, :, 17] += 22.0                                # entropies of 1e-6 and less
    b.d[:, :, 17] += 18.0
    b.x[:, ::2] = 17
    b.check(b.call())


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [6, 600])
@pytest.mark.parametrize("mask", [-math.inf, -1e9, torch.finfo(torch.bfloat16).min])
def test_masked_columns_and_lines_that_are_no_distribution(rows, mask):
    b = Batch(rows, 2, 5000, torch.bfloat16, seed=3)
    b.z[:, :, :4990] = mask                              # ten columns are left; drafts among them
    b.d[:, :, 100:] = mask                               # and others for the drafter
    b.x[0::2] = 4995
    b.x[1::2] = 50
    if mask == -1e9:
        b.d[:, :, 4990:] = 1.0
    b.check(b.call())
    # a line that is masked throughout, one with NaN, one with +inf; drafted ids outside the vocabulary; a drafter of NaN
    b = Batch(rows, 2, 5000, torch.bfloat16, seed=4)
    b.z[0, 0] = -math.inf
    b.z[1, 1, 77] = math.nan
    b.z[2, 0, 4999] = math.inf
    b.x[3, 0], b.x[4, 0] = -1, 5000
    b.d[5, 0, 3] = math.nan
    b.check(b.call())


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [5, 500])
def test_a_drafter_that_is_the_target(rows):
    b = Batch(rows, 3, 6000, torch.bfloat16, seed=8)
    b.d = b.z[:, :3].clone()
    assert bool((b.call()[0] == 3).all())                # u < 1: nothing is rejected
    # a rejected id outside the vocabulary leaves nothing of p - q: the draw is from p
    b.x[:, 1] = 6000
    got = b.call()
    b.check(got)
    assert bool((got[0] == 1).all())


@pytest.mark.gpu
def test_frequencies_are_the_targets():
    rows, V = 40_000, 12
    g = torch.Generator().manual_seed(1)
    z, d = torch.randn((1, 2, V), generator=g) * 1.5, torch.randn((1, 1, V), generator=g) * 1.5
    x = torch.multinomial(torch.softmax(d[0, 0], 0), rows, replacement=True, generator=g).to(torch.int32)[:, None].to(DEV)
    pad = lambda t: torch.nn.functional.pad(t, (0, 4)).to(DEV).expand(rows, -1, -1).contiguous()[..., :V]
    acc, tok, _, _ = e3.e3_verify_drafts(pad(z), x, pad(d), None, None, 1.0, 123)
    p = torch.softmax(z[0].double(), -1).numpy()
    first = np.bincount(tok[:, 0].cpu().numpy(), minlength=V)
    assert chisquare(first, p[0] * rows).pvalue > 1e-4
    second = np.bincount(tok[acc == 1, 1].cpu().numpy(), minlength=V)
    assert chisquare(second, p[1] * second.sum()).pvalue > 1e-4
    rate = float((acc == 1).double().mean())
    want = float(np.minimum(p[0], torch.softmax(d[0, 0].double(), -1).numpy()).sum())
    assert abs(rate - want) <= 4 * math.sqrt(want * (1 - want) / rows)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [9, 300])
def test_given_outputs_streams_repeats_and_batches(rows):
    b = Batch(rows, 4, 9000, torch.bfloat16, ragged=True, seed=6)
    first = b.call()
    need = e3.e3_verify_workspace_bytes(rows, 4, 9000)
    ws = torch.randint(0, 255, (need,), dtype=torch.uint8, device=DEV)
    outs = [torch.full_like(t, 7) for t in first]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = b.call(pad=64, accepted_out=outs[0], token_out=outs[1], logp_out=outs[2], entropy_out=outs[3], workspace=ws)
    side.synchronize()
    for a, o, f in zip(got, outs, first):
        assert a is o and torch.equal(o, f)
    # a row alone: the same random numbers, so the same tokens (near-ties aside: none among these)
    put = lambda t: t.to(DEV)
    one = e3.e3_verify_drafts(put(b.z[5:6]), put(b.x[5:6]), put(b.d[5:6]), put(b.lens[5:6]), put(b.tau[5:6]), 1.0, b.seed, 1005)
    assert torch.equal(one[0], first[0][5:6]) and torch.equal(one[1], first[1][5:6])
    assert torch.allclose(one[2], first[2][5:6], rtol=1e-4, atol=1e-6)
    z = put(b.z)
    with pytest.raises(ValueError):
        e3.e3_verify_drafts(z, put(b.x)[:, :3], None, None, None, 1.0, 1)
    with pytest.raises(ValueError):
        e3.e3_verify_drafts(z, put(b.x), put(b.d).float(), None, None, 1.0, 1)
    with pytest.raises(TypeError):
        e3.e3_verify_drafts(z.half(), put(b.x), None, None, None, 1.0, 1)
    with pytest.raises(e3.E3Error) as err:
        e3.e3_verify_drafts(z, put(b.x), None, None, None, 1.0, 1, workspace=ws[:256])
    assert err.value.status == -6
    with pytest.raises(e3.E3Error) as err:
        e3.e3_verify_drafts(z[..., :8999][..., 1:], put(b.x), None, None, None, 1.0, 1)
    assert err.value.status == -4
    assert e3.e3_verify_drafts(z[:0], put(b.x[:0]), None, None, None, 1.0, 1)[1].shape == (0, 5)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [6, 200])
def test_replayed_from_a_graph(rows):
    b = Batch(rows, 3, 4500, torch.bfloat16, seed=13)
    z, d, x, tau = (t.to(DEV) for t in (torch.nn.functional.pad(b.z, (0, 4)), torch.nn.functional.pad(b.d, (0, 4)), b.x, b.tau))
    ws = torch.empty(e3.e3_verify_workspace_bytes(rows, 3, 4500), dtype=torch.uint8, device=DEV)
    call = lambda **more: e3.e3_verify_drafts(z[..., :4500], x, d[..., :4500], None, tau, 1.0, 9, workspace=ws, **more)
    outs = [torch.empty_like(t) for t in call()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(accepted_out=outs[0], token_out=outs[1], logp_out=outs[2], entropy_out=outs[3])
    for i in range(4):
        z.copy_(z.roll(1, 0))
        d.copy_(d.roll(1, 0))
        want = [t.clone() for t in call()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, w in zip(outs, want):
            assert torch.equal(a, w)
