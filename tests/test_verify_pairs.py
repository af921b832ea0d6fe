"""Verification of drafted tokens on batches that fill the card, which go position by position ("pairs"), and on batches whose race
goes through long slices, against the restatement in 64 bits (tests/test_verify_drafts.py, whose batches all go through short slices).

How a batch goes is asserted from its workspace, which holds a line's sums (32 bytes a slice behind the line's own 16) only where
there are slices; the numbers of rows are taken from the number of compute units."""
import math

import pytest
import torch

import paper_2505_18573_amd as e3
from tests.test_verify_drafts import DEV, Batch

SHORT = 16_384                                           # columns up to which twelve positions per compute unit are needed, above two


def by_pairs(rows, K, V):
    return e3.e3_verify_workspace_bytes(rows, K, V) < rows * (2 * K + 1) * 48


def rows_for_pairs(K, V, more=3):
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    rows = -(-cus * (12 if V <= SHORT else 2) // (K + 1)) + more
    assert by_pairs(rows, K, V)
    return rows


def test_the_workspace_tells_the_ways_apart():
    assert not by_pairs(4, 3, 151_936) and not by_pairs(300, 3, 130)
    assert by_pairs(4096, 3, 151_936) and by_pairs(1 << 16, 0, 130)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("drafter", [True, False])
@pytest.mark.parametrize("K,V", [
    (3, 16_389), (4, 20_481), (1, 20_480),               # complete super-tiles of 4096 columns and what is left of the line
    (7, 4096), (2, 4099), (1, 130), (63, 100), (0, 513), (11, 1)])
def test_against_the_restatement(dtype, drafter, K, V):
    b = Batch(rows_for_pairs(K, V), K, V, dtype, drafter, ragged=K % 2 == 1, seed=K + V, draft_tau=V % 3 == 0)
    b.check(b.call())


@pytest.mark.gpu
@pytest.mark.parametrize("drafter", [True, False])
def test_positions_behind_a_rejection(drafter):
    # many more positions than workgroups at a time; half the rows end at their first draft, a quarter at the eighth
    K, V = 15, 1000
    b = Batch(rows_for_pairs(K, V, 300), K, V, torch.bfloat16, drafter, seed=21, spread=1.0)
    b.d = b.z[:, :K].clone() if drafter else None        # the others accept all where the drafts are the target's own
    b.z[::2, 0, 7], b.x[::2, 0] = -30.0, 7
    b.z[1::4, 7, 9], b.x[1::4, 7] = -30.0, 9
    if drafter:
        b.d[::2, 0, 7] = b.d[1::4, 7, 9] = 5.0
    got = b.call()
    b.check(got)
    assert bool((got[0][::2] == 0).all()) and bool((got[0][1::4] <= 7).all())
    if drafter:
        assert bool((got[0][3::4] == K).all())


@pytest.mark.gpu
def test_peaked_rows():
    b = Batch(rows_for_pairs(3, 3000), 3, 3000, torch.float32, seed=400, spread=1.0, tau=False)
    b.z[:, :, 17] += 22.0                                # entropies of 1e-6 and less
    b.d[:, :, 17] += 18.0
    b.x[:, ::2] = 17
    b.check(b.call())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("mask", [-math.inf, -1e9, torch.finfo(torch.bfloat16).min])
def test_masked_columns(dtype, mask):
    V = 16_400
    b = Batch(rows_for_pairs(2, V), 2, V, dtype, seed=3)
    b.z[:, :, :V - 10] = mask                            # ten columns are left; drafts among them
    b.d[:, :, 100:] = mask                               # and others for the drafter
    b.x[0::2] = V - 5
    b.x[1::2] = 50
    if mask == -1e9:
        b.d[:, :, V - 10:] = 1.0
    b.check(b.call())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("drafter", [True, False])
def test_lines_that_are_no_distribution(dtype, drafter):
    # a line that is masked throughout, one with NaN, one with +inf, at drafts and behind the last; ids outside the vocabulary; a
    # drafter of NaN, of +inf, masked throughout
    V = 16_400
    b = Batch(rows_for_pairs(2, V), 2, V, dtype, drafter, seed=4)
    b.z[0, 0] = -math.inf
    b.z[1, 1, 77] = math.nan
    b.z[2, 0, V - 1] = math.inf
    b.z[6, 2] = -math.inf
    b.z[7, 2, 4096] = math.nan
    b.x[3, 0], b.x[4, 0] = -1, V
    if drafter:
        b.d[5, 0, 3], b.d[8, 1, V - 1] = math.nan, math.inf
        b.d[9, 0] = -math.inf
    b.check(b.call())


@pytest.mark.gpu
def test_a_drafter_that_is_the_target():
    V = 16_389
    b = Batch(rows_for_pairs(3, V), 3, V, torch.bfloat16, seed=8)
    b.d = b.z[:, :3].clone()
    assert bool((b.call()[0] == 3).all())                # u < 1: nothing is rejected
    b.x[:, 1] = V                                        # rejected, and nothing of p - q is left: the draw is from p
    got = b.call()
    b.check(got)
    assert bool((got[0] == 1).all())


@pytest.mark.gpu
def test_streams_repeats_and_batches():
    K, V = 4, 16_385
    rows = rows_for_pairs(K, V)
    b = Batch(rows, K, V, torch.bfloat16, ragged=True, seed=6)
    first = b.call()
    ws = torch.randint(0, 255, (e3.e3_verify_workspace_bytes(rows, K, V),), dtype=torch.uint8, device=DEV)
    outs = [torch.full_like(t, 7) for t in first]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = b.call(pad=64, accepted_out=outs[0], token_out=outs[1], logp_out=outs[2], entropy_out=outs[3], workspace=ws)
    side.synchronize()
    for a, o, f in zip(got, outs, first):
        assert a is o and torch.equal(o, f)
    # the first rows alone, which then go through slices: the same random numbers, so the same tokens (near-ties aside: none among these)
    part = Batch.__new__(Batch)
    part.__dict__.update(b.__dict__, rows=5, z=b.z[:5], x=b.x[:5], d=b.d[:5], lens=b.lens[:5], tau=b.tau[:5])
    assert not by_pairs(5, K, V)
    for x, f in zip(part.call(), first):
        assert torch.equal(x, f[:5]) if not x.dtype.is_floating_point else torch.allclose(x, f[:5], rtol=1e-4, atol=1e-6)


@pytest.mark.gpu
def test_replayed_from_a_graph():
    K, V = 3, 16_388
    rows = rows_for_pairs(K, V)
    b = Batch(rows, K, V, torch.bfloat16, seed=13)
    z, d, x, tau = (t.to(DEV) for t in (torch.nn.functional.pad(b.z, (0, 4)), torch.nn.functional.pad(b.d, (0, 4)), b.x, b.tau))
    ws = torch.empty(e3.e3_verify_workspace_bytes(rows, K, V), dtype=torch.uint8, device=DEV)
    call = lambda **more: e3.e3_verify_drafts(z[..., :V], x, d[..., :V], None, tau, 1.0, 9, workspace=ws, **more)
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


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,drafter,K", [(torch.bfloat16, True, 1), (torch.float32, False, 0)])
def test_a_race_through_long_slices(dtype, drafter, K):
    # just below the number of positions that go by pairs: few slices a row, each of eight super-tiles or more, a wave's each
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    rows = 2 * cus // (K + 1) - 2
    V = 4096 * 8 * -(-5 * cus // rows) + 5
    assert not by_pairs(rows, K, V)
    b = Batch(rows, K, V, dtype, drafter, seed=30 + K)
    b.check(b.call())
