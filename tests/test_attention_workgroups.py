"""The prefix attention's items of more than 16 queries, which a workgroup takes together with the keys in LDS: pages that do not exist,
values that are no numbers, replays and streams there (tests/test_prefix_attention.py has them for a wave's items).  Tolerances are
those of that file."""
import math

import pytest
import torch

import paper_2505_18573_amd as e3
from tests.test_prefix_attention import BF16, DEV, FP8, Step

# query heads per key head and queries a row: 21 queries (two tiles, two waves on each), 39 and 65 (four tiles, the last one in a
# workgroup of its own)
QUERIES = [(7, 3), (13, 3), (13, 5)]


@pytest.mark.gpu
@pytest.mark.parametrize("cache_type", [FP8, BF16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("R,T", QUERIES)
def test_values_that_are_no_number_stay_where_they_are_seen(cache_type, D, R, T):
    # the last tokens, all but the first query's, hold NaN and inf in turn: queries that do not see them are not touched
    s = Step([2, 1], [37, 64], [50, 34, 131], T, R, 2, D, 32, cache_type, seed=4)
    for r, n in enumerate(s.rows_len):
        for back in range(1, T):
            slot = torch.tensor([s.rp[r, (n - back) // 32] * 32 + (n - back) % 32], device=DEV)
            x = torch.full((1, 2, D), math.nan if back % 2 else math.inf, dtype=torch.float32, device=DEV)
            e3.e3_cache_append(s.cache, s.kr[r][n - back][None].float().to(DEV), x, slot)
    out, lse = e3.e3_prefix_attention(s.q.to(DEV), *s.args())
    want, size, want_lse = s.reference()
    err = (out[:, 0].double().cpu() - want[:, 0]).abs()
    assert bool((err <= (2.0 ** -8 + 1e-4) * size[:, 0]).all())
    assert bool((~torch.isfinite(out[:, 1:])).all())
    assert bool(((lse.double().cpu() - want_lse).abs() <= 2e-5).all())           # the keys are numbers
    # one column of one token only: the other columns are not touched
    t = Step([2, 1], [37, 64], [50, 34, 131], T, R, 2, D, 32, cache_type, seed=4)
    for r, n in enumerate(t.rows_len):
        slot = torch.tensor([t.rp[r, (n - 1) // 32] * 32 + (n - 1) % 32], device=DEV)
        x = t.vr[r][n - 1][None].float().to(DEV)
        x[:, :, 5] = math.nan
        e3.e3_cache_append(t.cache, t.kr[r][n - 1][None].float().to(DEV), x, slot)
    out, lse = e3.e3_prefix_attention(t.q.to(DEV), *t.args())
    want, size, want_lse = t.reference()
    ok = ((out.double().cpu() - want).abs() <= (2.0 ** -8 + 1e-4) * size)
    assert bool(torch.isnan(out[:, T - 1, :, 5]).all())
    ok[:, T - 1, :, 5] = True
    assert bool(ok.all())
    # a key that is no number: the queries that see it are no numbers, the others are not touched
    n = t.rows_len[2]
    slot = torch.tensor([t.rp[2, (n - 1) // 32] * 32 + (n - 1) % 32], device=DEV)
    e3.e3_cache_append(t.cache, torch.full((1, 2, D), math.nan, device=DEV), torch.ones((1, 2, D), device=DEV), slot)
    out2, lse2 = e3.e3_prefix_attention(t.q.to(DEV), *t.args())
    assert torch.equal(out2[:, :T - 1], out[:, :T - 1]) and torch.equal(lse2[:, :T - 1], lse[:, :T - 1])
    assert bool(torch.isnan(out2[2, T - 1]).all()) and bool(torch.isnan(lse2[2, T - 1]).all())


@pytest.mark.gpu
@pytest.mark.parametrize("cache_type", [FP8, BF16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("R,T", QUERIES)
def test_pages_outside_the_cache_hide_their_tokens(cache_type, D, R, T):
    s = Step([2, 1], [200, 33], [290, 40, 70], T, R, 2, D, 32, cache_type, seed=6)
    args = list(s.args())
    args[2], args[4] = args[2].clone(), args[4].clone()
    args[2][0, 1] = -1                                   # tokens 32 .. 63 of the first prefix
    args[2][0, 6] = -7                                   # and its last eight, 192 .. 199
    args[2][1, 0] = 1 << 30                              # tokens 0 .. 31 of the second
    args[4][0, 0] = 1 << 30                              # tokens 0 .. 31 of row 0
    args[4][0, 4:8] = -1                                 # and 128 .. 255: a whole round of four waves
    cut = lambda xs, keep: [x[k] for x, k in zip(xs, keep)]
    at = [torch.arange(n) for n in s.prefix]
    keep = [(at[0] // 32 != 1) & (at[0] < 192), at[1] >= 32]
    s.kp, s.vp = cut(s.kp, keep), cut(s.vp, keep)
    at = [torch.arange(n) for n in s.rows_len]
    keep = [(at[0] >= 32) & ((at[0] < 128) | (at[0] >= 256)), at[1] >= 0, at[2] >= 0]
    s.kr, s.vr = cut(s.kr, keep), cut(s.vr, keep)
    s.rows_len = [130, 40, 70]
    out, lse = e3.e3_prefix_attention(s.q.to(DEV), *args)
    s.check(out, lse)
    # no page of a unit exists, and the lengths end with the tables
    args[2].fill_(-1)
    args[4].fill_(1 << 30)
    args[3].fill_(1 << 30)
    args[5].fill_(1 << 30)
    out, lse = e3.e3_prefix_attention(s.q.to(DEV), *args)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


@pytest.mark.gpu
@pytest.mark.parametrize("cache_type", [FP8, BF16])
@pytest.mark.parametrize("R,T", QUERIES)
def test_strides_streams_and_replays_with_other_lengths(cache_type, R, T):
    s = Step([2, 2], [300, 37], [150, 10, 33, 129], T, R, 2, 64, 64, cache_type, seed=12)
    args = s.args()
    q = s.q.to(DEV)
    ws = torch.randint(0, 255, (e3.e3_prefix_attention_workspace_bytes(4, T, 2 * R, 2, 64, 2),), dtype=torch.uint8, device=DEV)
    first, first_lse = e3.e3_prefix_attention(q, *args)
    s.check(first, first_lse)
    turned = q.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out, lse = e3.e3_prefix_attention(turned, *args, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, first) and torch.equal(lse, first_lse)
    out, lse = torch.empty_like(first), torch.empty_like(first_lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        e3.e3_prefix_attention(q, *args, out=out, lse_out=lse, workspace=ws)
    for lens in ([150, 10, 33, 129], [1, 0, 30, 65], [150, 1, 2, 128], [0, 0, 0, 0]):
        args[5].copy_(torch.tensor(lens, dtype=torch.int32))
        want, want_lse = e3.e3_prefix_attention(q, *args)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
