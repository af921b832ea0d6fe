"""Attention over a paged cache with a sliding window and first tokens that stay visible, against plain attention in 64 bits.

Tolerance of an output: it is rounded to bf16 (2^-8 |out| at most, and |out| <= sum p|v|); the weights have sixteen bits at least
(2^-17) and all else is fp32: scores of at most 40 in magnitude with 128 products, relative weight errors below 1e-4.  So
|out - ref| <= (2^-8 + 1e-4) sum p|v|.  lse: 2e-5 absolute (scores' fp32 errors)."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2505_18573_amd as e3
from tests.test_kv_cache import cache_struct

DEV = "cuda:0"
FP8, BF16 = torch.float8_e4m3fn, torch.bfloat16


def test_argument_checks_without_gpu():
    L = e3.lib()
    need = e3.e3_window_attention_workspace_bytes(4, 9, 4, 2, 128)
    assert need > 0
    for bad in ((4, 9, 5, 2, 128), (4, 9, 4, 2, 96), (-1, 9, 4, 2, 128), (4, -1, 4, 2, 128), (0, 9, 4, 2, 128), (4, 0, 4, 2, 128), (4, 9, 1, 2, 64)):
        assert e3.e3_window_attention_workspace_bytes(*bad) == 0

    def call(c=cache_struct(), q=0x1000, tokens=9, heads=4, strides=(512, 128), off=0x2000, rows=4, rp=0x5000, rw=2, rl=0x6000, window=5, sinks=1,
             scale=0.1, out=0x7000, ws=0x10000, ws_bytes=need):
        return L.e3_window_attention(C.byref(c) if c is not None else None, q, tokens, heads, *strides, off, rows, rp, rw, rl, window, sinks, scale,
                                     out, None, ws, ws_bytes, None)

    assert call(c=None) == -1 and call(c=cache_struct(page=24)) == -2 and call(c=cache_struct(dtype=0)) == -3 and call(c=cache_struct(v=None)) == -1
    assert call(heads=5) == -2 and call(tokens=-1) == -2 and call(rows=-1) == -2 and call(rw=-1) == -2
    assert call(scale=0.0) == -5 and call(scale=float("nan")) == -5 and call(scale=float("inf")) == -5
    assert call(window=0) == -5 and call(window=-3) == -5 and call(sinks=-1) == -5
    for name in ("q", "out", "rl", "rp", "off"):
        assert call(**{name: None}) == -1
    assert call(ws=None) == -6 and call(ws_bytes=need - 1) == -6
    assert call(q=0x1008) == -4 and call(out=0x7008) == -4 and call(ws=0x10010) == -4 and call(strides=(512, 132)) == -4 and call(strides=(508, 128)) == -4
    assert call(rows=0, q=None, out=None, rl=None, ws=None) == 0 and call(tokens=0, q=None, out=None, ws=None) == 0


def test_shapes_beyond_a_launch_are_refused():
    need = e3.e3_window_attention_workspace_bytes
    assert need(1 << 23, 1 << 23, 2, 2, 64) == 0                       # rows x key heads
    assert need(4, 1 << 26, 32, 2, 64) == 0                            # queries x heads
    L, c = e3.lib(), cache_struct()
    assert L.e3_window_attention(C.byref(c), 0x1000, 1 << 26, 32, 512, 128, 0x2000, 4, 0x5000, 2, 0x6000, 5, 1, 0.1, 0x7000, None, 0x10000, 1 << 40, None) == -2


class Batch:
    """Rows of ns[i] queries at the end of lens[i] tokens; keys and values in 64 bits."""

    def __init__(self, ns, lens, R, H, D, page, cache_type, window, sinks, seed=0, loud=1.0, spare=3):
        g = torch.Generator().manual_seed(seed)
        rows = len(ns)
        width = max(1, -(-max(lens) // page))
        order = torch.randperm(rows * width, generator=g) + spare
        self.ns, self.lens, self.R, self.H, self.D, self.page, self.window, self.sinks = ns, lens, R, H, D, page, window, sinks
        self.rows, self.tokens = rows, sum(ns)
        self.table = order.reshape(rows, width)
        self.q = (torch.randn((self.tokens, H * R, D), generator=g) * loud).to(BF16)
        self.scale = D ** -0.5
        self.offsets = np.concatenate([[0], np.cumsum(ns)])
        self.cache = e3.new_cache(rows * width + spare, page, H, D, cache_type, DEV)
        for t in self.cache:                             # what no query sees is no number
            if t is not None:
                t.view(torch.uint8).fill_(255)
        self.k, self.v, self.seen = [], [], []
        used = torch.zeros(rows, width, dtype=torch.bool)
        for r in range(rows):
            n = lens[r]
            p = n - ns[r] + torch.arange(ns[r])
            j = torch.arange(n)
            seen = (j <= p[:, None]) & ((j > p[:, None] - window) | (j < sinks))         # [queries, tokens]
            at = torch.nonzero(seen.any(0))[:, 0]
            k, v = (torch.full((n, H, D), 1e30, dtype=torch.float64) for _ in range(2))
            if len(at):
                x = [torch.randn((len(at), H, D), generator=g).to(BF16) for _ in range(2)]
                slots = (self.table[r, at // page] * page + at % page).to(DEV)
                e3.e3_cache_append(self.cache, x[0].to(DEV), x[1].to(DEV), slots)
                k[at], v[at] = (t.cpu().double() for t in e3.e3_cache_read(self.cache, slots, torch.float32))
                used[r, at // page] = True
            self.k.append(k)
            self.v.append(v)
            self.seen.append(seen)
        # pages of which nothing is seen have gone to others, or nowhere
        stray = torch.randint(-3, rows * width + 2 * spare, (rows, width), generator=g)
        self.table = torch.where(used, self.table, stray)

    def args(self):
        i32 = lambda t: torch.as_tensor(t, dtype=torch.int32).contiguous().to(DEV)
        return self.cache, i32(self.offsets), i32(self.table), i32(self.lens), self.window, self.sinks, self.scale

    def reference(self):
        """out, sum p|v| and lse in 64 bits."""
        Hq = self.H * self.R
        out = torch.zeros((self.tokens, Hq, self.D), dtype=torch.float64)
        size, lse = torch.zeros_like(out), torch.full((self.tokens, Hq), -math.inf, dtype=torch.float64)
        for r in range(self.rows):
            if not self.ns[r]:
                continue
            q = self.q[self.offsets[r]:self.offsets[r + 1]].double().transpose(0, 1)                   # [Hq, n, D]
            k, v = (x[r].transpose(0, 1).repeat_interleave(self.R, 0) for x in (self.k, self.v))      # [Hq, tokens, D]
            s = (q @ k.transpose(1, 2)) * self.scale
            s = torch.where(self.seen[r], s, torch.full_like(s, -math.inf))
            m = s.amax(-1, keepdim=True) if s.shape[-1] else torch.full(s.shape[:2] + (1,), -math.inf, dtype=torch.float64)
            e = torch.exp(s - torch.where(m == -math.inf, torch.zeros_like(m), m))
            total = e.sum(-1, keepdim=True)
            p = e / torch.where(total > 0, total, torch.ones_like(total))
            at = slice(self.offsets[r], self.offsets[r + 1])
            out[at], size[at] = (p @ v).transpose(0, 1), (p @ v.abs()).transpose(0, 1)
            lse[at] = (m + torch.log(total))[..., 0].t()
        return out, size, lse

    def check(self, got, lse):
        want, size, want_lse = self.reference()
        err = (got.double().cpu() - want).abs()
        bound = (2.0 ** -8 + 1e-4) * size
        assert bool((err <= bound).all()), (float((err / bound.clamp(min=1e-30)).max()), torch.nonzero(~(err <= bound))[:5].tolist())
        none = want_lse == -math.inf
        lse = lse.double().cpu()
        assert torch.equal(lse == -math.inf, none)
        assert bool(((lse - want_lse)[~none].abs() <= 2e-5).all()), float((lse - want_lse)[~none].abs().max())


EDGES = [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 300]


@pytest.mark.gpu
@pytest.mark.parametrize("cache_type", [FP8, BF16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("R", [1, 7, 16, 17, 32])
@pytest.mark.parametrize("window,sinks", [(1, 0), (5, 4), (32, 0), (64, 33), (1000, 0), (100, 200)])
def test_one_query(cache_type, D, R, window, sinks):
    b = Batch([1] * len(EDGES), EDGES, R, 2, D, 32 if R % 2 else 64, cache_type, window, sinks, seed=R + window)
    b.check(*e3.e3_window_attention(b.q.to(DEV), *b.args()))


@pytest.mark.gpu
@pytest.mark.parametrize("cache_type", [FP8, BF16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("R", [1, 4, 7])
@pytest.mark.parametrize("window,sinks", [(1, 1), (50, 0), (64, 4), (129, 70), (1 << 40, 1 << 35)])
def test_mixed_rows(cache_type, D, R, window, sinks):
    # rows of no, one, a few and many queries: nothing before them, a little, much; more queries than tokens
    ns = [0, 1, 3, 33, 128, 129, 300, 5, 1, 64, 17, 2, 9, 70]
    lens = [10, 1, 64, 33, 128, 300, 311, 2, 200, 1000, 700, 0, 333, 31]
    b = Batch(ns, lens, R, 2, D, 32 if R % 2 else 64, cache_type, window, sinks, seed=R * 10 + sinks % 97)
    b.check(*e3.e3_window_attention(b.q.to(DEV), *b.args()))


@pytest.mark.gpu
@pytest.mark.parametrize("cache_type,D,page", [(FP8, 128, 32), (BF16, 64, 128), (BF16, 128, 64)])
def test_long_rows_are_cut_and_joined(cache_type, D, page):
    # few rows of many tokens: an item's steps are spread over many workers, of either kind
    for ns, lens, window, sinks in (([1, 2], [9001, 4097], 1 << 30, 0), ([40], [7000], 5000, 100), ([130, 1], [6003, 8001], 1 << 30, 3), ([1], [20_000], 9000, 1000)):
        b = Batch(ns, lens, 3, 1, D, page, cache_type, window, sinks, seed=lens[0])
        b.check(*e3.e3_window_attention(b.q.to(DEV), *b.args()))


@pytest.mark.gpu
def test_many_rows():
    # more rows than the plan keeps in LDS, rows without queries among them
    rng = np.random.default_rng(3)
    ns = rng.integers(0, 3, 9001).tolist()
    lens = [int(n + x) for n, x in zip(ns, rng.integers(0, 40, 9001))]
    b = Batch(ns, lens, 2, 1, 64, 32, BF16, 20, 2)
    b.check(*e3.e3_window_attention(b.q.to(DEV), *b.args()))


@pytest.mark.gpu
@pytest.mark.parametrize("cache_type", [FP8, BF16])
def test_loud_scores(cache_type):
    # maxima that rise along the keys, scores of up to 40
    b = Batch([1, 200, 20], [400, 500, 450], 2, 2, 128, 64, cache_type, 300, 2, loud=7.0)
    b.check(*e3.e3_window_attention(b.q.to(DEV), *b.args()))


@pytest.mark.gpu
@pytest.mark.parametrize("cache_type", [FP8, BF16])
def test_values_that_are_no_numbers(cache_type):
    # a value that is no number: the column is none either for the queries that see it, all others are as without it
    b = Batch([100, 4, 1], [150, 90, 40], 2, 2, 64, 32, cache_type, 40, 3)
    q = b.q.to(DEV)
    out, lse = e3.e3_window_attention(q, *b.args())
    for r, j, col in ((0, 60, 5), (0, 1, 63), (0, 149, 0), (1, 87, 17), (1, 0, 3), (2, 39, 9)):
        b2 = Batch([100, 4, 1], [150, 90, 40], 2, 2, 64, 32, cache_type, 40, 3)
        page, at = int(b2.table[r, j // 32]), j % 32
        b2.cache.v.view(torch.uint8).view(cache_type)[page, 1, at // 8, col, at % 8] = float("nan")
        got, got_lse = e3.e3_window_attention(q, *b2.args())
        hit = torch.zeros_like(out, dtype=torch.bool)
        hit[b.offsets[r]:b.offsets[r + 1], 2:, col] = b.seen[r][:, j].to(DEV)[:, None]
        assert bool(torch.isnan(got[hit]).all()) and torch.equal(got[~hit], out[~hit]) and torch.equal(got_lse, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("cache_type", [FP8, BF16])
def test_pages_that_do_not_exist_hide_their_tokens(cache_type):
    for ns, lens in (([1, 3], [200, 170]), ([150], [230]), ([20], [200])):
        b = Batch(ns, lens, 4, 1, 64, 32, cache_type, 90, 5)
        for r in range(len(ns)):
            for at, bad in ((lens[r] // 32 - 1, -1), (0, 1 << 30)):
                b.table[r, at] = bad
                b.seen[r][:, at * 32:(at + 1) * 32] = False
        b.check(*e3.e3_window_attention(b.q.to(DEV), *b.args()))
    # lengths beyond the table are cut to it, negative ones are none
    b = Batch([2, 2], [64, 64], 1, 1, 64, 32, cache_type, 100, 0)
    args = list(b.args())
    args[3] = torch.tensor([1000, 64], dtype=torch.int32, device=DEV)
    b.check(*e3.e3_window_attention(b.q.to(DEV), *args))
    args[3] = torch.tensor([-5, 64], dtype=torch.int32, device=DEV)
    out, lse = e3.e3_window_attention(b.q.to(DEV), *args)
    assert not out[:2].any() and bool((lse[:2] == -math.inf).all()) and not torch.isnan(out).any()


@pytest.mark.gpu
def test_few_rows_in_a_wide_table():
    # so wide that their steps might not fit the short plan
    b = Batch([1, 0, 30, 200, 5], [40, 9, 64, 300, 5], 2, 8, 64, 32, FP8, 1 << 40, 0)
    cache, offsets, table, lens, *rest = b.args()
    b.check(*e3.e3_window_attention(b.q.to(DEV), cache, offsets, table, lens, *rest))
    wide = torch.full((5, 40_000), -1, dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = table
    b.check(*e3.e3_window_attention(b.q.to(DEV), cache, offsets, wide, lens, *rest))


@pytest.mark.gpu
@pytest.mark.parametrize("cache_type,D,spare", [(BF16, 128, 270_000), (FP8, 64, 1_060_000)])
def test_pages_behind_four_gigabytes(cache_type, D, spare):
    b = Batch([1, 40, 3], [200, 500, 64], 4, 1, D, 64, cache_type, 100, 4, spare=spare)
    assert spare * 64 * D * b.cache.k.element_size() > 1 << 32
    # a stray page may be any, but those before the spare ones hold what others do
    b.check(*e3.e3_window_attention(b.q.to(DEV), *b.args()))


@pytest.mark.gpu
def test_strides_outputs_and_queries_behind_the_last_row():
    b = Batch([3, 40, 1], [100, 77, 50], 4, 2, 128, 64, FP8, 60, 1)
    want, want_lse = e3.e3_window_attention(b.q.to(DEV), *b.args())
    b.check(want, want_lse)
    # queries as a part of wider rows, and a few more of them behind the last row's
    wide = torch.randn((50, 12, 128), generator=torch.Generator().manual_seed(1)).to(BF16)
    wide[:44, 2:10] = b.q
    out = torch.full((50, 8, 128), 3.0, dtype=BF16, device=DEV)
    lse = torch.full((50, 8), 5.0, device=DEV)
    ws = torch.full((e3.e3_window_attention_workspace_bytes(3, 50, 8, 2, 128),), 255, dtype=torch.uint8, device=DEV)
    got = e3.e3_window_attention(wide.to(DEV)[:, 2:10], *b.args(), out=out, lse_out=lse, workspace=ws)
    assert got[0] is out and got[1] is lse
    assert torch.equal(out[:44], want) and torch.equal(lse[:44], want_lse) and bool((out[44:] == 3.0).all()) and bool((lse[44:] == 5.0).all())
    # heads before tokens; without lse
    q = b.q.transpose(0, 1).contiguous().to(DEV).transpose(0, 1)
    got, none = e3.e3_window_attention(q, *b.args(), want_lse=False)
    assert torch.equal(got, want) and none is None


@pytest.mark.gpu
def test_same_bits_graph_and_streams():
    b = Batch([1, 150, 9, 0, 33], [900, 300, 64, 7, 200], 7, 2, 128, 32, FP8, 128, 4)
    q, args = b.q.to(DEV), b.args()
    same = lambda x, y: torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    want, want_lse = e3.e3_window_attention(q, *args)
    b.check(want, want_lse)
    ws = torch.empty(e3.e3_window_attention_workspace_bytes(5, b.tokens, 14, 2, 128), dtype=torch.uint8, device=DEV)
    out, lse = torch.zeros_like(want), torch.zeros_like(want_lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        e3.e3_window_attention(q, *args, out=out, lse_out=lse, workspace=ws)
    for i in range(4):
        out.zero_()
        lse.zero_()
        ws.fill_(i * 85)
        graph.replay()
        torch.cuda.synchronize()
        assert same(out, want) and same(lse, want_lse)
        # shorter rows, read by the same graph: their windows reach tokens that are no numbers, whose bits are compared as well
        if i == 2:
            args[3].sub_(torch.tensor([100, 0, 1, 0, 3], dtype=torch.int32, device=DEV))
            want, want_lse = e3.e3_window_attention(q, *args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got, got_lse = e3.e3_window_attention(q, *args)
    torch.cuda.current_stream().wait_stream(side)
    assert same(got, want) and same(got_lse, want_lse)


@pytest.mark.gpu
def test_agrees_with_prefix_attention():
    # a window of any length, one query a row, no groups: the same attention
    lens = [1, 70, 333, 64]
    b = Batch([1] * 4, lens, 6, 2, 128, 64, BF16, 1 << 20, 0)
    out, lse = e3.e3_window_attention(b.q.to(DEV), *b.args())
    args = b.args()
    want, want_lse = e3.e3_prefix_attention(b.q.to(DEV)[:, None], b.cache, None, None, None, args[2], args[3], b.scale)
    assert bool((out.float() - want[:, 0].float()).abs().max() <= 2.0 ** -7) and bool((lse - want_lse[:, 0]).abs().max() <= 4e-5)


@pytest.mark.gpu
@pytest.mark.parametrize("far", [1 << 63, 1 << 64, (1 << 64) + 5, -(1 << 64) + 7])
def test_numbers_that_64_bits_do_not_hold(far):
    # cut to 64 bits they would be other windows; the largest that they hold is plain causal attention
    cache = e3.new_cache(4, 32, 1, 64, torch.bfloat16, DEV)
    for t in cache[:2]:
        t.normal_()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    q = torch.randn((3, 2, 64), device=DEV).to(torch.bfloat16)
    args = q, cache, i32([0, 3]), i32([[0, 1, 2]]), i32([70])
    for window, sinks in ((far, 0), (5, far)):
        with pytest.raises(ValueError, match="64 bits"):
            e3.e3_window_attention(*args, window, sinks, 0.125)
    want = e3.e3_window_attention(*args, 70, 0, 0.125)
    for window, sinks in (((1 << 63) - 1, 0), (1, (1 << 63) - 1)):
        assert all(torch.equal(a, b) for a, b in zip(e3.e3_window_attention(*args, window, sinks, 0.125), want))
