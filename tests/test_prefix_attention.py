"""Attention of a decode step over a paged cache, rows of a group sharing a prefix, against plain attention in 64 bits.

Tolerance of an output: it is rounded to bf16 (2^-8 |out| at most, and |out| <= sum p|v|); the weights have sixteen bits and all
else is fp32: scores of at most 40 in magnitude with 128 products, relative weight errors below 1e-4.  So
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
    need = e3.e3_prefix_attention_workspace_bytes(4, 1, 4, 2, 128, 2)
    assert need > 0
    assert e3.e3_prefix_attention_workspace_bytes(4, 1, 5, 2, 128, 2) == 0       # heads do not divide
    assert e3.e3_prefix_attention_workspace_bytes(4, 0, 4, 2, 128, 2) == 0
    assert e3.e3_prefix_attention_workspace_bytes(4, 1, 4, 2, 96, 2) == 0
    assert e3.e3_prefix_attention_workspace_bytes(-1, 1, 4, 2, 128, 2) == 0

    def call(c=cache_struct(), q=0x1000, rows=4, T=1, heads=4, strides=(512, 512, 128), off=0x2000, groups=2, pp=0x3000,
             pw=3, pl=0x4000, rp=0x5000, rw=2, rl=0x6000, scale=0.1, out=0x7000, ws=0x10000, ws_bytes=need):
        return L.e3_prefix_attention(C.byref(c), q, rows, T, heads, *strides, off, groups, pp, pw, pl, rp, rw, rl, scale, out, None,
                                     ws, ws_bytes, None)

    assert call(c=cache_struct(page=24)) == -2 and call(c=cache_struct(dtype=0)) == -3 and call(c=cache_struct(v=None)) == -1
    assert call(heads=5) == -2 and call(T=0) == -2 and call(rows=-1) == -2 and call(groups=-1) == -2 and call(rw=-1) == -2
    assert call(rows=1 << 20, T=1 << 10, heads=4) == -2
    assert call(scale=0.0) == -5 and call(scale=float("nan")) == -5 and call(scale=float("inf")) == -5
    for name in ("q", "out", "rl", "rp", "off", "pl", "pp"):
        assert call(**{name: None}) == -1
    assert call(ws=None) == -6 and call(ws_bytes=need - 1) == -6
    assert call(q=0x1008) == -4 and call(ws=0x10010) == -4 and call(strides=(512, 512, 132)) == -4
    assert call(rows=0, q=None, out=None, rl=None, ws=None) == 0


def test_shapes_beyond_a_launch_are_refused():
    # 2^24 rows times key heads: the join would pass 2^32 threads
    assert e3.e3_prefix_attention_workspace_bytes((1 << 23) - 1, 1, 2, 2, 64, 0) > 0
    assert e3.e3_prefix_attention_workspace_bytes(1 << 23, 1, 2, 2, 64, 0) == 0


class Step:
    """One decode step's inputs, and its keys and values in 64 bits."""

    def __init__(self, sizes, prefix, rows_len, T, R, H, D, page, cache_type, seed=0, poison=True, grouped=True, spare=0, loud=1.0):
        g = torch.Generator().manual_seed(seed)
        rows, G = sum(sizes), len(sizes)
        wide = lambda n: max(1, -(-max(n, default=0) // page))
        pw, rw = wide(prefix), wide(rows_len)
        pages = G * pw + rows * rw + spare
        order = torch.randperm(G * pw + rows * rw, generator=g) + spare
        self.pp, self.rp = order[:G * pw].reshape(G, pw), order[G * pw:].reshape(rows, rw)
        self.sizes, self.prefix, self.rows_len, self.T, self.R, self.H, self.D, self.page = sizes, prefix, rows_len, T, R, H, D, page
        self.rows, self.G, self.grouped = rows, G, grouped
        self.q = (torch.randn((rows, T, H * R, D), generator=g) * loud).to(BF16)
        self.scale = D ** -0.5
        self.cache = e3.new_cache(pages, page, H, D, cache_type, DEV)
        if poison:                                       # what lies behind the lengths is no number
            for t in self.cache:
                if t is not None:
                    t.view(torch.uint8).fill_(255)
        self.kp, self.vp = zip(*[self.fill(self.pp[i], n, g) for i, n in enumerate(prefix)]) if G else ((), ())
        self.kr, self.vr = zip(*[self.fill(self.rp[i], n, g) for i, n in enumerate(rows_len)])
        self.offsets = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32)

    def fill(self, pages, n, g):
        x = [torch.randn((n, self.H, self.D), generator=g).to(BF16) for _ in range(2)]
        if n:
            at = torch.arange(n)
            slots = (pages[at // self.page] * self.page + at % self.page).to(DEV)
            e3.e3_cache_append(self.cache, x[0].to(DEV), x[1].to(DEV), slots)
            x = [t.cpu() for t in e3.e3_cache_read(self.cache, slots, torch.float32)]
        return x[0].double(), x[1].double()

    def args(self):
        i32 = lambda t: torch.as_tensor(t, dtype=torch.int32).contiguous().to(DEV)
        if not self.grouped:
            return self.cache, None, None, None, i32(self.rp), i32(self.rows_len), self.scale
        return self.cache, i32(self.offsets), i32(self.pp), i32(self.prefix), i32(self.rp), i32(self.rows_len), self.scale

    def reference(self):
        """out, sum p|v| and lse in 64 bits."""
        Hq = self.H * self.R
        out = torch.zeros((self.rows, self.T, Hq, self.D), dtype=torch.float64)
        size, lse = torch.zeros_like(out), torch.full((self.rows, self.T, Hq), -math.inf, dtype=torch.float64)
        group = np.repeat(np.arange(self.G), self.sizes)
        for r in range(self.rows):
            for t in range(self.T):
                own = max(0, self.rows_len[r] - (self.T - 1 - t))
                k, v = self.kr[r][:own], self.vr[r][:own]
                if self.grouped:
                    k, v = torch.cat([self.kp[group[r]], k]), torch.cat([self.vp[group[r]], v])
                if not k.shape[0]:
                    continue
                for h in range(Hq):
                    s = k[:, h // self.R] @ self.q[r, t, h].double() * self.scale
                    p = torch.softmax(s, 0)
                    out[r, t, h], size[r, t, h] = p @ v[:, h // self.R], p @ v[:, h // self.R].abs()
                    lse[r, t, h] = torch.logsumexp(s, 0)
        return out, size, lse

    def check(self, got, lse):
        want, size, want_lse = self.reference()
        err = (got.double().cpu() - want).abs()
        bound = (2.0 ** -8 + 1e-4) * size
        assert bool((err <= bound).all()), float((err / bound.clamp(min=1e-30)).max())
        none = want_lse == -math.inf
        lse = lse.double().cpu()
        assert torch.equal(lse == -math.inf, none)
        assert bool(((lse - want_lse)[~none].abs() <= 2e-5).all()), float((lse - want_lse)[~none].abs().max())


EDGES = [0, 1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 300]


@pytest.mark.gpu
@pytest.mark.parametrize("cache_type", [FP8, BF16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("R,T", [(1, 1), (7, 1), (16, 1), (1, 3), (4, 5), (17, 1), (8, 5), (13, 7)])
def test_lengths_heads_and_queries(cache_type, D, R, T):
    # own lengths and prefixes on both sides of a step of 32 tokens, a page and a round of four waves; groups of 0 to 9 rows;
    # 1 to 91 queries of a row and key head: one, two, three and more tiles of 16
    sizes = [1, 0, 3, 9, 1]
    rows_len = EDGES[:sum(sizes)]
    prefix = [0, 5, 33, 131, 64]
    s = Step(sizes, prefix, rows_len, T, R, 2, D, 32 if R % 2 else 64, cache_type, seed=R * 10 + T)
    out, lse = e3.e3_prefix_attention(s.q.to(DEV), *s.args())
    s.check(out, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("cache_type", [FP8, BF16])
def test_no_groups_and_rows_without_any_key(cache_type):
    s = Step([4], [0], [0, 1, 40, 0], 1, 3, 1, 64, 32, cache_type, grouped=False)
    out, lse = e3.e3_prefix_attention(s.q.to(DEV), *s.args())
    s.check(out, lse)
    assert bool((out[0] == 0).all()) and bool((lse[0] == -math.inf).all())
    # groups that do not begin at row 0, and end before the last: the others have no prefix
    t = Step([2, 2], [40, 70], [3, 0, 33, 9], 2, 2, 2, 128, 32, cache_type)
    args = list(t.args())
    args[1] = torch.tensor([1, 1, 3], dtype=torch.int32, device=DEV)
    out, lse = e3.e3_prefix_attention(t.q.to(DEV), *args)
    for r, group in ((0, None), (1, 1), (2, 1), (3, None)):
        one = Step([1], [0], [t.rows_len[r]], 2, 2, 2, 128, 32, cache_type)
        one.q, one.kr, one.vr = t.q[r:r + 1], t.kr[r:r + 1], t.vr[r:r + 1]
        one.kp, one.vp = (t.kp[group:group + 1], t.vp[group:group + 1]) if group is not None else (one.kp, one.vp)
        one.check(out[r:r + 1], lse[r:r + 1])


@pytest.mark.gpu
@pytest.mark.parametrize("groups", [64, 65, 130, 4200])
def test_many_groups(groups):
    # a row finds its group among more than 64, and more than 64 * 64, of them; most are empty where there are very many
    sizes = [(g * 7 % 3 if groups < 1000 else int(g % 17 == 3 or g == groups - 1)) for g in range(groups)]
    prefix = [1 + g * 5 % 40 for g in range(groups)]
    rows_len = [r % 35 for r in range(sum(sizes))]
    s = Step(sizes, prefix, rows_len, 1, 3, 1, 64, 64, FP8, seed=groups)
    out, lse = e3.e3_prefix_attention(s.q.to(DEV), *s.args())
    s.check(out, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("cache_type,H,prefix,rows_len", [
    (FP8, 8, 40_003, [7, 1200, 0]),          # a long prefix in many runs, joined for every row
    (BF16, 2, 3, [150_017, 20, 33]),         # a long row of its own
])
def test_long_axes_are_cut_and_joined(cache_type, H, prefix, rows_len):
    s = Step([3], [prefix], rows_len, 1, 2, H, 128, 128, cache_type, seed=3)
    out, lse = e3.e3_prefix_attention(s.q.to(DEV), *s.args())
    s.check(out, lse)


@pytest.mark.gpu
def test_many_rows():
    rng = np.random.default_rng(0)
    sizes = rng.integers(0, 7, 500).tolist()
    n = sum(sizes)
    s = Step(sizes, rng.integers(0, 60, 500).tolist(), rng.integers(0, 50, n).tolist(), 1, 2, 1, 64, 32, FP8, seed=5)
    out, lse = e3.e3_prefix_attention(s.q.to(DEV), *s.args())
    s.check(out, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("loud", [8.0, 0.0])
def test_scores_that_are_far_apart_and_all_equal(loud):
    s = Step([3], [200], [100, 7, 64], 1, 4, 2, 128, 64, FP8, seed=9, loud=loud)
    out, lse = e3.e3_prefix_attention(s.q.to(DEV), *s.args())
    s.check(out, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("cache_type", [FP8, BF16])
def test_values_that_are_no_number_stay_where_they_are_seen(cache_type):
    # the last two of the three drafted tokens hold NaN and inf: queries that do not see them are not touched
    s = Step([2], [37], [50, 34], 3, 2, 2, 64, 32, cache_type, seed=4)
    for r, n in enumerate(s.rows_len):
        for back, bad in ((1, math.nan), (2, math.inf)):
            slot = torch.tensor([s.rp[r, (n - back) // 32] * 32 + (n - back) % 32], device=DEV)
            x = torch.full((1, 2, 64), bad, dtype=torch.float32, device=DEV)
            k = s.kr[r][n - back][None].float().to(DEV)
            e3.e3_cache_append(s.cache, k, x, slot)
    out, lse = e3.e3_prefix_attention(s.q.to(DEV), *s.args())
    want, size, want_lse = s.reference()
    err = (out[:, 0].double().cpu() - want[:, 0]).abs()
    assert bool((err <= (2.0 ** -8 + 1e-4) * size[:, 0]).all())
    assert bool((~torch.isfinite(out[:, 1:])).all())
    assert bool(((lse.double().cpu() - want_lse).abs() <= 2e-5).all())           # the keys are numbers
    # a key that is no number: the queries that see it are no numbers, the others are not touched
    slot = torch.tensor([s.rp[0, 49 // 32] * 32 + 49 % 32], device=DEV)
    e3.e3_cache_append(s.cache, torch.full((1, 2, 64), math.nan, device=DEV), torch.ones((1, 2, 64), device=DEV), slot)
    out2, lse2 = e3.e3_prefix_attention(s.q.to(DEV), *s.args())
    assert torch.equal(out2[:, 0], out[:, 0]) and torch.equal(lse2[:, :2], lse[:, :2])
    assert bool(torch.isnan(out2[0, 2]).all()) and bool(torch.isnan(lse2[0, 2]).all())


@pytest.mark.gpu
def test_pages_outside_the_cache_hide_their_tokens_and_lengths_end_with_the_tables():
    s = Step([2], [70], [90, 40], 1, 2, 2, 64, 32, FP8, seed=6)
    args = list(s.args())
    args[2] = args[2].clone()
    args[2][0, 1] = -1                                   # tokens 32 .. 63 of the prefix
    args[4] = args[4].clone()
    args[4][0, 0] = 1 << 30                              # tokens 0 .. 31 of row 0
    s.kp = [torch.cat([s.kp[0][:32], s.kp[0][64:]])]
    s.vp = [torch.cat([s.vp[0][:32], s.vp[0][64:]])]
    s.kr, s.vr = [s.kr[0][32:], s.kr[1]], [s.vr[0][32:], s.vr[1]]
    s.rows_len = [58, 40]
    out, lse = e3.e3_prefix_attention(s.q.to(DEV), *args)
    s.check(out, lse)
    t = Step([1], [32], [64], 1, 1, 1, 64, 32, BF16, seed=7)
    args = list(t.args())
    args[3] = torch.tensor([1 << 30], dtype=torch.int32, device=DEV)
    args[5] = torch.tensor([1 << 30], dtype=torch.int32, device=DEV)
    out, lse = e3.e3_prefix_attention(t.q.to(DEV), *args)
    t.check(out, lse)
    args[3] = torch.tensor([-5], dtype=torch.int32, device=DEV)
    args[5] = torch.tensor([-1], dtype=torch.int32, device=DEV)
    out, lse = e3.e3_prefix_attention(t.q.to(DEV), *args)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


@pytest.mark.gpu
def test_elements_behind_2_to_the_32():
    H, D, page = 8, 128, 128
    s = Step([2], [150], [100, 3], 1, 1, H, D, page, FP8, seed=8, spare=2 ** 32 // (H * D * page), poison=False)
    out, lse = e3.e3_prefix_attention(s.q.to(DEV), *s.args())
    s.check(out, lse)


@pytest.mark.gpu
def test_strides_given_outputs_streams_and_repeats():
    s = Step([3, 2], [100, 37], [50, 0, 33, 129, 64], 2, 3, 2, 64, 64, FP8, seed=2)
    args = s.args()
    first, first_lse = e3.e3_prefix_attention(s.q.to(DEV), *args)
    # queries as part of the projection's output; rows and heads in another order in memory
    wide = torch.randn((5, 2, 10, 64), device=DEV).to(BF16)
    wide[:, :, 2:8] = s.q.to(DEV)
    turned = s.q.to(DEV).permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
    need = e3.e3_prefix_attention_workspace_bytes(5, 2, 6, 2, 64, 2)
    ws = torch.randint(0, 255, (need,), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    for q in (wide[:, :, 2:8], turned):
        out, lse = torch.full_like(first, math.nan), torch.full_like(first_lse, math.nan)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = e3.e3_prefix_attention(q, *args, out=out, lse_out=lse, workspace=ws)
        torch.cuda.current_stream().wait_stream(side)
        assert got[0] is out and got[1] is lse
        assert torch.equal(out, first) and torch.equal(lse, first_lse)
    assert e3.e3_prefix_attention(s.q.to(DEV), *args, want_lse=False)[1] is None
    assert e3.e3_prefix_attention(torch.empty((0, 1, 6, 64), dtype=BF16, device=DEV), s.cache, None, None, None,
                                  torch.empty((0, 1), dtype=torch.int32, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV),
                                  0.1)[0].shape == (0, 1, 6, 64)
    with pytest.raises(ValueError):
        e3.e3_prefix_attention(s.q.to(DEV)[..., :32], *args)
    with pytest.raises(ValueError):
        e3.e3_prefix_attention(s.q.to(DEV).float(), *args)
    with pytest.raises(ValueError):
        e3.e3_prefix_attention(s.q.to(DEV), args[0], args[1], args[2][:1], *args[3:])
    with pytest.raises(e3.E3Error) as err:
        e3.e3_prefix_attention(s.q.to(DEV), *args, workspace=ws[:1024])
    assert err.value.status == -6
    with pytest.raises(e3.E3Error) as err:
        e3.e3_prefix_attention(s.q.to(DEV)[:, :, :5], *args)
    assert err.value.status == -2


@pytest.mark.gpu
def test_replayed_from_a_graph_with_other_lengths():
    s = Step([2, 2], [100, 37], [50, 10, 33, 129], 1, 3, 2, 64, 64, FP8, seed=12)
    q, args = s.q.to(DEV), s.args()
    ws = torch.empty(e3.e3_prefix_attention_workspace_bytes(4, 1, 6, 2, 64, 2), dtype=torch.uint8, device=DEV)
    out, lse = e3.e3_prefix_attention(q, *args, workspace=ws)
    out2, lse2 = torch.empty_like(out), torch.empty_like(lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        e3.e3_prefix_attention(q, *args, out=out2, lse_out=lse2, workspace=ws)
    for lens in ([50, 10, 33, 129], [1, 0, 30, 65], [50, 1, 2, 128]):
        args[5].copy_(torch.tensor(lens, dtype=torch.int32))
        want, want_lse = e3.e3_prefix_attention(q, *args)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out2, want) and torch.equal(lse2, want_lse)
