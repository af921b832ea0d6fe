"""Beam search: the selection over beams and vocabulary, the reordering of the beams' pages and the copies of their last ones.

Selected beams and tokens are compared exactly with the definition in 64 bits (neighbours within 2e-6 of each other are decided in fp64 by
the kernel).  A score is that of the definition up to the fp32 sums' error, 2e-6, and its rounding, 2^-24 of it."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2505_18573_amd as e3
from tests.test_kv_cache import cache_struct

DEV = "cuda:0"


def test_argument_checks_without_gpu():
    L = e3.lib()
    need = e3.e3_beam_workspace_bytes(3, 4, 100)
    assert need > 0
    for bad in ((0, 4, 100), (-1, 4, 100), (3, 0, 100), (3, 33, 100), (3, 4, 0), (3, 4, 1 << 21), (1 << 22, 1, 1), (1 << 21, 32, 1 << 20)):
        assert e3.e3_beam_workspace_bytes(*bad) == 0

    def call(z=0x1000, dtype=1, seqs=3, beams=4, V=100, strides=(416, 104), scores=0x2000, keep=8, tau=1.0, fin=None, eos=-1, parent=0x3000,
             token=0x4000, score=0x5000, ws=0x10000, ws_bytes=need):
        return L.e3_beam_select(z, dtype, seqs, beams, V, *strides, scores, keep, tau, fin, eos, parent, token, score, ws, ws_bytes, None)

    assert call(dtype=2) == -3
    assert call(seqs=-1) == -2 and call(beams=0) == -2 and call(beams=33) == -2 and call(V=0) == -2 and call(V=1 << 21) == -2
    assert call(keep=0) == -2 and call(keep=65) == -2 and call(strides=(416, 96)) == -2 and call(seqs=1 << 22, ws_bytes=1 << 60) == -2
    assert call(tau=0.0) == -5 and call(tau=float("nan")) == -5 and call(tau=float("inf")) == -5
    assert call(fin=0x6000) == -5 and call(fin=0x6000, eos=100) == -5
    for name in ("z", "scores", "parent", "token", "score"):
        assert call(**{name: None}) == -1
    assert call(ws=None) == -6 and call(ws_bytes=need - 1) == -6
    assert call(z=0x1008) == -4 and call(ws=0x10010) == -4 and call(strides=(412, 104)) == -4 and call(dtype=0, strides=(416, 102)) == -4
    assert call(seqs=0, z=None, scores=None, parent=None, ws=None) == 0

    def reorder(parent=0x1000, seqs=3, beams=4, pages=0x2000, width=5, lens=0x3000, page=64, out=(0x4000, 0x5000, 0x6000, 0x7000, 0x8000)):
        return L.e3_beam_reorder(parent, seqs, beams, pages, width, lens, page, *out, None)

    assert reorder(seqs=-1) == -2 and reorder(beams=0) == -2 and reorder(beams=33) == -2 and reorder(width=-1) == -2 and reorder(seqs=1 << 24) == -2
    assert reorder(page=48) == -2 and reorder(page=16) == -2
    assert reorder(parent=None) == -1 and reorder(pages=None) == -1 and reorder(lens=None) == -1
    for i in range(5):
        assert reorder(out=tuple(None if i == j else 0x4000 + 64 * j for j in range(5))) == -1
    assert reorder(pages=0x4000) == -5 and reorder(lens=0x5000) == -5
    assert reorder(seqs=0, parent=None, lens=None) == 0

    def copy(c, src=0x1000, dst=0x2000, counts=0x3000, n=4):
        return L.e3_cache_copy(C.byref(c) if c is not None else None, src, dst, counts, n, None)

    assert copy(None) == -1 and copy(cache_struct(page=48)) == -2 and copy(cache_struct(dtype=0)) == -3 and copy(cache_struct(k=0x10008)) == -4
    assert copy(cache_struct(), n=-1) == -2 and copy(cache_struct(), n=1 << 24) == -2 and copy(cache_struct(heads=64), n=1 << 18) == -2
    assert copy(cache_struct(), src=None) == -1 and copy(cache_struct(), dst=None) == -1 and copy(cache_struct(), counts=None) == -1
    assert copy(cache_struct(), n=0, src=None, dst=None, counts=None) == 0


def reference(z, scores, keep, tau, finished=None, eos=-1):
    z, scores = z.double().cpu(), scores.double().cpu()
    n, B, V = z.shape
    parent, token = (torch.full((n, keep), -1, dtype=torch.int32) for _ in range(2))
    score = torch.full((n, keep), -math.inf, dtype=torch.float64)
    for i in range(n):
        rows = []
        for b in range(B):
            x = torch.full((V,), -math.inf, dtype=torch.float64)
            if math.isfinite(scores[i, b]):
                if finished is not None and finished[i, b]:
                    x[eos] = scores[i, b]
                else:
                    a = z[i, b] / tau
                    a = torch.where(z[i, b] <= -1e30, torch.full_like(a, -math.inf), a)
                    total = torch.logsumexp(a, 0)
                    if math.isfinite(total):
                        x = scores[i, b] + a - total
            rows.append(x)
        x = torch.cat(rows).numpy()
        order = np.argsort(-x, kind="stable")[:keep]
        order = order[x[order] > -math.inf]
        m = len(order)
        parent[i, :m], token[i, :m] = torch.from_numpy(order // V).int(), torch.from_numpy(order % V).int()
        score[i, :m] = torch.from_numpy(x[order])
    return parent, token, score


def check(got, want):
    for g, w in zip(got[:2], want[:2]):
        assert g.dtype is torch.int32 and torch.equal(g.cpu(), w), (g.cpu()[(g.cpu() != w).any(1)][:2].tolist(), w[(g.cpu() != w).any(1)][:2].tolist())
    s, w = got[2].cpu().double(), want[2]
    none = w == -math.inf
    assert torch.equal(s == -math.inf, none)
    assert bool(((s - w)[~none].abs() <= 2e-6 + w[~none].abs() * 2.0 ** -24).all())


def padded(n, B, V, dtype, g, scale=3.0):
    per = 8 if dtype is torch.bfloat16 else 4
    z = (torch.randn((n, B, -(-V // per) * per), generator=g) * scale).to(dtype)
    z[..., V:] = float("nan")                                    # behind a row nothing counts
    return z


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [1, 5, 8, 511, 512, 513, 2049, 4096, 4097, 70_005])
@pytest.mark.parametrize("n,B,keep", [(1, 1, 1), (3, 1, 4), (2, 3, 3), (1, 8, 16), (2, 32, 64), (1, 5, 64)])
def test_select(dtype, V, n, B, keep):
    g = torch.Generator().manual_seed(V + B)
    z = padded(n, B, V, dtype, g)
    scores = -5.0 * torch.rand((n, B), generator=g)
    got = e3.e3_beam_select(z.to(DEV)[..., :V], scores.to(DEV), keep, 0.8)
    check(got, reference(z[..., :V], scores, keep, float(np.float32(0.8))))


@pytest.mark.gpu
def test_select_a_model_s_vocabulary():
    g = torch.Generator().manual_seed(1)
    V = 151_936
    z = padded(2, 32, V, torch.bfloat16, g)
    z.scatter_add_(2, torch.randint(0, V, (2, 32, 20), generator=g), torch.full((2, 32, 20), 8.0, dtype=torch.bfloat16))
    scores = -20.0 - 3.0 * torch.rand((2, 32), generator=g)
    want = reference(z, scores, 64, 1.0)
    check(e3.e3_beam_select(z.to(DEV), scores.to(DEV), 64), want)
    check(e3.e3_beam_select(z.to(DEV), scores.to(DEV), 17), [w[:, :17] for w in want])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_equal_values_go_to_the_lowest_index(dtype):
    # a vocabulary of equal logits; few different logits; beams that are the same
    V, g = 3000, torch.Generator().manual_seed(2)
    z = torch.zeros((1, 2, V), dtype=dtype)
    scores = torch.tensor([[-1.0, -1.5]])
    check(e3.e3_beam_select(z.to(DEV), scores.to(DEV), 64), reference(z, scores, 64, 1.0))
    z = torch.randint(0, 3, (3, 4, V), generator=g).to(dtype)
    scores = -torch.rand((3, 4), generator=g)
    check(e3.e3_beam_select(z.to(DEV), scores.to(DEV), 40), reference(z, scores, 40, 1.0))
    z = (torch.randn((2, 1, V), generator=g) * 2).to(dtype).expand(2, 6, V).contiguous()
    scores = torch.full((2, 6), -2.0)
    check(e3.e3_beam_select(z.to(DEV), scores.to(DEV), 30), reference(z, scores, 30, 1.0))
    # zeros of either sign are equal
    z = torch.full((1, 1, V), -4.0, dtype=dtype)
    z[0, 0, 700], z[0, 0, 900] = -0.0, 0.0
    check(e3.e3_beam_select(z.to(DEV), scores[:1, :1].contiguous().to(DEV), 5), reference(z, scores[:1, :1], 5, 1.0))


@pytest.mark.gpu
def test_near_scores_of_two_beams():
    # beams of the same logits in another order, whose fp32 sums differ by rounding, and scores a few 1e-7 apart: fp64 decides
    g, V = torch.Generator().manual_seed(3), 20_000
    one = torch.randn(V, generator=g) * 3
    z = torch.stack([one[torch.randperm(V, generator=g)] for _ in range(4)])[None].repeat(8, 1, 1)
    scores = torch.full((8, 4), -1.0)
    for i in range(8):
        scores[i] += torch.randperm(4, generator=g) * (2.0 ** -23 * (1 + i))
    want = reference(z, scores, 20, 1.0)
    check(e3.e3_beam_select(z.to(DEV), scores.to(DEV), 20), want)
    for keep in (1, 2, 3, 5):                                     # the border lies among them
        check(e3.e3_beam_select(z.to(DEV), scores.to(DEV), keep), [w[:, :keep] for w in want])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("apart", [3, 300, 4000])
def test_near_scores_behind_equal_ones(dtype, apart):
    # Beam 0 has its best logit twice, in one chunk of columns or two; beam 1 the same logits in another order, its score 2^-29 above
    # or below: with the last place taken by one of the equal ones, the candidate next to it is the other, and beam 1's lies behind that.
    g, n, V = torch.Generator().manual_seed(apart), 128, 8192
    z = (torch.randn((n, 2, V), generator=g) * 3).clamp(max=9.0).to(dtype)
    for i in range(n):
        z[i, 0, 17], z[i, 0, 17 + apart] = 10.0, 10.0
        z[i, 1] = z[i, 0, torch.randperm(V, generator=g)]
    scores = torch.zeros((n, 2))
    scores[:, 1] = 2.0 ** -29 * (2 * torch.randint(0, 2, (n,), generator=g) - 1)
    want = reference(z, scores, 3, 1.0)
    for keep in (1, 2, 3):
        check(e3.e3_beam_select(z.to(DEV), scores.to(DEV), keep), [w[:, :keep] for w in want])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_masks_and_values_that_are_no_numbers(dtype):
    g, V = torch.Generator().manual_seed(4), 5000
    z = (torch.randn((6, 4, V), generator=g) * 2).to(dtype)
    z[0, :, 100:] = -math.inf                                     # few tokens allowed, the rest masked one way or another
    z[1, :, 3:] = -1e9
    z[2, 1] = -math.inf                                           # nothing allowed
    z[2, 2, 17:] = -1e30
    z[3, 0, 4000] = float("nan")
    z[3, 3, 5] = math.inf
    z[4] = -math.inf
    z[4, 2, 9], z[4, 2, 4999] = 1.0, 2.0                          # two candidates in all
    z[5] = -math.inf                                              # none
    scores = -torch.rand((6, 4), generator=g)
    got = e3.e3_beam_select(z.to(DEV), scores.to(DEV), 12)
    check(got, reference(z, scores, 12, 1.0))
    assert got[0][4].tolist() == [2, 2] + [-1] * 10 and got[1][4].tolist() == [4999, 9] + [-1] * 10 and not (got[0][5] >= 0).any()


@pytest.mark.gpu
def test_first_steps_and_finished_beams():
    g, V = torch.Generator().manual_seed(5), 700
    z = padded(5, 4, V, torch.bfloat16, g)[..., :V]
    scores = -3.0 * torch.rand((5, 4), generator=g)
    scores[0, 1:] = -math.inf                                     # a first step: one beam
    scores[1, 2] = float("nan")
    scores[2] = -math.inf
    finished = torch.zeros((5, 4), dtype=torch.uint8)
    finished[3, 1] = finished[3, 3] = 1
    finished[4] = 1
    finished[2, 0] = 1
    rows = torch.full((5, 4, 704), float("nan"), dtype=torch.bfloat16)
    rows[..., :V] = z
    rows[finished.bool()] = float("nan")                          # what a finished beam's row holds does not count
    for keep in (4, 8):
        for eos in (0, 650):
            got = e3.e3_beam_select(rows.to(DEV)[..., :V], scores.to(DEV), keep, 0.5, finished.to(DEV), eos)
            check(got, reference(z, scores, keep, 0.5, finished, eos))
    got = e3.e3_beam_select(rows.to(DEV)[..., :V], scores.to(DEV), 4, 0.5, finished.to(DEV), 650)
    assert got[1][4].tolist() == [650] * 4 and torch.equal(got[2][4].cpu(), scores[4].sort(descending=True).values)


@pytest.mark.gpu
def test_select_strides_outputs_graph_and_streams():
    g, V = torch.Generator().manual_seed(6), 1001
    z = padded(4, 6, V, torch.bfloat16, g)
    scores = (-torch.rand((4, 3), generator=g)).to(DEV)
    part = z.to(DEV)[:, 1:6:2, :V]                                # every other beam of a larger tensor
    want = reference(z[:, 1:6:2, :V], scores, 6, 1.0)
    got = e3.e3_beam_select(part, scores, 6)
    check(got, want)
    outs = [torch.full((4, 6), 9, dtype=t.dtype, device=DEV) for t in got]
    ws = torch.full((e3.e3_beam_workspace_bytes(4, 3, V),), 255, dtype=torch.uint8, device=DEV)
    back = e3.e3_beam_select(part, scores, 6, parent_out=outs[0], token_out=outs[1], score_out=outs[2], workspace=ws)
    assert all(a is b for a, b in zip(back, outs)) and all(torch.equal(a, b) for a, b in zip(outs, got))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        e3.e3_beam_select(part, scores, 6, parent_out=outs[0], token_out=outs[1], score_out=outs[2], workspace=ws)
    for i in range(3):
        for t in outs:
            t.zero_()
        ws.fill_(i * 100)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, got))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = e3.e3_beam_select(part, scores, 6)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(again, got))
    assert e3.e3_beam_select(part[:0], scores[:0], 6)[0].shape == (0, 6)


@pytest.mark.gpu
def test_logits_and_pages_behind_four_gigabytes():
    g, V, apart = torch.Generator().manual_seed(8), 1000, (1 << 31) + 8
    z = (torch.randn((2, 3, V), generator=g) * 3).to(torch.bfloat16)
    room = torch.empty(apart + 3 * V, dtype=torch.bfloat16, device=DEV)
    far = room.as_strided((2, 3, V), (apart, V, 1))
    far.copy_(z.to(DEV))
    scores = -torch.rand((2, 3), generator=g)
    check(e3.e3_beam_select(far, scores.to(DEV), 6), reference(z, scores, 6, 1.0))
    del far, room
    pages = 1_060_000
    cache = e3.new_cache(pages, 64, 1, 64, device=DEV)
    for t in cache:
        t[pages - 3].view(torch.uint8).random_(1, 100)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    e3.e3_cache_copy(cache, i32([pages - 3]), i32([pages - 1]), i32([64]))
    for t in cache:
        a, b, c = (t[p].view(torch.uint8) for p in (pages - 3, pages - 1, pages - 2))
        assert torch.equal(a, b) and bool((a > 0).all()) and not bool((c > 0).any())


# ---------------------------------------------------------------- pages
def reordered(parent, table, lens, page):
    """Lists: the new tables and lengths, and (source, destination, tokens) of the copies."""
    n, B = len(parent), len(parent[0])
    width = len(table[0])
    own = [table[r][lens[r] // page] if lens[r] // page < width else -1 for r in range(n * B)]
    pages, out_lens, copies = [], [], []
    for i in range(n):
        of = [p if 0 <= p < B else b for b, p in enumerate(parent[i])]
        free = [b for b in range(B) if b not in of]
        had = set()
        for b in range(B):
            p = i * B + of[b]
            last = own[p] if of[b] not in had else own[i * B + free.pop(0)]
            row = list(table[p])
            if lens[p] // page < width:
                row[lens[p] // page] = last
            n_copy = lens[p] % page
            copies.append((own[p], last, n_copy) if of[b] in had and n_copy and last >= 0 and own[p] >= 0 else (-1, -1, 0))
            had.add(of[b])
            pages.append(row)
            out_lens.append(lens[p])
        assert not free
    return pages, out_lens, copies


@pytest.mark.gpu
@pytest.mark.parametrize("n,B", [(1, 1), (1, 4), (5, 3), (40, 8), (3, 32)])
@pytest.mark.parametrize("kind", [torch.float8_e4m3fn, torch.bfloat16])
def test_reorder_and_copy(n, B, kind):
    g = torch.Generator().manual_seed(n * B)
    page, heads, D, width = 32, 3, 64, 5
    rows = n * B
    lens = torch.randint(0, width * page, (rows,), generator=g).to(torch.int32)
    lens[0] = 64                                                  # at a page's end
    lens[rows // 2] = width * page                                # the table is full
    lens[rows - 1] = 0
    table = torch.randperm(rows * width, generator=g).reshape(rows, width).to(torch.int32)
    parent = torch.randint(-1, B + 1, (n, B), generator=g).to(torch.int32)
    cache = e3.new_cache(rows * width, page, heads, D, kind, DEV)
    for t in cache:
        if t is not None:
            t.view(torch.uint8).copy_(torch.randint(0, 120, t.view(torch.uint8).shape, generator=g).to(torch.uint8))
    before = [t.clone() if t is not None else None for t in cache]
    pages, out_lens, src, dst, counts = e3.e3_beam_reorder(parent.to(DEV), table.to(DEV), lens.to(DEV), page)
    e3.e3_cache_copy(cache, src, dst, counts)
    want, want_lens, copies = reordered(parent.tolist(), table.tolist(), lens.tolist(), page)
    assert pages.tolist() == want and out_lens.tolist() == want_lens
    assert list(zip(src.tolist(), dst.tolist(), counts.tolist())) == copies
    for a, b, m in copies:
        if m:
            m = -(-m // 8) * 8
            before[0][b, :, :m] = before[0][a, :, :m]
            before[1][b, :, :m // 8] = before[1][a, :, :m // 8]
            for t in before[2:]:
                if t is not None:
                    t[b, :, :m] = t[a, :, :m]
    for t, w in zip(cache, before):
        assert (t is None and w is None) or torch.equal(t.view(torch.uint8), w.view(torch.uint8))


@pytest.mark.gpu
def test_copies_that_are_none():
    cache = e3.new_cache(6, 32, 2, 64, device=DEV)
    for t in cache:
        t.view(torch.uint8).random_(0, 100)
    before = [t.clone() for t in cache]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    e3.e3_cache_copy(cache, i32([-1, 6, 0, 2, 1, 3]), i32([0, 1, -1, 1 << 30, 1, 4]), i32([32, 32, 32, 32, 32, -7]))
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(cache, before))
    e3.e3_cache_copy(cache, i32([0]), i32([5]), i32([1000]))       # cut to the page
    assert torch.equal(cache.k[5].view(torch.uint8), before[0][0].view(torch.uint8)) and torch.equal(cache.v_scale[5], before[3][0])
    assert torch.equal(cache.k[4].view(torch.uint8), before[0][4].view(torch.uint8))


@pytest.mark.gpu
@pytest.mark.parametrize("n,B", [(1, 1), (5, 3), (7, 32), (0, 4)])
def test_reordered_tensors_are_apart(n, B):
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=DEV)
    outs = e3.e3_beam_reorder(i32(n, B), i32(n * B, 3), i32(n * B), 32)
    assert [tuple(t.shape) for t in outs] == [(n * B, 3)] + 4 * [(n * B,)]
    assert all(t.dtype is torch.int32 and t.is_contiguous() and t.device == torch.device(DEV) and not t.requires_grad for t in outs)
    for i, t in enumerate(outs):                                  # written one by one, none changes another
        t.fill_(i + 1)
    assert all(bool((t == i + 1).all()) for i, t in enumerate(outs)) and all(torch.equal(t.clone(), t) and t.data_ptr() % 16 == 0 for t in outs)


@pytest.mark.gpu
def test_reorder_into_given_tensors_and_a_graph():
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    parent, table, lens = i32([[1, 1, 0], [2, 2, 2]]), i32(list(range(12))).reshape(6, 2).contiguous(), i32([5, 5, 5, 40, 40, 40])
    want, want_lens, copies = reordered(parent.tolist(), table.tolist(), lens.tolist(), 32)
    outs = [torch.zeros((6, 2), dtype=torch.int32, device=DEV)] + [torch.zeros(6, dtype=torch.int32, device=DEV) for _ in range(4)]
    cache = e3.new_cache(12, 32, 1, 64, torch.bfloat16, DEV)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        e3.e3_beam_reorder(parent, table, lens, 32, *outs)
        e3.e3_cache_copy(cache, *outs[2:])
    for _ in range(3):
        cache.k.normal_()
        cache.v.normal_()
        k = cache.k.clone()
        graph.replay()
        torch.cuda.synchronize()
        assert outs[0].tolist() == want and outs[1].tolist() == want_lens
        assert list(zip(*(t.tolist() for t in outs[2:]))) == copies
        for a, b, m in copies:
            if m:
                assert torch.equal(cache.k[b, :, :-(-m // 8) * 8], k[a, :, :-(-m // 8) * 8])
    with pytest.raises(e3.E3Error):
        e3.e3_beam_reorder(parent, table, lens, 32, pages_out=table)
