"""Rotary positions: rows of heads turned (forward and backward), and the keys of a cache turned on the way in.

The kernels take angles in turns with an error far below fp32's, and sine and cosine in fp32: z = theta - quarter turns carries three
roundings (2^-24 of at most pi / 4 each), the polynomials less than four more, so each of them is off by at most 6 x 2^-24.
A turned element is two products and a sum: |error| <= (|x1| + |x2|) (6 + 2) 2^-24 = (|x1| + |x2|) 2^-21, and half a step
of the output's type."""
import ctypes as C
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2505_18573_amd as e3
from tests.test_kv_cache import quantised

DEV = "cuda:0"
TRIG = 2.0 ** -21
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def turned(x, freqs, axis, positions, neighbours, inverse=False):
    """x [tokens, heads, D] in 64 bits, and the sum of magnitudes that an element was made of."""
    x = x.double().cpu()
    n = freqs.numel()
    freqs, positions = freqs.cpu(), positions.cpu().reshape(-1, x.shape[0])
    axis = torch.zeros(n, dtype=torch.int64) if axis is None else axis.cpu().long()
    there = axis < positions.shape[0]
    angle = positions[axis.clamp(max=positions.shape[0] - 1)].double().t() * freqs * there       # [tokens, n]
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None] * (-1.0 if inverse else 1.0)
    at = torch.arange(n)
    a, b = (2 * at, 2 * at + 1) if neighbours else (at, at + n)
    y, size = x.clone(), x.abs()
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return y, size


def rotary_of(rot, axes, neighbours, dev, spread=False):
    n = rot // 2
    freqs = torch.tensor([10000.0 ** (-i / n) for i in range(n)], dtype=torch.float64, device=dev)
    axis = None
    if axes > 1:
        axis = (torch.arange(n) % axes if spread else torch.arange(n) * axes // n).to(torch.uint8).to(dev)
    return e3.E3Rotary(freqs, axis, neighbours)


def cache_struct(k=0x10000, v=0x20000, ks=0x30000, vs=0x40000, pages=4, page=64, heads=2, dim=128, dtype=2):
    return e3.binding._CacheStruct(k, v, ks, vs, pages, page, heads, dim, dtype)


def test_argument_checks_without_gpu():
    L = e3.lib()

    def struct(freqs=0x1000, axis=None, rot=64, axes=1, neighbours=0):
        return e3.binding._RotaryStruct(freqs, axis, rot, axes, neighbours)

    def rotate(r, pos=0x2000, x=0x3000, dtype=1, tokens=3, heads=2, dim=128, xs=(256, 128), out=0x4000, os=(256, 128), inverse=0):
        return L.e3_rotate(C.byref(r) if r is not None else None, pos, 0, x, dtype, tokens, heads, dim, *xs, out, *os, inverse, None)

    def append(r, pos=0x2000, x=0x3000, dtype=1, tokens=3, heads=2, xs=(256, 128), out=0x4000, os=(256, 128), c=None, slots=0x5000, k=0x6000):
        c = cache_struct() if c is None else c
        return L.e3_cache_append_rotated(C.byref(c), C.byref(r) if r is not None else None, pos, 0, x, k, 0x7000, dtype, tokens, heads, *xs,
                                         256, 128, 256, 128, slots, out, *os, None)

    for call in (rotate, append):
        assert call(None) == -1
        for bad in (dict(rot=8), dict(rot=0), dict(rot=24), dict(rot=144), dict(axes=0), dict(axes=9, axis=0x10)):
            assert call(struct(**bad)) == -2
        assert call(struct(neighbours=2)) == -5
        assert call(struct(freqs=None)) == -1 and call(struct(axes=2)) == -1 and call(struct(freqs=0x1004)) == -4
        assert call(struct(), dtype=2) == -3 and call(struct(), tokens=-1) == -2 and call(struct(), tokens=(1 << 25) + 1) == -2
        assert call(struct(), heads=-1) == -2 and call(struct(), heads=65537) == -2
        assert call(struct(), pos=None) == -1 and call(struct(), x=None) == -1 and call(struct(), out=None) == -1
        assert call(struct(), pos=0x2004) == -4 and call(struct(), x=0x3008) == -4 and call(struct(), out=0x4002) == -4
        assert call(struct(), xs=(250, 128)) == -4 and call(struct(), os=(256, 130), dtype=0) == -4
        assert call(struct(), out=0x3000, os=(512, 128)) == -5 and call(struct(), out=0x3000, os=(256, 256)) == -5
        assert call(struct(), tokens=0, pos=None, x=None, out=None) == 0
    assert rotate(struct(), heads=0, x=None, out=None) == 0
    assert rotate(struct(), dim=1032) == -2 and rotate(struct(), dim=60) == -2 and rotate(struct(rot=16), dim=8) == -2
    assert rotate(struct(), inverse=2) == -5
    assert append(struct(), c=cache_struct(page=48)) == -2 and append(struct(), c=cache_struct(dtype=0)) == -3
    assert append(struct(), slots=None) == -1 and append(struct(), k=None) == -1
    assert append(struct(), c=cache_struct(heads=16), tokens=(1 << 24) + 1) == -2


def test_binding_refuses():
    with pytest.raises(ValueError):
        e3.new_rotary(24, device="cpu")
    with pytest.raises(ValueError):
        e3.new_rotary(32, sections=(4, 4), device="cpu")
    r = e3.new_rotary(32, sections=(10, 4, 2), device="cpu")
    assert r.axis.tolist() == [0] * 10 + [1] * 4 + [2] * 2 and r.freqs.dtype is torch.float64 and r.freqs[1] == 10000.0 ** (-1 / 16)
    with pytest.raises(ValueError):
        e3.e3_rotate(torch.zeros(2, 1, 32), r, torch.zeros(3, 2, dtype=torch.int64))            # on the host


def test_the_reference_turns():
    # a quarter turn, and the gradient against differences
    x = torch.randn(3, 2, 32, dtype=torch.float64, generator=torch.Generator().manual_seed(1))
    f = torch.full((16,), math.pi / 2, dtype=torch.float64)
    y, _ = turned(x, f, None, torch.tensor([1, 2, 0]), False)
    assert torch.allclose(y[0, :, :16], -x[0, :, 16:]) and torch.allclose(y[1], -x[1]) and torch.equal(y[2], x[2])
    r = rotary_of(32, 2, True, "cpu")
    pos = torch.tensor([[5, -7, 100], [0, 3, 9]])
    w = torch.randn(3, 2, 32, dtype=torch.float64, generator=torch.Generator().manual_seed(2))
    grad, _ = turned(w, r.freqs, r.axis, pos, True, inverse=True)
    step = torch.randn(3, 2, 32, dtype=torch.float64, generator=torch.Generator().manual_seed(3))
    diff = ((turned(x + step, r.freqs, r.axis, pos, True)[0] - turned(x - step, r.freqs, r.axis, pos, True)[0]) * w).sum() / 2
    assert abs(float((grad * step).sum() - diff)) < 1e-9


def check(got, want, size, dtype):
    allowed = size * TRIG + (want.abs() + size * TRIG) * HALF_STEP[dtype] + 1e-38
    off = (got.double().cpu() - want).abs()
    assert bool((off <= allowed).all()), float((off / allowed).max())


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [1, 5, 129, 1030])
@pytest.mark.parametrize("heads,D,rot", [(1, 16, 16), (3, 64, 64), (7, 80, 32), (28, 128, 128), (2, 256, 192), (1, 1024, 1024), (40, 24, 16)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rotate(tokens, heads, D, rot, dtype):
    g = torch.Generator().manual_seed(tokens + D)
    for neighbours in (False, True):
        for axes, inverse in ((1, False), (3, True)):
            r = rotary_of(rot, axes, neighbours, DEV, spread=neighbours)
            x = (torch.randn((tokens, heads, D), generator=g) * torch.exp(torch.randn((tokens, heads, 1), generator=g) * 2)).to(dtype)
            pos = torch.randint(-5, 100_000, (axes, tokens), generator=g)
            y = e3.e3_rotate(x.to(DEV), r, pos.to(DEV) if axes > 1 else pos[0].to(DEV), inverse=inverse)
            assert y.dtype is dtype and y.shape == x.shape
            want, size = turned(x, r.freqs, r.axis, pos, neighbours, inverse)
            check(y, want, size, dtype)
            assert torch.equal(y.cpu()[..., rot:], x[..., rot:])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rotate_strides_and_places(dtype):
    g = torch.Generator().manual_seed(4)
    n, H, D = 37, 5, 64
    r = rotary_of(48, 2, False, DEV)
    pos = torch.randint(0, 999, (2, n), generator=g)
    big = torch.randn((n, H + 3, D), generator=g).to(dtype)
    want, size = turned(big[:, 1:1 + H], r.freqs, r.axis, pos, False)
    # a part of a wider tensor, positions as rows of a longer table, heads before tokens in the output
    x = big.to(DEV)
    table = torch.zeros((2, n + 11), dtype=torch.int64, device=DEV)
    table[:, 4:4 + n] = pos.to(DEV)
    out = torch.zeros((H, n, D), dtype=dtype, device=DEV).transpose(0, 1)
    y = e3.e3_rotate(x[:, 1:1 + H], r, table[:, 4:4 + n], out=out)
    assert y is out
    check(y, want, size, dtype)
    # in place: the neighbours stay
    e3.e3_rotate(x[:, 1:1 + H], r, pos.to(DEV), out=x[:, 1:1 + H])
    check(x[:, 1:1 + H], want, size, dtype)
    assert torch.equal(x[:, 0].cpu(), big[:, 0]) and torch.equal(x[:, 1 + H:].cpu(), big[:, 1 + H:]) and torch.equal(x[:, 1:1 + H], y)
    # and back
    back = e3.e3_rotate(y, r, pos.to(DEV), inverse=True)
    off = (back.double().cpu() - big[:, 1:1 + H].double()).abs()
    assert bool((off <= 2 * size * (TRIG + HALF_STEP[dtype]) * 2).all())
    # a pair without an axis stays, an empty batch does nothing
    axis = r.axis.clone()
    axis[3] = 2
    y = e3.e3_rotate(big.to(DEV), e3.E3Rotary(r.freqs, axis), pos.to(DEV))
    assert torch.equal(y[..., 3].cpu(), big[..., 3]) and torch.equal(y[..., 3 + 24].cpu(), big[..., 3 + 24])
    assert e3.e3_rotate(big[:0].to(DEV), r, pos[:, :0].to(DEV)).shape == (0, H + 3, D)


@pytest.mark.gpu
def test_more_than_four_gigabytes():
    n, H, D = (1 << 21) + 5, 9, 128                               # of bf16, in place
    r = rotary_of(D, 1, False, DEV)
    g = torch.Generator().manual_seed(11)
    x = torch.zeros((n, H, D), dtype=torch.bfloat16, device=DEV)
    assert x.numel() * 2 > 1 << 32
    pos = torch.arange(n, device=DEV)
    some = torch.tensor([0, 1, (1 << 20) + 3, n - 2, n - 1])
    part = torch.randn((len(some), H, D), generator=g).to(torch.bfloat16)
    x[some.to(DEV)] = part.to(DEV)
    assert e3.e3_rotate(x, r, pos, x) is x
    want, size = turned(part, r.freqs, r.axis, some[None], False)
    check(x[some.to(DEV)], want, size, torch.bfloat16)


@pytest.mark.gpu
def test_far_positions():
    # the angle of a position near 2^50, taken in rational numbers
    pi = Fraction("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803482534211706798")
    freqs = torch.tensor([1.0, 0.7, 1e-3, 1e-7, 3.0, 1e-12, 0.1, 2.0 ** -30], dtype=torch.float64)
    pos = torch.tensor([0, 1, 999_983, 2 ** 31 + 5, 2 ** 40 + 12345, 2 ** 50 + 7, -2 ** 49 - 3])
    x = torch.zeros((len(pos), 1, 16))
    x[..., :8] = 1.0                                            # out: the cosine, then the sine
    y = e3.e3_rotate(x.to(DEV), e3.E3Rotary(freqs.to(DEV)), pos.to(DEV)).cpu().double()
    for t, p in enumerate(pos.tolist()):
        for i, f in enumerate(freqs.tolist()):
            theta = Fraction(p) * Fraction(f)
            theta = float(theta - 2 * pi * round(theta / (2 * pi)))
            assert abs(float(y[t, 0, i]) - math.cos(theta)) <= TRIG and abs(float(y[t, 0, 8 + i]) - math.sin(theta)) <= TRIG


@pytest.mark.gpu
def test_values_that_are_no_numbers():
    x = torch.ones((3, 2, 32), device=DEV)
    x[1, 0, 5] = float("nan")
    x[2, 1, 20] = float("inf")
    r = rotary_of(16, 1, False, DEV)
    y = e3.e3_rotate(x, r, torch.tensor([3, 4, 5], device=DEV))
    bad = ~torch.isfinite(y)
    assert bad.sum() == 3 and bad[1, 0, 5] and bad[1, 0, 13] and bad[2, 1, 20]       # the pair; a column that is copied


def step_inputs(n, q_heads, heads, D, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, q_heads + 2 * heads, D), generator=g) * torch.exp(torch.randn((n, q_heads + 2 * heads, 1), generator=g))
    return x.to(dtype), g


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 8, 9, 203])
@pytest.mark.parametrize("q_heads,heads,D,rot", [(4, 1, 64, 64), (6, 3, 64, 32), (28, 4, 128, 128), (5, 5, 128, 48), (0, 2, 128, 128)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", [torch.float8_e4m3fn, torch.bfloat16])
def test_append_rotated(n, q_heads, heads, D, rot, dtype, kind):
    x, g = step_inputs(n, q_heads, heads, D, dtype, n + rot)
    pages = 16
    slots = torch.randperm(pages * 32, generator=g)[:n] if n % 2 else torch.arange(n) + 5
    slots[n // 2] = -1 if n > 1 else slots[n // 2]
    for neighbours, axes in ((False, 1), (True, 3), (False, 2)):
        r = rotary_of(rot, axes, neighbours, DEV, spread=axes == 2)
        pos = torch.randint(0, 70_000, (axes, n), generator=g)
        xd = x.to(DEV)
        q, k, v = xd[:, :q_heads], xd[:, q_heads:q_heads + heads], xd[:, q_heads + heads:]
        cache = e3.new_cache(pages, 32, heads, D, kind, DEV)
        plain = e3.new_cache(pages, 32, heads, D, kind, DEV)
        q_out = e3.e3_cache_append_rotated(cache, q if q_heads else None, k, v, r, pos.to(DEV), slots.to(DEV))
        e3.e3_cache_append(plain, k, v, slots.to(DEV))
        # values as e3_cache_append stores them, bit for bit, nothing written elsewhere
        assert torch.equal(cache.v.view(torch.uint8), plain.v.view(torch.uint8))
        if kind is not torch.bfloat16:
            assert torch.equal(cache.v_scale, plain.v_scale)
        assert torch.equal(cache.k.view(torch.uint8).any(-1).sum(), plain.k.view(torch.uint8).any(-1).sum())
        if q_heads:
            want, size = turned(x[:, :q_heads], r.freqs, r.axis, pos, neighbours)
            check(q_out, want, size, dtype)
        else:
            assert q_out is None
        got = e3.e3_cache_read(cache, slots.to(DEV), torch.float32)[0].double().cpu()
        want, size = turned(x[:, q_heads:q_heads + heads], r.freqs, r.axis, pos, neighbours)
        off = (got - want).abs()[slots >= 0]
        want, size = want[slots >= 0], size[slots >= 0]
        if kind is torch.bfloat16:
            allowed = size * TRIG + (want.abs() + size * TRIG) * HALF_STEP[torch.bfloat16]
        else:
            # half a step of e4m3: 2^-4 of the value, 2^-10 of the scale for the smallest.  The scale is twice as large where the
            # largest element lies within rounding of the border.
            a = want.abs().amax(-1, keepdim=True)
            scale = torch.exp2(torch.ceil(torch.log2(a / 448 * (1 + 2.0 ** -19))))
            allowed = size * TRIG + (want.abs() + size * TRIG) * 2.0 ** -4 + scale * 2.0 ** -10
        assert bool((off <= allowed).all()), float((off / allowed).max())


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.float8_e4m3fn, torch.bfloat16])
@pytest.mark.parametrize("neighbours", [False, True])
def test_quarter_turns_are_exact(kind, neighbours):
    # by quarter turns keys change places and signs: what is stored is bit for bit what e3_cache_append makes of that
    n, heads, D = 50, 3, 64
    g = torch.Generator().manual_seed(6)
    k = (torch.rand((n, heads, D), generator=g) + 0.5) * torch.where(torch.rand((n, heads, D), generator=g) < 0.5, -1.0, 1.0)
    v = torch.randn((n, heads, D), generator=g)
    pos = torch.randint(-9, 1000, (n,), generator=g)
    r = e3.E3Rotary(torch.full((D // 2,), math.pi / 2, dtype=torch.float64, device=DEV), None, neighbours)
    a, b = (k[..., 0::2], k[..., 1::2]) if neighbours else (k[..., :D // 2], k[..., D // 2:])
    by = (pos % 4)[:, None, None]
    c, s = torch.tensor([1.0, 0.0, -1.0, 0.0])[by], torch.tensor([0.0, 1.0, 0.0, -1.0])[by]
    ya, yb = torch.where(s == 0, a * c, -b * s), torch.where(s == 0, b * c, a * s)
    y = torch.stack([ya, yb], -1).flatten(-2) if neighbours else torch.cat([ya, yb], -1)
    slots = torch.randperm(8 * 32, generator=g)[:n].to(DEV)
    one, two = (e3.new_cache(8, 32, heads, D, kind, DEV) for _ in range(2))
    q = e3.e3_cache_append_rotated(one, k.to(DEV), k.to(DEV), v.to(DEV), r, pos.to(DEV), slots)
    e3.e3_cache_append(two, y.to(DEV), v.to(DEV), slots)
    assert torch.equal(q.cpu(), y)
    for x, w in zip(one, two):
        assert (x is None and w is None) or torch.equal(x.view(torch.uint8), w.view(torch.uint8))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.float8_e4m3fn, torch.bfloat16])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_keys_are_rounded_once(kind, dtype):
    # turned in 64 bits: every stored key is what rounding the definition's value gives, bit for bit
    n, heads, D = 300, 4, 128
    x, g = step_inputs(n, 0, heads, D, dtype, 21)
    k, v = x[:, :heads], x[:, heads:]
    pos = torch.randint(0, 1 << 20, (3, n), generator=g)
    slots = torch.randperm(16 * 32, generator=g)[:n].to(DEV)
    for neighbours in (False, True):
        r = rotary_of(D, 3, neighbours, DEV)
        cache = e3.new_cache(16, 32, heads, D, kind, DEV)
        e3.e3_cache_append_rotated(cache, None, k.to(DEV), v.to(DEV), r, pos.to(DEV), slots)
        want = turned(k, r.freqs, r.axis, pos, neighbours)[0].numpy()
        if kind is torch.bfloat16:
            step = 2.0 ** (np.floor(np.log2(np.abs(want))) - 7)
            want = np.rint(want / step) * step
        else:
            want = quantised(want)[0]
        got = e3.e3_cache_read(cache, slots, torch.float32)[0].cpu().double().numpy()
        assert np.array_equal(got, want)


@pytest.mark.gpu
def test_graph_streams_and_in_place():
    n, heads, D = 65, 2, 128
    x, g = step_inputs(n, 8, heads, D, torch.bfloat16, 9)
    x = x.to(DEV)
    q, k, v = x[:, :8], x[:, 8:10], x[:, 10:]
    r = rotary_of(128, 1, False, DEV)
    pos, slots = torch.arange(n, device=DEV) * 977, torch.arange(n, device=DEV) + 3
    cache = e3.new_cache(8, 32, heads, D, device=DEV)
    want_q = e3.e3_cache_append_rotated(cache, q, k, v, r, pos, slots)
    want_k = cache.k.view(torch.uint8).clone()
    turned_x = e3.e3_rotate(q, r, pos)
    assert torch.equal(turned_x, want_q)                          # the same arithmetic in both calls
    cache.k.view(torch.uint8).zero_()
    out = torch.empty_like(want_q)
    y = torch.empty_like(want_q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        e3.e3_cache_append_rotated(cache, q, k, v, r, pos, slots, q_out=out)
        e3.e3_rotate(q, r, pos, out=y)
    for i in range(3):
        out.zero_()
        y.zero_()
        cache.k.view(torch.uint8).zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want_q) and torch.equal(y, want_q) and torch.equal(cache.k.view(torch.uint8), want_k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cache.k.view(torch.uint8).zero_()
        e3.e3_cache_append_rotated(cache, q, k, v, r, pos, slots, q_out=q)              # in place
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(q, want_q) and torch.equal(cache.k.view(torch.uint8), want_k)
