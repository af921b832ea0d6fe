"""The paged cache of keys and values: writing (with quantisation) and reading back, against the definition in 64 bits.

Everything here is exact: the scale is a power of two, rounding to e4m3 is to nearest even, widening is exact.  So the tests compare
bits, with no tolerance."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2505_18573_amd as e3

DEV = "cuda:0"


def quantised(x):
    """x [..., D] -> the values that an 8-bit cache stands for, and the exponents, in 64 bits (numpy)."""
    x = np.asarray(x, dtype=np.float64)
    finite = np.isfinite(x)
    a = np.abs(np.where(finite, x, 0.0)).max(-1)
    e = np.full(a.shape, -126)
    for i in np.ndindex(a.shape):
        while e[i] < 127 and a[i] > 448.0 * 2.0 ** e[i]:
            e[i] += 1
    y = np.where(finite, x, 0.0) / 2.0 ** e[..., None].astype(np.float64)
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6))) - 3)
    return np.where(finite, np.rint(y / step) * step * 2.0 ** e[..., None].astype(np.float64), np.nan), e


def test_the_reference_knows_the_format():
    # e4m3: 448 is the largest value, 2^-9 the smallest, steps of 2^-3 of the leading bit, ties to even
    v, e = quantised(np.array([[448.0, 17.0, 19.0, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, 0.0, -np.inf]]))
    assert e[0] == 0
    assert v[0, :7].tolist() == [448.0, 16.0, 20.0, 2.0 ** -9, 0.0, 2 * 2.0 ** -9, 0.0] and np.isnan(v[0, 7])
    assert quantised(np.array([[449.0]]))[1][0] == 1 and quantised(np.array([[0.0]]))[1][0] == -126
    assert quantised(np.array([[3.0e38]]))[1][0] == 120


def cache_struct(k=0x10000, v=0x20000, ks=0x30000, vs=0x40000, pages=4, page=64, heads=2, dim=128, dtype=2):
    return e3.binding._CacheStruct(k, v, ks, vs, pages, page, heads, dim, dtype)


def test_argument_checks_without_gpu():
    L = e3.lib()

    def append(c, k=0x1000, v=0x2000, dtype=1, tokens=3, strides=(256, 128, 256, 128), slots=0x3000):
        return L.e3_cache_append(C.byref(c) if c is not None else None, k, v, dtype, tokens, *strides, slots, None)

    def read(c, slots=0x3000, tokens=3, k=0x1000, v=0x2000, dtype=1):
        return L.e3_cache_read(C.byref(c) if c is not None else None, slots, tokens, k, v, dtype, None)

    for call in (append, read):
        assert call(None) == -1
        assert call(cache_struct(dtype=0)) == -3 and call(cache_struct(dtype=3)) == -3
        assert call(cache_struct(page=48)) == -2 and call(cache_struct(page=16)) == -2 and call(cache_struct(page=0)) == -2
        assert call(cache_struct(dim=96)) == -2 and call(cache_struct(heads=0)) == -2 and call(cache_struct(pages=0)) == -2
        assert call(cache_struct(k=None)) == -1 and call(cache_struct(vs=None)) == -1
        assert call(cache_struct(k=0x10008)) == -4 and call(cache_struct(ks=0x30004)) == -4
        assert call(cache_struct(), dtype=2) == -3
        assert call(cache_struct(), tokens=-1) == -2 and call(cache_struct(), tokens=1 << 31) == -2
        assert call(cache_struct(), k=None) == -1 and call(cache_struct(), slots=None) == -1
        assert call(cache_struct(), v=0x2008) == -4
        assert call(cache_struct(), tokens=0, k=None, v=None, slots=None) == 0
    assert append(cache_struct(), strides=(256, 100, 256, 128)) == -4          # 200 bytes
    assert append(cache_struct(), dtype=0, strides=(256, 130, 256, 128)) == -4


def test_calls_beyond_a_launch_are_refused():
    # more than 2^28 tokens times heads: the launch would pass 2^32 threads
    L, c = e3.lib(), cache_struct(heads=16)
    for tokens in ((1 << 24) + 1, 1 << 28):
        assert L.e3_cache_append(C.byref(c), 0x1000, 0x2000, 1, tokens, 0, 0, 0, 0, 0x3000, None) == -2
        assert L.e3_cache_read(C.byref(c), 0x3000, tokens, 0x1000, 0x2000, 1, None) == -2


def test_binding_refuses():
    with pytest.raises(TypeError):
        e3.new_cache(2, 64, 1, 64, torch.float16, device="cpu")
    with pytest.raises(ValueError):
        e3.new_cache(2, 40, 1, 64, device="cpu")
    c = e3.new_cache(2, 64, 1, 64, device="cpu")
    assert c.k.shape == (2, 1, 64, 64) and c.v.shape == (2, 1, 8, 64, 8) and c.k_scale.shape == (2, 1, 64)
    with pytest.raises(ValueError):
        e3.e3_cache_read(c, torch.zeros(1, dtype=torch.int64))                 # on the host


def inputs(n, heads, D, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, heads, D), generator=g) * torch.exp(torch.randn((n, heads, 1), generator=g) * 3)
    return x.to(dtype)


def slots_of(kind, n, capacity, g):
    if kind == "run":                                    # one sequence, starting anywhere in a block
        return torch.arange(n) + 5
    if kind == "aligned":
        return torch.arange(n) + 32
    if kind == "scattered":
        return torch.randperm(capacity, generator=g)[:n]
    # several sequences of odd lengths on shuffled pages of 32, some padding in between
    s = torch.full((n,), -1, dtype=torch.int64)
    pages = torch.randperm(capacity // 32, generator=g)
    at, p = 0, 0
    while at < n:
        m = min(n - at, int(torch.randint(1, 75, (1,), generator=g)))
        for i in range(m):
            s[at + i] = pages[p + i // 32] * 32 + i % 32
        p += -(-m // 32)
        at += m + int(torch.randint(0, 3, (1,), generator=g))
    return s


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["run", "aligned", "scattered", "sequences"])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 203])
@pytest.mark.parametrize("heads,D", [(1, 64), (3, 64), (2, 128), (5, 128)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_written_and_read_back(kind, n, heads, D, dtype):
    g = torch.Generator().manual_seed(n)
    pages = 64
    slots = slots_of(kind, n, pages * 32, g)
    k, v = inputs(n, heads, D, dtype, 2 * n), inputs(n, heads, D, dtype, 2 * n + 1)
    for cache_type in (torch.float8_e4m3fn, torch.bfloat16):
        cache = e3.new_cache(pages, 32, heads, D, cache_type, DEV)
        # projections give keys and values as parts of one tensor
        both = torch.cat([k, v], 1).to(DEV)
        e3.e3_cache_append(cache, both[:, :heads], both[:, heads:], slots.to(DEV))
        want = []
        for x in (k, v):
            w = torch.from_numpy(quantised(x.double().numpy())[0]) if cache_type is torch.float8_e4m3fn else x.to(torch.bfloat16).double()
            w[slots < 0] = 0.0
            want.append(w)
        for out in (torch.float32, torch.bfloat16):
            got = e3.e3_cache_read(cache, slots.to(DEV), out)
            for x, w in zip(got, want):
                assert x.dtype is out
                assert torch.equal(x.cpu(), w.to(out))
        # the documented layout, element by element
        at = slots[slots >= 0]
        page, tok = at // 32, at % 32
        kl, vl = (t.cpu().float() if t.dtype is torch.bfloat16 else t.cpu().view(torch.uint8).view(torch.float8_e4m3fn).float()
                  for t in (cache.k, cache.v))
        kl = kl[page, :, tok]
        vl = vl[page, :, tok // 8, :, tok % 8]
        if cache.k_scale is not None:
            kl = torch.ldexp(kl, cache.k_scale.cpu()[page, :, tok].int()[..., None] - 127)
            vl = torch.ldexp(vl, cache.v_scale.cpu()[page, :, tok].int()[..., None] - 127)
        assert torch.equal(kl.double(), want[0][slots >= 0]) and torch.equal(vl.double(), want[1][slots >= 0])
        # nothing else was written
        used = torch.zeros(pages * 32, dtype=torch.bool)
        used[at] = True
        rest = e3.e3_cache_read(cache, torch.arange(pages * 32, device=DEV), torch.float32)
        assert all(bool((r.cpu()[~used] == 0).all()) for r in rest)


@pytest.mark.gpu
def test_values_at_the_edges_of_the_format():
    D = 64
    rows = [np.zeros(D), np.full(D, 448.0), np.full(D, 464.0), np.full(D, 2.0 ** -126), np.full(D, 2.0 ** -149),
            np.full(D, 3.3e38), np.full(D, -3.3e38)]
    # everything between two representable values and their ties, at several scales
    codes = np.array([(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8)] + [m * 2.0 ** -9 for m in range(8)])
    codes = np.unique(codes[codes <= 448.0])
    ties = (codes[1:] + codes[:-1]) / 2
    for s in (1.0, 2.0 ** -20, 2.0 ** 30):
        for part in np.array_split(np.concatenate([codes, ties, np.nextafter(ties.astype(np.float32), np.float32(1e9)).astype(np.float64),
                                                   np.nextafter(ties.astype(np.float32), np.float32(0)).astype(np.float64)]), 9):
            r = np.zeros(D)
            r[:part.size] = part * s
            r[-1] = 448.0 * s                            # the scale is s
            rows.append(r)
    bad = np.linspace(-5, 5, D)
    bad[3], bad[9], bad[20] = np.nan, np.inf, -np.inf
    rows += [bad, np.full(D, np.nan), np.full(D, np.inf)]
    x = np.stack(rows).astype(np.float32)[:, None]
    n = x.shape[0]
    want, e = quantised(x.astype(np.float64))
    cache = e3.new_cache(-(-n // 32), 32, 1, D, torch.float8_e4m3fn, DEV)
    t = torch.from_numpy(x).to(DEV)
    slots = torch.arange(n, device=DEV)
    e3.e3_cache_append(cache, t, -t, slots)
    k, v = e3.e3_cache_read(cache, slots, torch.float32)
    with np.errstate(over="ignore"):
        want32 = want.astype(np.float32)
    assert np.array_equal(k.cpu().numpy(), want32, equal_nan=True)
    assert np.array_equal(v.cpu().numpy(), -want32, equal_nan=True)
    assert np.array_equal(cache.k_scale.cpu().numpy().reshape(-1)[:n], (e + 127).reshape(-1))
    # read back and written again: the same bits (3.3e38 rounds to 2^128, which fp32 reads as inf)
    again = e3.new_cache(-(-n // 32), 32, 1, D, torch.float8_e4m3fn, DEV)
    e3.e3_cache_append(again, k, v, slots)
    with np.errstate(over="ignore"):
        finite = np.isfinite(want.astype(np.float32)).all(-1).reshape(-1)
    for a, b in zip(e3.e3_cache_read(again, slots, torch.float32), (k, v)):
        assert torch.equal(a.cpu()[finite], b.cpu()[finite])


@pytest.mark.gpu
def test_slots_outside_the_cache_and_behind_2_to_the_32():
    heads, D, page = 8, 128, 128
    pages = 2 ** 32 // (heads * D * page) + 3            # elements of the last pages lie behind 2^32
    cache = e3.new_cache(pages, page, heads, D, torch.float8_e4m3fn, DEV)
    last = pages * page
    slots = torch.tensor([last - 1, -1, last, last - 130, 2 ** 40, -2 ** 40, 3] + list(range(last - 24, last - 8)), device=DEV)
    n = slots.numel()
    x = inputs(n, heads, D, torch.bfloat16, 5).to(DEV)
    e3.e3_cache_append(cache, x, x, slots)
    ok = ((slots >= 0) & (slots < last)).cpu()
    want = torch.from_numpy(quantised(x.double().cpu().numpy())[0]).float()
    want[~ok] = 0.0
    for got in e3.e3_cache_read(cache, slots, torch.float32):
        assert torch.equal(got.cpu(), want)


@pytest.mark.gpu
def test_empty_calls_outputs_given_and_another_stream():
    cache = e3.new_cache(2, 32, 2, 64, torch.float8_e4m3fn, DEV)
    z = torch.empty((0, 2, 64), dtype=torch.bfloat16, device=DEV)
    none = torch.empty(0, dtype=torch.int64, device=DEV)
    e3.e3_cache_append(cache, z, z, none)
    assert e3.e3_cache_read(cache, none)[0].shape == (0, 2, 64)
    x = inputs(5, 2, 64, torch.float32, 1).to(DEV)
    slots = torch.tensor([3, 9, 10, 40, 63], device=DEV)
    k, v = torch.empty_like(x), torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        e3.e3_cache_append(cache, x, 2 * x, slots)
        out = e3.e3_cache_read(cache, slots, torch.float32, k_out=k, v_out=v)
    torch.cuda.current_stream().wait_stream(side)
    assert out[0] is k and out[1] is v
    want = torch.from_numpy(quantised(x.double().cpu().numpy())[0]).float()
    assert torch.equal(k.cpu(), want) and torch.equal(v.cpu(), 2 * want)
    with pytest.raises(ValueError):
        e3.e3_cache_append(cache, x[:, :1], x, slots)
    with pytest.raises(ValueError):
        e3.e3_cache_append(cache, x, x.to(torch.bfloat16), slots)
    with pytest.raises(ValueError):
        e3.e3_cache_append(cache, x, x, slots.int())
    with pytest.raises(TypeError):
        e3.e3_cache_read(cache, slots, torch.float16)
    with pytest.raises(e3.E3Error) as err:
        wide = torch.zeros((5, 2, 66), device=DEV)[:, :, :64]                  # rows of 264 bytes
        e3.e3_cache_append(cache, wide, x, slots)
    assert err.value.status == -4
