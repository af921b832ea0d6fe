"""The decode step's calls through the binding's native code against its Python path: the same outputs bit for bit, the same
errors."""
import pytest
import torch

import paper_2505_18573_amd as e3

DEV = "cuda:0"


def _calls(dev):
    g = torch.Generator().manual_seed(1)
    rows, T, heads, D, page = 3, 2, 2, 64, 32
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
    f32 = lambda *s: torch.zeros(s, dtype=torch.float32, device=dev)
    cache = e3.new_cache(8, page, heads, D, device=dev)
    plain = e3.new_cache(8, page, heads, D, torch.bfloat16, device=dev)
    kv = torch.randn((40, 2 * heads, D), generator=g).to(dev)
    slots = torch.arange(40, device=dev) + 3
    q = torch.randn((rows, T, 4, D), generator=g).to(torch.bfloat16).to(dev)
    z = torch.randn((rows, 3, 104), generator=g).to(dev)
    d = torch.randn((rows, 2, 104), generator=g).to(dev)
    x = torch.randint(0, 100, (rows, 2), generator=g).to(torch.int32).to(dev)
    attend = dict(q=q, cache=cache, group_offsets=i32([0, 2, 3]), prefix_pages=i32([[0, 1], [2, 0]]), prefix_lens=i32([35, 4]),
                  row_pages=i32([[3], [4], [5]]), row_lens=i32([2, 30, 7]), scale=0.1)
    verify = dict(logits=z[..., :100], draft_tokens=x, draft_logits=d[..., :100], draft_lens=i32([2, 0, 1]), tau_rows=f32(rows) + 0.8,
                  tau_scalar=1.0, seed=-5, row_base=1 << 35)
    return {
        "append": (e3.e3_cache_append, dict(cache=cache, k=kv[:, :heads], v=kv[:, heads:], slots=slots)),
        "append_bf16": (e3.e3_cache_append, dict(cache=plain, k=kv[:, :heads].bfloat16(), v=kv[:, heads:].bfloat16(), slots=slots)),
        "read": (e3.e3_cache_read, dict(cache=cache, slots=slots)),
        "read_into": (e3.e3_cache_read, dict(cache=plain, slots=slots, dtype=torch.float32, k_out=f32(40, heads, D), v_out=f32(40, heads, D))),
        "attend": (e3.e3_prefix_attention, attend),
        "attend_plain": (e3.e3_prefix_attention, dict(attend, cache=plain, group_offsets=None, prefix_pages=None, prefix_lens=None,
                                                      want_lse=False, scale=1)),
        "attend_into": (e3.e3_prefix_attention, dict(attend, out=torch.zeros_like(q), lse_out=f32(rows, T, 4),
                                                     workspace=torch.zeros(e3.e3_prefix_attention_workspace_bytes(rows, T, 4, heads, D, 2),
                                                                           dtype=torch.uint8, device=dev))),
        "verify": (e3.e3_verify_drafts, verify),
        "verify_lookup": (e3.e3_verify_drafts, dict(verify, logits=z.bfloat16()[..., :100], draft_logits=None, draft_lens=None, tau_rows=None,
                                                    tau_scalar=0.7, draft_tau_rows=f32(rows) + 0.9)),
        "verify_into": (e3.e3_verify_drafts, dict(verify, accepted_out=torch.zeros(rows, dtype=torch.int32, device=dev),
                                                  token_out=torch.zeros((rows, 3), dtype=torch.int32, device=dev), logp_out=f32(rows, 3),
                                                  entropy_out=f32(rows, 3),
                                                  workspace=torch.zeros(e3.e3_verify_workspace_bytes(rows, 2, 100), dtype=torch.uint8, device=dev))),
        "verify_none": (e3.e3_verify_drafts, dict(logits=z[:, :1, :100], draft_tokens=None, draft_logits=None, draft_lens=None, tau_rows=None,
                                                  tau_scalar=1.0, seed=2)),
    }


NAMES = list(_calls("cpu"))


def _outcome(f, kw, monkeypatch, native):
    e3.lib()
    with monkeypatch.context() as m:
        if not native:
            m.setattr(e3.binding, "_native", None)
        try:
            out = f(**kw)
        except Exception as e:                            # the error is what is compared
            return type(e), str(e)
    if out is None:                                       # a cache that was written: its contents
        out = tuple(t for t in kw["cache"] if t is not None)
    if torch.cuda.is_available():
        torch.cuda.synchronize()
    return tuple(t.clone() if t is not None else None for t in out)


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_same_outputs_as_the_python_path(name, monkeypatch):
    f, kw = _calls(DEV)[name]
    e3.lib()
    served = []
    real = e3.binding._native
    for call in ("cache_append", "cache_read", "attention", "verify"):
        assert hasattr(real, call)
    monkeypatch.setattr(e3.binding, "_ordinary", lambda n, *a, keep=e3.binding._ordinary: (lambda r: (served.append((n, r is not None)), r)[1])(keep(n, *a)))
    want = _outcome(f, kw, monkeypatch, native=False)
    f, kw = _calls(DEV)[name]
    served.clear()
    got = _outcome(f, kw, monkeypatch, native=True)
    assert served and all(ok for _, ok in served)         # the native call did it
    assert len(got) == len(want)
    for a, b in zip(got, want):
        if b is None:
            assert a is None
        else:
            assert a.dtype is b.dtype and a.device == b.device and a.shape == b.shape and torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def _spoilt(kw):
    """One argument at a time replaced by what the checks on the host refuse."""
    for key, v in kw.items():
        if key == "cache":
            for i, t in enumerate(v):
                if t is not None:
                    for bad in (t.cpu() if t.is_cuda else t[:1], t.float(), t[:, :1], None):
                        yield dict(kw, cache=e3.E3Cache(*(bad if j == i else x for j, x in enumerate(v))))
            yield dict(kw, cache=tuple(v)[:3])
        elif torch.is_tensor(v):
            if key != "workspace":
                yield dict(kw, **{key: v.to(torch.float16)})
                yield dict(kw, **{key: v[None]})
            yield dict(kw, **{key: v.repeat_interleave(2, -1)[..., ::2]})
            yield dict(kw, **{key: v.cpu() if v.is_cuda else v.double()})
            yield dict(kw, **{key: 5})
        elif key in ("scale", "tau_scalar"):
            yield dict(kw, **{key: -1.0})
            yield dict(kw, **{key: float("nan")})
            yield dict(kw, **{key: "x"})


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_same_errors(name, monkeypatch):
    f, kw = _calls(DEV)[name]
    for bad in _spoilt(kw):
        want, got = (_outcome(f, bad, monkeypatch, native=n) for n in (False, True))
        if isinstance(want[0], type):
            assert got == want, bad
        else:                                             # taken (a scalar that a tensor of rows makes unused): taken either way
            assert not isinstance(got[0], type), bad


@pytest.mark.parametrize("name", NAMES)
def test_tensors_on_the_host_are_refused(name, monkeypatch):
    if torch.cuda.is_available():
        pytest.skip("tensors on the CPU")
    f, kw = _calls("cpu")[name]
    for native in (False, True):
        kind, text = _outcome(f, kw, monkeypatch, native)
        assert kind is ValueError and "GPU" in text


@pytest.mark.gpu
@pytest.mark.parametrize("native", [True, False])
def test_strides_of_single_elements_do_not_count(native, monkeypatch):
    # torch may report anything as the stride of a dimension of one
    e3.lib()
    if not native:
        monkeypatch.setattr(e3.binding, "_native", None)
    g = torch.Generator().manual_seed(4)
    data = torch.randn(256, generator=g).to(DEV)
    slots = torch.tensor([5, 6, 9], device=DEV)
    for shape, strides, heads in (((1, 2, 64), (5, 64, 1), 2), ((3, 1, 64), (64, 3, 1), 1)):
        x = data.as_strided(shape, strides)
        caches = [e3.new_cache(1, 32, heads, 64, device=DEV) for _ in range(2)]
        e3.e3_cache_append(caches[0], x, x, slots[:shape[0]])
        e3.e3_cache_append(caches[1], x.flatten().reshape(shape), x.flatten().reshape(shape), slots[:shape[0]])
        for a, b in zip(*caches):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    cache = e3.new_cache(1, 32, 2, 64, torch.bfloat16, device=DEV)
    e3.e3_cache_append(cache, data[:128].reshape(1, 2, 64), data[128:].reshape(1, 2, 64), torch.zeros(1, dtype=torch.int64, device=DEV))
    q = data.to(torch.bfloat16).as_strided((1, 1, 4, 64), (13, 7, 64, 1))
    i32 = lambda t: torch.tensor(t, dtype=torch.int32, device=DEV)
    args = (cache, None, None, None, i32([[0]]), i32([1]), 0.125)
    out, lse = e3.e3_prefix_attention(q, *args)
    want, want_lse = e3.e3_prefix_attention(data.to(torch.bfloat16).reshape(1, 1, 4, 64), *args)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    # no drafts, and an empty tensor of their logits whose strides are odd
    z = torch.randn((2, 1, 104), generator=g).to(DEV)[..., :101]
    a = e3.e3_verify_drafts(z, None, torch.empty((2, 0, 101), device=DEV), None, None, 1.0, 3)
    b = e3.e3_verify_drafts(z, None, None, None, None, 1.0, 3)
    assert all(torch.equal(s, t) for s, t in zip(a, b))
