"""What a rollout's decode step in front of the sampler is measured on: the cache that holds keys and values in
8 bits, the attention of groups of rollouts that share their question's prompt, and the verification of drafted
tokens.

A case is a dict of plain values.  `prepare` makes what a program has in hand before the call, `run` is one pass:
with `own` through the entry points of `paper_2505_18573_amd`, without it the operators in plain torch (32 bits,
rounded once at the end).  `exact` gives the same results in 64 bits, `work` what a pass cannot do without.

The cache's layout (both forms read it): keys [pages, heads, page, D], values [pages, heads, page / 8, D, 8] (eight
tokens of one column next to each other), one exponent byte e + 127 per token and head for each where the cache holds
8 bits; an element is code * 2^e.  Random numbers are words of Philox4x32-10 named by seed, row and index.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # the keys and values of one decode step of 64 questions x 8 rollouts, one token each, written and read back
        {"name": "cache_step_512", "kind": "cache", "tokens": 512, "heads": 4, "D": 128, "page": 64, "dtype": "bf16",
         "whole": False},
        # the prompts of a step's questions, all at once: runs of tokens of odd lengths
        {"name": "cache_prompts", "kind": "cache", "tokens": 60_001, "heads": 4, "D": 128, "page": 64, "dtype": "bf16",
         "whole": True},
        # fp32 projections, narrow heads, many of them
        {"name": "cache_f32_ragged", "kind": "cache", "tokens": 3001, "heads": 12, "D": 64, "page": 32, "dtype": "f32",
         "whole": True},
        # a single rollout with a short prompt: launches and latency
        {"name": "attend_1_row", "kind": "attend", "groups": 1, "size": 1, "mixed": False, "T": 1, "q_heads": 12,
         "heads": 2, "D": 128, "page": 64, "cache": "fp8", "prefix_lo": 150, "prefix_hi": 150, "suffix_lo": 77, "suffix_hi": 77},
        # a decode step of 64 questions x 8 rollouts at all stages of responses of up to 6000 tokens
        {"name": "attend_512_rows", "kind": "attend", "groups": 64, "size": 8, "mixed": False, "T": 1, "q_heads": 28,
         "heads": 4, "D": 128, "page": 64, "cache": "fp8", "prefix_lo": 100, "prefix_hi": 1000, "suffix_lo": 1, "suffix_hi": 6000},
        # rollout budgets of 4 to 12, four drafted tokens and one more to verify in each row
        {"name": "attend_drafts", "kind": "attend", "groups": 16, "size": 8, "mixed": True, "T": 5, "q_heads": 12,
         "heads": 2, "D": 128, "page": 32, "cache": "fp8", "prefix_lo": 65, "prefix_hi": 1500, "suffix_lo": 5, "suffix_hi": 2500},
        # few rollouts of one very long prompt, 16-bit cache
        {"name": "attend_long_prefix", "kind": "attend", "groups": 1, "size": 12, "mixed": False, "T": 1, "q_heads": 32,
         "heads": 8, "D": 128, "page": 128, "cache": "bf16", "prefix_lo": 32_771, "prefix_hi": 32_771, "suffix_lo": 1, "suffix_hi": 700},
        # as many key heads as query heads, narrow ones
        {"name": "attend_mha_64", "kind": "attend", "groups": 24, "size": 4, "mixed": True, "T": 1, "q_heads": 16,
         "heads": 16, "D": 64, "page": 64, "cache": "bf16", "prefix_lo": 33, "prefix_hi": 900, "suffix_lo": 0, "suffix_hi": 2000},
        # four drafted tokens for each of 512 rollouts, drafted by a model of its own
        {"name": "verify_512x4", "kind": "verify", "rows": 512, "drafts": 4, "V": 151_936, "dtype": "bf16",
         "drafter": True, "ragged": False, "tau": "rows"},
        # a few interactive sequences: launches and latency
        {"name": "verify_4x3", "kind": "verify", "rows": 4, "drafts": 3, "V": 151_936, "dtype": "bf16",
         "drafter": True, "ragged": False, "tau": "scalar"},
        # drafts looked up in the context (no draft distribution), different numbers of them, fp32 logits
        {"name": "verify_lookup_f32", "kind": "verify", "rows": 100, "drafts": 5, "V": 70_005, "dtype": "f32",
         "drafter": False, "ragged": True, "tau": "rows"},
        # a smaller vocabulary and a middling batch
        {"name": "verify_64x7_32000", "kind": "verify", "rows": 64, "drafts": 7, "V": 32_000, "dtype": "bf16",
         "drafter": True, "ragged": True, "tau": "scalar"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["cache", "attend", "attend", "verify", "verify"])
    if kind == "cache":
        c = {"kind": kind, "tokens": _log_int(rng, 1, 60_000), "heads": rng.choice([2, 4, 8, 12]), "D": rng.choice([64, 128]),
             "page": rng.choice([32, 64, 128]), "dtype": rng.choice(["bf16", "bf16", "f32"]), "whole": rng.random() < 0.6}
        while c["tokens"] * c["heads"] * c["D"] * (2 if c["dtype"] == "f32" else 1) > 60_001 * 4 * 128:
            c["tokens"] = c["tokens"] * 2 // 3
        return c
    if kind == "attend":
        heads = rng.choice([2, 4, 8])
        c = {"kind": kind, "groups": _log_int(rng, 1, 64), "size": rng.choice([1, 4, 8, 12]), "mixed": rng.random() < 0.5,
             "T": rng.choice([1, 1, 1, 3, 5]), "q_heads": heads * rng.choice([1, 4, 6, 7, 8]), "heads": heads,
             "D": rng.choice([64, 128, 128]), "page": rng.choice([32, 64, 128]), "cache": rng.choice(["fp8", "fp8", "bf16"]),
             "prefix_lo": _log_int(rng, 1, 200), "prefix_hi": _log_int(rng, 200, 8000),
             "suffix_lo": rng.choice([0, 1, 40]), "suffix_hi": _log_int(rng, 40, 6000)}
        # no more to read, and no more products, than the largest listed case has
        most = _attend_work(listed()[4])
        for key in ("suffix", "prefix", "groups"):
            for _ in range(12):
                w = _attend_work(c)
                held = c["groups"] * c["size"] * (c["prefix_hi"] + c["suffix_hi"]) * c["heads"] * c["D"]
                if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"] and held <= 512 * 7000 * 4 * 128:
                    break
                if key == "groups":
                    c["groups"] = max(1, c["groups"] * 2 // 3)
                else:
                    c[key + "_hi"] = max(c[key + "_lo"], 40, c[key + "_hi"] * 2 // 3)
        return c
    c = {"kind": kind, "rows": _log_int(rng, 1, 512), "drafts": rng.choice([1, 2, 3, 4, 6, 8]),
         "V": rng.choice([151_936, 32_000, 128_000, _log_int(rng, 1000, 260_000)]), "dtype": rng.choice(["bf16", "bf16", "f32"]),
         "drafter": rng.random() < 0.7, "ragged": rng.random() < 0.5, "tau": rng.choice(["rows", "scalar"])}
    most = work(listed()[8])["bytes"]
    while work(c)["bytes"] > most:
        c["rows"] = max(1, c["rows"] * 2 // 3)
    return c


# ---------------------------------------------------------------- inputs (from the seed alone)
def _rand(g, *shape):
    return torch.rand(shape, generator=g, device=DEV)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _sizes(case):
    """Rollouts of each question: the same number, or budgets around it (their sum is the same for every seed)."""
    n, s = case["groups"], case["size"]
    return [max(1, s + (i % (s + 1)) - s // 2) for i in range(n)] if case["mixed"] else [s] * n


def _spread(lo, hi, n):
    return [round(lo + (hi - lo) * (i / (n - 1) if n > 1 else 1.0)) for i in range(n)]


def _shuffled(values, g):
    v = torch.tensor(values, device=DEV)
    return v[torch.randperm(len(values), generator=g, device=DEV)]


def _tables(lens_max, units, page, first):
    """Page tables of `units` sequences, `wide` pages each, numbered from `first`."""
    wide = max(1, -(-lens_max // page))
    return first + torch.arange(units * wide, device=DEV).reshape(units, wide), units * wide


def _cache_of(pages, heads, page, D, kind, g):
    """Keys and values of unit variance with a few louder columns and tokens of different size."""
    col = 1.0 + 3.0 * (_rand(g, heads, 1, D) < 0.03).float()
    k = torch.empty((pages, heads, page, D), dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    for p0 in range(0, pages, 4096):
        n = min(4096, pages - p0)
        k[p0:p0 + n] = _randn(g, n, heads, page, D).mul_(col)
        v[p0:p0 + n] = _randn(g, n, heads, page, D).mul_(0.5 + _rand(g, n, heads, page, 1))
    if kind == "bf16":
        return k, v.reshape(pages, heads, page // 8, 8, D).transpose(-1, -2).contiguous(), None, None
    made = []
    for x in (k, v):
        codes = torch.empty((pages, heads, page, D), dtype=torch.uint8, device=DEV)
        scale = torch.empty((pages, heads, page), dtype=torch.uint8, device=DEV)
        for p0 in range(0, pages, 4096):
            y, e = _to_fp8(x[p0:p0 + 4096].float())
            codes[p0:p0 + 4096], scale[p0:p0 + 4096] = y.view(torch.uint8), (e + 127).to(torch.uint8)
        made.append((codes, scale))
    (k, ks), (v, vs) = made
    v = v.reshape(pages, heads, page // 8, 8, D).transpose(-1, -2).contiguous()
    return k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), ks, vs


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return {"cache": _prepare_cache, "attend": _prepare_attend, "verify": _prepare_verify}[case["kind"]](case, g, seed)


def _prepare_cache(case, g, seed):
    n, H, D, page = case["tokens"], case["heads"], case["D"], case["page"]
    # one row of the projection's output: query heads, then key heads, then value heads
    qkv = (_randn(g, n, 3 * H, D) * (0.2 + 3.0 * _rand(g, n, 3 * H, 1))).to(DTYPES[case["dtype"]])
    if case["whole"]:                              # sequences of odd lengths, each from the start of a page of its own
        lens, left = [], n
        while left:
            lens.append(min(left, 1 + (len(lens) * 397 + seed) % 1531))
            left -= lens[-1]
        need = [-(-l // page) for l in lens]
        pages = sum(need)
        order = torch.randperm(pages, generator=g, device=DEV)
        lens_d, need_d = torch.tensor(lens, device=DEV), torch.tensor(need, device=DEV)
        first = torch.cumsum(need_d, 0) - need_d
        seq = torch.repeat_interleave(torch.arange(len(lens), device=DEV), lens_d)
        at = torch.arange(n, device=DEV) - (torch.cumsum(lens_d, 0) - lens_d)[seq]
        slots = order[first[seq] + at // page] * page + at % page
    else:                                          # one token of each sequence, at any place of its last page
        pages = n
        slots = torch.randperm(pages, generator=g, device=DEV) * page + torch.randint(0, page, (n,), generator=g, device=DEV)
    cache = (torch.zeros((pages, H, page, D), dtype=torch.float8_e4m3fn, device=DEV),
             torch.zeros((pages, H, page // 8, D, 8), dtype=torch.float8_e4m3fn, device=DEV),
             torch.zeros((pages, H, page), dtype=torch.uint8, device=DEV),
             torch.zeros((pages, H, page), dtype=torch.uint8, device=DEV))
    return {"case": case, "k": qkv[:, H:2 * H], "v": qkv[:, 2 * H:], "slots": slots.long(), "cache": cache}


def _prepare_attend(case, g, seed):
    sizes = _shuffled(_sizes(case), g)
    G, rows, page = case["groups"], sum(_sizes(case)), case["page"]
    offsets = torch.zeros(G + 1, dtype=torch.int32, device=DEV)
    offsets[1:] = torch.cumsum(sizes, 0)
    prefix_pages, n_prefix = _tables(case["prefix_hi"], G, page, 0)
    row_pages, n_rows = _tables(case["suffix_hi"], rows, page, n_prefix)
    pages = n_prefix + n_rows
    order = torch.randperm(pages, generator=g, device=DEV)
    q = _randn(g, rows, case["T"], case["q_heads"], case["D"]).to(torch.bfloat16)
    return {"case": case, "q": q, "cache": _cache_of(pages, case["heads"], page, case["D"], case["cache"], g),
            "offsets": offsets, "prefix_pages": order[prefix_pages].to(torch.int32),
            "prefix_lens": _shuffled(_spread(case["prefix_lo"], case["prefix_hi"], G), g).to(torch.int32),
            "row_pages": order[row_pages].to(torch.int32),
            "row_lens": _shuffled(_spread(case["suffix_lo"], case["suffix_hi"], rows), g).to(torch.int32), "scale": case["D"] ** -0.5}


def _prepare_verify(case, g, seed):
    rows, K, V = case["rows"], case["drafts"], case["V"]
    per = 8 if case["dtype"] == "bf16" else 4                        # rows start on 16 bytes
    pitch = -(-V // per) * per
    logits = torch.empty((rows, K + 1, pitch), dtype=DTYPES[case["dtype"]], device=DEV)
    drafter = torch.empty((rows, K, pitch), dtype=DTYPES[case["dtype"]], device=DEV) if case["drafter"] else None
    tau = (0.6 + 0.8 * _rand(g, rows)).float() if case["tau"] == "rows" else None
    tokens = torch.empty((rows, K), dtype=torch.int32, device=DEV)
    for r0 in range(0, rows, 64):
        n = min(64, rows - r0)
        x = _randn(g, n, K + 1, pitch).mul_(3.0)
        cols = torch.randint(0, V, (n, K + 1, 20), generator=g, device=DEV)
        x.scatter_(2, cols, torch.gather(x, 2, cols) + 8.0)
        logits[r0:r0 + n] = x
        d = x[:, :K]
        if drafter is not None:                                      # a smaller model: the same distribution with errors
            drafter[r0:r0 + n] = d + 0.6 * _randn(g, n, K, pitch)
            d = drafter[r0:r0 + n].float()
        t = tau[r0:r0 + n, None, None] if tau is not None else 0.9
        noise = _rand(g, n, K, pitch).clamp_(min=1e-9).log_().neg_()
        tokens[r0:r0 + n] = ((d / t)[..., :V] - noise[..., :V].log()).argmax(-1).to(torch.int32)
    lens = torch.randint(0, K + 1, (rows,), generator=g, device=DEV).to(torch.int32) if case["ragged"] else None
    return {"case": case, "logits": logits[..., :V], "drafter": drafter[..., :V] if drafter is not None else None,
            "tokens": tokens, "lens": lens, "tau_rows": tau, "tau": 0.9, "seed": seed % 1_000_003}


# ---------------------------------------------------------------- one pass
def run(s):
    kind = s["case"]["kind"]
    if own:
        import paper_2505_18573_amd as e3
        if kind == "cache":
            cache = e3.E3Cache(*s["cache"])
            e3.e3_cache_append(cache, s["k"], s["v"], s["slots"])
            k, v = e3.e3_cache_read(cache, s["slots"])
            return {"k": k, "v": v}
        if kind == "attend":
            out, lse = e3.e3_prefix_attention(s["q"], e3.E3Cache(*s["cache"]), s["offsets"], s["prefix_pages"], s["prefix_lens"],
                                              s["row_pages"], s["row_lens"], s["scale"])
            return {"out": out, "lse": lse}
        accepted, token, logp, entropy = e3.e3_verify_drafts(s["logits"], s["tokens"], s["drafter"], s["lens"], s["tau_rows"],
                                                             s["tau"], s["seed"])
        return {"accepted": accepted, "token": token, "logp": logp, "entropy": entropy}
    if kind == "cache":
        return {"k": _plain_stored(s["k"]), "v": _plain_stored(s["v"])}
    return _plain_attend(s) if kind == "attend" else _plain_verify(s)


def _to_fp8(x):
    """Codes and exponents of the last axis' vectors: the smallest power of two that brings the largest to at most 448."""
    a = x.abs().amax(-1)
    m, e = torch.frexp(a)                                            # a = m 2^e, m in [1/2, 1); 448 = 7/8 2^9
    e = (e - 9 + (m > 0.875)).clamp(-126, 127)
    return torch.ldexp(x, -e[..., None]).to(torch.float8_e4m3fn), e


def _plain_stored(x):
    y, e = _to_fp8(x.float())
    return torch.ldexp(y.float(), e[..., None]).to(torch.bfloat16)


def _plain_pages(s, pages):
    """Keys and values of the pages [rows, n] as [rows, heads, n * page, D]."""
    k, v, ks, vs = s["cache"]
    rows, n = pages.shape
    _, H, page, D = k.shape
    kind = k.dtype

    def of(x, scale, order):
        x = (x.view(torch.uint8) if kind != torch.bfloat16 else x)[pages]
        x = (x.view(kind) if kind != torch.bfloat16 else x).float().permute(order).reshape(rows, H, n * page, D)
        if scale is not None:
            x *= torch.exp2(scale[pages].float() - 127.0).transpose(1, 2).reshape(rows, H, n * page, 1)
        return x

    return of(k, ks, (0, 2, 1, 3, 4)), of(v, vs, (0, 2, 1, 3, 5, 4))


def _plain_attend(s):
    q, T = s["q"], s["case"]["T"]
    rows, _, Hq, D = q.shape
    H = s["cache"][0].shape[1]
    page = s["cache"][0].shape[2]
    R = Hq // H
    sizes = (s["offsets"][1:] - s["offsets"][:-1]).long()
    group = torch.repeat_interleave(torch.arange(sizes.numel(), device=q.device), sizes, output_size=rows)
    pages = torch.cat([s["prefix_pages"][group], s["row_pages"]], 1).long()
    k, v = _plain_pages(s, pages)
    Lp = s["prefix_pages"].shape[1] * page
    at = torch.arange(k.shape[2], device=q.device)
    t = torch.arange(T, device=q.device)
    in_prefix = (at < s["prefix_lens"][group][:, None])[:, None]                                  # [rows, 1, L]
    limit = s["row_lens"][:, None] - (T - 1 - t)                                                    # [rows, T]
    seen = torch.where(at < Lp, in_prefix, at - Lp < limit[..., None])                              # [rows, T, L]
    qh = q.float().reshape(rows, T, H, R, D).permute(0, 2, 1, 3, 4).reshape(rows, H, T * R, D)
    x = torch.matmul(qh, k.transpose(-1, -2).contiguous()) * s["scale"]
    x = x.reshape(rows, H, T, R, -1).masked_fill_(~seen[:, None, :, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    x = torch.exp(x - m)
    total = x.sum(-1, keepdim=True)
    out = torch.matmul(x.reshape(rows, H, T * R, -1), v).reshape(rows, H, T, R, D) / total
    out = torch.where(total > 0, out, torch.zeros_like(out))
    lse = (m + torch.log(total))[..., 0]
    return {"out": out.permute(0, 2, 1, 3, 4).reshape(rows, T, Hq, D).to(torch.bfloat16),
            "lse": lse.permute(0, 2, 1, 3).reshape(rows, T, Hq)}


def _words(index, row, stream, seed):
    """Word index % 4 of Philox4x32-10(counter (index / 4, row, 0, stream), key = seed): index and row in int64, broadcast."""
    low = 0xFFFFFFFF
    c0, c1 = torch.broadcast_tensors(index >> 2, row)
    c2, c3 = torch.zeros_like(c0), torch.full_like(c0, stream)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57                       # the low 64 bits are right in two's complement
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    w = torch.stack([c0, c1, c2, c3], -1)
    return torch.gather(w, -1, (index & 3).expand(c0.shape)[..., None])[..., 0]


def _uniform(index, row, stream, seed):
    return ((_words(index, row, stream, seed) >> 9).float() + 0.5) * 2.0 ** -23


def _first_max(x):
    """The lowest index of each row's maximum."""
    at = torch.arange(x.shape[1], device=x.device)
    return torch.where(x == x.amax(1, keepdim=True), at, x.shape[1]).amin(1)


def _plain_softmax(z, tau):
    t = (z.float() - z.float().amax(-1, keepdim=True)) / tau
    e = torch.exp(t)
    total = e.sum(-1, keepdim=True)
    entropy = torch.log(total) - (e * t).sum(-1, keepdim=True) / total
    return e / total, (t - torch.log(total)), entropy[..., 0]


def _plain_verify(s):
    z, K, V = s["logits"], s["case"]["drafts"], s["case"]["V"]
    rows = z.shape[0]
    dev = z.device
    tau = s["tau_rows"][:, None, None] if s["tau_rows"] is not None else s["tau"]
    p, logp, entropy = _plain_softmax(z, tau)
    q = _plain_softmax(s["drafter"], tau)[0] if s["drafter"] is not None else None
    row = torch.arange(rows, device=dev)
    draft = s["tokens"].long()
    lens = s["lens"].long() if s["lens"] is not None else torch.full((rows,), K, device=dev)
    at = torch.arange(K + 1, device=dev)
    u = _uniform(at[None, :K], row[:, None], 5, s["seed"])
    px = torch.gather(p[:, :K], 2, draft[..., None])[..., 0]
    qx = torch.gather(q, 2, draft[..., None])[..., 0] if q is not None else torch.ones_like(px)
    ok = (u * qx < px) & (at[:K] < lens[:, None])
    n = torch.cumprod(ok.long(), 1).sum(1)
    pn, cut = p[row, n], (n < lens)[:, None]
    qn = q[row, n.clamp(max=K - 1)] if q is not None else \
        torch.zeros_like(pn).scatter_(1, draft[row, n.clamp(max=K - 1)][:, None], 1.0)
    rest = torch.where(cut, (pn - qn).clamp_(min=0.0), pn)
    rest = torch.where(rest.amax(1, keepdim=True) > 0, rest, pn)
    # the draw: first a tile (512 columns of every 4096 are dealt in chunks of 8 to 64 tiles), then a column of it
    steps = -(-V // 4096)
    rest = torch.nn.functional.pad(rest, (0, steps * 4096 - V)).reshape(rows, steps, 8, 64, 8)
    mass = rest.sum((2, 4)).reshape(rows, steps * 64)
    tiles = torch.arange(steps * 64, device=dev)
    tile = _first_max(mass / -torch.log(_uniform(tiles[None], row[:, None], 6, s["seed"])))
    inside = rest[row, tile // 64, :, tile % 64].reshape(rows, 64)
    j = torch.arange(64, device=dev)
    cols = (tile // 64 * 4096 + tile % 64 * 8)[:, None] + (j // 8 * 512 + j % 8)[None]
    best = _first_max(inside / -torch.log(_uniform(cols, row[:, None], 7, s["seed"])))
    last = cols[row, best]
    token = torch.cat([draft, draft[:, :1]], 1)
    token = torch.where(at == n[:, None], last[:, None], torch.where(at < n[:, None], token, -1))
    out = at <= n[:, None]
    logp = torch.gather(logp, 2, token.clamp(min=0)[..., None])[..., 0]
    return {"accepted": n.to(torch.int32), "token": token.to(torch.int32),
            "logp": torch.where(out, logp, 0.0), "entropy": torch.where(out, entropy, 0.0)}


# ---------------------------------------------------------------- from the definition, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"cache": _exact_cache, "attend": _exact_attend, "verify": _exact_verify}[case["kind"]](s)


def _exact_cache(s):
    made = {}
    for name in ("k", "v"):
        x = s[name].double()
        largest = x.abs().amax(-1, keepdim=True)
        e = torch.ceil(torch.log2(largest / 448.0)).clamp(-126, 127)
        e = torch.where(largest > 448.0 * torch.exp2(e), e + 1, torch.where(largest <= 448.0 * torch.exp2(e - 1), e - 1, e)).clamp(-126, 127)
        y = x / torch.exp2(e)
        # three bits behind the leading one, in steps of 2^-9 below 2^-6
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
        made[name] = torch.round(y / step) * step * torch.exp2(e)
    return made


def _exact_attend(s):
    q, (k, v, ks, vs) = s["q"].double(), s["cache"]
    rows, T, Hq, D = q.shape
    H = k.shape[1]
    out = torch.zeros((rows, T, Hq, D), dtype=torch.float64, device=q.device)
    lse = torch.full((rows, T, Hq), -math.inf, dtype=torch.float64, device=q.device)

    def tokens(pages, n):
        a, b = (x.view(torch.uint8)[pages].view(x.dtype) if ks is not None else x[pages] for x in (k, v))
        a = a.double().transpose(0, 1).reshape(H, -1, D)
        b = b.double().permute(1, 0, 2, 4, 3).reshape(H, -1, D)
        if ks is not None:
            a, b = (x * torch.exp2(y[pages].double() - 127).transpose(0, 1).reshape(H, -1, 1) for x, y in ((a, ks), (b, vs)))
        return a[:, :n], b[:, :n]

    offsets, prefix_lens, row_lens = (s[n].tolist() for n in ("offsets", "prefix_lens", "row_lens"))
    for g in range(len(prefix_lens)):
        kp, vp = tokens(s["prefix_pages"][g].long(), prefix_lens[g])
        for r in range(offsets[g], offsets[g + 1]):
            kr, vr = tokens(s["row_pages"][r].long(), row_lens[r])
            ka, va = torch.cat([kp, kr], 1), torch.cat([vp, vr], 1)
            for t in range(T):
                n = prefix_lens[g] + max(0, row_lens[r] - (T - 1 - t))
                if not n:
                    continue
                x = torch.bmm(q[r, t].reshape(H, Hq // H, D), ka[:, :n].transpose(1, 2).contiguous()) * s["scale"]
                lse[r, t] = torch.logsumexp(x, -1).reshape(Hq)
                out[r, t] = torch.bmm(torch.softmax(x, -1), va[:, :n].contiguous()).reshape(Hq, D)
    return {"out": out, "lse": lse}


def _exact_verify(s):
    z, drafter = s["logits"], s["drafter"]
    rows, K, V = z.shape[0], s["case"]["drafts"], s["case"]["V"]
    dev = z.device
    accepted = torch.zeros(rows, dtype=torch.int32, device=dev)
    token = torch.full((rows, K + 1), -1, dtype=torch.int32, device=dev)
    logp = torch.zeros((rows, K + 1), dtype=torch.float64, device=dev)
    entropy = torch.zeros((rows, K + 1), dtype=torch.float64, device=dev)
    every = torch.arange(V, device=dev)
    tile_of = every // 4096 * 64 + every % 512 // 8
    tiles = torch.arange(-(-V // 4096) * 64, device=dev)
    lens = s["lens"].tolist() if s["lens"] is not None else [K] * rows
    taus = s["tau_rows"].double().tolist() if s["tau_rows"] is not None else [s["tau"]] * rows
    drafts = s["tokens"].tolist()
    one = torch.zeros(1, dtype=torch.int64, device=dev)

    def uniform(index, r, stream):
        return ((_words(index, one + r, stream, s["seed"]) >> 9).double() + 0.5) / 8_388_608

    for r in range(rows):
        ln_p = torch.log_softmax(z[r, :lens[r] + 1].double() / taus[r], -1)
        p = ln_p.exp()
        h = -torch.where(p > 0, p * ln_p, torch.zeros_like(p)).sum(-1)
        q = torch.softmax(drafter[r].double() / taus[r], -1) if drafter is not None else torch.nn.functional.one_hot(s["tokens"][r].long(), V).double()
        u = uniform(torch.arange(K, device=dev), r, 5)
        d = s["tokens"][r].long()[:lens[r]]
        won = (u[:lens[r]] * q[torch.arange(lens[r], device=dev), d] < p[torch.arange(lens[r], device=dev), d]).tolist()
        n = won.index(False) if False in won else lens[r]
        rest = (p[n] - q[n]).clamp(min=0) if n < lens[r] else p[n]
        rest = rest if float(rest.max()) > 0 else p[n]
        mass = torch.zeros(tiles.numel(), dtype=torch.float64, device=dev).index_add_(0, tile_of, rest)
        tile = torch.argmax(mass / -torch.log(uniform(tiles, r, 6)))
        cols = every[tile_of == tile]
        last = int(cols[torch.argmax(rest[cols] / -torch.log(uniform(cols, r, 7)))])
        accepted[r] = n
        said = drafts[r][:n] + [last]
        ids = torch.tensor(said, device=dev)
        token[r, :n + 1] = ids.to(torch.int32)
        logp[r, :n + 1] = ln_p[:n + 1].gather(1, ids[:, None])[:, 0]
        entropy[r, :n + 1] = h[:n + 1]
    return {"accepted": accepted, "token": token, "logp": logp, "entropy": entropy}


# ---------------------------------------------------------------- what a pass cannot do without
def _attend_work(case):
    sizes = _sizes(case)
    rows = sum(sizes)
    prefix, suffix = _spread(case["prefix_lo"], case["prefix_hi"], case["groups"]), _spread(case["suffix_lo"], case["suffix_hi"], rows)
    per = 2 * case["heads"] * (case["D"] + 1 if case["cache"] == "fp8" else 2 * case["D"])        # of a token
    kept = sum(prefix) + sum(suffix)
    seen = sum(suffix) + sum(prefix) * rows / case["groups"]
    out = rows * case["T"] * case["q_heads"] * (2 * 2 * case["D"] + 4)
    return {"bytes": kept * per + out + 4 * kept / case["page"], "flops": 4.0 * case["D"] * case["q_heads"] * case["T"] * seen}


def work(case):
    if case["kind"] == "attend":
        return _attend_work(case)
    if case["kind"] == "cache":                    # written once as codes, read once as codes, given back in bf16
        size = 4 if case["dtype"] == "f32" else 2
        return {"bytes": case["tokens"] * (2 * case["heads"] * ((size + 2) * case["D"] + 2 * (case["D"] + 1)) + 16), "flops": 0}
    size = 4 if case["dtype"] == "f32" else 2
    K = case["drafts"]
    read = case["rows"] * case["V"] * ((K + 1) + (K if case["drafter"] else 0))
    return {"bytes": read * size + case["rows"] * (4 * K + 4 + 12 * (K + 1)), "flops": 4.0 * read}
