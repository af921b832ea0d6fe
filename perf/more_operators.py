"""What the steps around a model's attention are measured on: rotary positions (for training, and on the way into the paged
cache), attention with a sliding window and first tokens that stay visible, and beam search (the selection, and the reordering of
the beams' pages).

A case is a dict of plain values.  `prepare` makes what a program has in hand before the call, `run` is one pass:
with `own` through the entry points of `paper_2505_18573_amd`, without it the operators in plain torch (32 bits, 64 for angles and
for scores that are compared, rounded once at the end).  `exact` gives the same results in 64 bits, `work` what a pass cannot
do without.

The cache's layout (both forms read it): keys [pages, heads, page, D], values [pages, heads, page / 8, D, 8] (eight
tokens of one column next to each other), one exponent byte e + 127 per token and head for each where the cache holds
8 bits; an element is code * 2^e.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # the queries of a training batch of finished rollouts: 16 thousand tokens, all columns turned, one axis
        {"name": "rotate_batch", "kind": "rotate", "tokens": 16_384, "heads": 28, "D": 128, "rot": 128, "axes": 1, "order": "block",
         "pairs": "halves", "dtype": "bf16", "inverse": False, "far": 6000},
        # the gradient for the queries of image patches: narrow heads, three axes (time, height, width), an odd number of tokens
        {"name": "rotate_patches_grad", "kind": "rotate", "tokens": 5003, "heads": 16, "D": 80, "rot": 80, "axes": 3, "order": "block",
         "pairs": "halves", "dtype": "f32", "inverse": True, "far": 2000},
        # one decode step of 64 questions x 8 rollouts: a token each, at any position of long sequences
        {"name": "append_step_512", "kind": "append", "tokens": 512, "q_heads": 28, "heads": 4, "D": 128, "rot": 128, "axes": 1,
         "order": "block", "pairs": "halves", "page": 64, "cache": "fp8", "dtype": "bf16", "whole": False, "far": 1_000_000},
        # prompts with text, images and video among them, all at once: three axes dealt to the columns in turn
        {"name": "append_prompts", "kind": "append", "tokens": 30_001, "q_heads": 28, "heads": 4, "D": 128, "rot": 128, "axes": 3,
         "order": "turns", "pairs": "halves", "page": 64, "cache": "fp8", "dtype": "bf16", "whole": True, "far": 20_000},
        # a single sequence's next token: launches and latency
        {"name": "window_1_row", "kind": "window", "rows": 1, "q_lo": 1, "q_hi": 1, "past_lo": 226, "past_hi": 226, "window": 128,
         "sinks": 4, "q_heads": 12, "heads": 2, "D": 128, "page": 64, "cache": "fp8"},
        # a decode step of 512 rollouts at all stages of responses of up to 6000 tokens
        {"name": "window_512_rows", "kind": "window", "rows": 512, "q_lo": 1, "q_hi": 1, "past_lo": 0, "past_hi": 7000, "window": 4096,
         "sinks": 4, "q_heads": 28, "heads": 4, "D": 128, "page": 64, "cache": "fp8"},
        # rows of one token, of drafted tokens and of pieces of prompts in one batch
        {"name": "window_mixed", "kind": "window", "rows": 33, "q_lo": 1, "q_hi": 300, "past_lo": 0, "past_hi": 2500, "window": 1000,
         "sinks": 16, "q_heads": 12, "heads": 2, "D": 64, "page": 32, "cache": "bf16"},
        # whole prompts of odd lengths, longer than the window
        {"name": "window_prompts", "kind": "window", "rows": 8, "q_lo": 1000, "q_hi": 4001, "past_lo": 0, "past_hi": 0, "window": 1024,
         "sinks": 4, "q_heads": 28, "heads": 4, "D": 128, "page": 64, "cache": "bf16"},
        # 64 sequences of eight beams, twice as many candidates as beams
        {"name": "beam_64x8", "kind": "beam", "seqs": 64, "beams": 8, "keep": 16, "V": 151_936, "dtype": "bf16", "ends": False},
        # one sequence of four beams, some of them finished: launches and latency
        {"name": "beam_1x4", "kind": "beam", "seqs": 1, "beams": 4, "keep": 4, "V": 32_000, "dtype": "f32", "ends": True},
        # the beams' pages after a step of 64 sequences
        {"name": "states_64x8", "kind": "states", "seqs": 64, "beams": 8, "heads": 4, "D": 128, "page": 64, "len_lo": 40, "len_hi": 700},
        # the same for one sequence
        {"name": "states_1x4", "kind": "states", "seqs": 1, "beams": 4, "heads": 2, "D": 64, "page": 32, "len_lo": 301, "len_hi": 301},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _rotary_of(rng, D):
    return {"rot": rng.choice([D, D, D // 32 * 16]), "axes": rng.choice([1, 1, 2, 3]), "order": rng.choice(["block", "turns"]),
            "pairs": rng.choice(["halves", "halves", "neighbours"])}


def draw(rng):
    kind = rng.choice(["rotate", "append", "window", "window", "window", "beam", "beam", "states"])
    if kind == "rotate":
        D = rng.choice([64, 80, 96, 128, 256])
        c = {"kind": kind, "tokens": _log_int(rng, 1, 16_384), "heads": rng.choice([1, 2, 7, 16, 28]), "D": D, **_rotary_of(rng, D),
             "dtype": rng.choice(["bf16", "bf16", "f32"]), "inverse": rng.random() < 0.5, "far": _log_int(rng, 100, 1_000_000)}
        while work(c)["bytes"] > work(listed()[0])["bytes"]:
            c["tokens"] = max(1, c["tokens"] * 2 // 3)
        return c
    if kind == "append":
        heads, D = rng.choice([1, 2, 4, 8]), rng.choice([64, 128])
        c = {"kind": kind, "tokens": _log_int(rng, 1, 30_000), "q_heads": heads * rng.choice([1, 4, 7, 8]), "heads": heads, "D": D,
             **_rotary_of(rng, D), "page": rng.choice([32, 64, 128]), "cache": rng.choice(["fp8", "fp8", "bf16"]),
             "dtype": rng.choice(["bf16", "bf16", "f32"]), "whole": rng.random() < 0.6, "far": _log_int(rng, 100, 1_000_000)}
        while work(c)["bytes"] > work(listed()[3])["bytes"]:
            c["tokens"] = max(1, c["tokens"] * 2 // 3)
        return c
    if kind == "window":
        heads = rng.choice([1, 2, 4, 8])
        shape = rng.choice(["step", "drafts", "mixed", "prompts"])
        lo, hi = {"step": (1, 1), "drafts": (2, 8), "mixed": (0, _log_int(rng, 8, 600)), "prompts": (1, _log_int(rng, 100, 4000))}[shape]
        c = {"kind": kind, "rows": _log_int(rng, 1, 512 if shape in ("step", "drafts") else 40), "q_lo": lo, "q_hi": hi, "past_lo": 0,
             "past_hi": 0 if shape == "prompts" else _log_int(rng, 1, 7000), "window": _log_int(rng, 1, 8000), "sinks": rng.choice([0, 1, 4, 16, 100]),
             "q_heads": heads * rng.choice([1, 4, 7, 8]), "heads": heads, "D": rng.choice([64, 128, 128]), "page": rng.choice([32, 64, 128]),
             "cache": rng.choice(["fp8", "fp8", "bf16"])}
        # no more than the largest listed cases: what is read, what is multiplied, and what the plain form spreads out
        most = [_window_work(listed()[5])["bytes"], _window_work(listed()[7])["flops"], _spread_out(listed()[7]), _held(listed()[5])]
        for _ in range(40):
            w = _window_work(c)
            now = [w["bytes"], w["flops"], _spread_out(c), _held(c)]
            if all(a <= b for a, b in zip(now, most)):
                break
            c["rows"] = max(1, c["rows"] * 2 // 3)
            if c["rows"] == 1:
                c["past_hi"], c["q_hi"] = c["past_hi"] * 2 // 3, max(c["q_lo"], c["q_hi"] * 2 // 3)
        return c
    if kind == "beam":
        beams = _log_int(rng, 1, 16)
        c = {"kind": kind, "seqs": _log_int(rng, 1, 64), "beams": beams, "keep": rng.choice([beams, 2 * beams, 2 * beams, beams + 1]),
             "V": rng.choice([151_936, 32_000, 128_000, _log_int(rng, 1000, 260_000)]), "dtype": rng.choice(["bf16", "bf16", "f32"]),
             "ends": rng.random() < 0.4}
        while work(c)["bytes"] > work(listed()[8])["bytes"]:
            c["seqs"] = max(1, c["seqs"] * 2 // 3)
        return c
    c = {"kind": kind, "seqs": _log_int(rng, 1, 64), "beams": _log_int(rng, 1, 16), "heads": rng.choice([1, 2, 4, 8]),
         "D": rng.choice([64, 128]), "page": rng.choice([32, 64, 128]), "len_lo": _log_int(rng, 1, 300), "len_hi": _log_int(rng, 300, 1500)}
    while c["seqs"] * c["beams"] * (c["len_hi"] + c["page"]) * c["heads"] * c["D"] > 512 * 764 * 4 * 128:
        c["seqs"], c["len_hi"] = max(1, c["seqs"] * 2 // 3), max(c["len_lo"], c["len_hi"] * 4 // 5)
    return c


# ---------------------------------------------------------------- inputs (from the seed alone)
def _rand(g, *shape):
    return torch.rand(shape, generator=g, device=DEV)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _spread(lo, hi, n):
    return [round(lo + (hi - lo) * (i / (n - 1) if n > 1 else 1.0)) for i in range(n)]


def _queries(case):
    """Queries of each row; in mixed batches most rows bring few of them."""
    n = _spread(0, 1000, case["rows"])
    return [case["q_lo"] + round((case["q_hi"] - case["q_lo"]) * (x / 1000) ** (1 if case["q_lo"] >= 1000 else 3)) for x in n]


def _shuffled(values, g):
    v = torch.tensor(values, device=DEV)
    return v[torch.randperm(len(values), generator=g, device=DEV)]


def _cache_of(pages, heads, page, D, kind, g):
    """Keys and values of unit variance with a few louder columns and tokens of different size."""
    col = 1.0 + 3.0 * (_rand(g, heads, 1, D) < 0.03).float()
    made = [[], []]
    for p0 in range(0, pages, 4096):
        n = min(4096, pages - p0)
        made[0].append(_randn(g, n, heads, page, D).mul_(col).to(torch.bfloat16))
        made[1].append(_randn(g, n, heads, page, D).mul_(0.5 + _rand(g, n, heads, page, 1)).to(torch.bfloat16))
    if kind == "bf16":
        k, v = (torch.cat(m) for m in made)
        return k, v.reshape(pages, heads, page // 8, 8, D).transpose(-1, -2).contiguous(), None, None
    out = []
    for parts in made:
        both = [_to_fp8(x.float()) for x in parts]
        out.append((torch.cat([y.view(torch.uint8) for y, _ in both]), torch.cat([(e + 127).to(torch.uint8) for _, e in both])))
    (k, ks), (v, vs) = out
    v = v.reshape(pages, heads, page // 8, 8, D).transpose(-1, -2).contiguous()
    return k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), ks, vs


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return {"rotate": _prepare_rotate, "append": _prepare_append, "window": _prepare_window, "beam": _prepare_beam,
            "states": _prepare_states}[case["kind"]](case, g, seed)


def _rotary(case):
    """Angles per position of each pair of columns, in 64 bits, and the axis each pair goes by."""
    n, axes = case["rot"] // 2, case["axes"]
    i = torch.arange(n, device=DEV)
    freqs = torch.exp(i.double() * (-2.0 * math.log(10_000.0) / case["rot"]))
    axis = (i % axes if case["order"] == "turns" else i * axes // n).to(torch.uint8) if axes > 1 else None
    return freqs, axis


def _positions(case, g):
    """Positions on each axis; the axes of one token are near each other, as those of a picture in a text are."""
    at = torch.randint(0, case["far"], (1, case["tokens"]), generator=g, device=DEV)
    return at + torch.randint(0, 100, (case["axes"], case["tokens"]), generator=g, device=DEV)


def _prepare_rotate(case, g, seed):
    n, H, D = case["tokens"], case["heads"], case["D"]
    x = _randn(g, n, H + 2, D).to(DTYPES[case["dtype"]])[:, :H]          # a part of a projection's rows
    return {"case": case, "x": x, "rotary": _rotary(case), "positions": _positions(case, g)}


def _prepare_append(case, g, seed):
    n, Hq, H, D, page = case["tokens"], case["q_heads"], case["heads"], case["D"], case["page"]
    # one row of the projection's output: query heads, then key heads, then value heads
    qkv = (_randn(g, n, Hq + 2 * H, D) * (0.2 + 3.0 * _rand(g, n, Hq + 2 * H, 1))).to(DTYPES[case["dtype"]])
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
    if case["cache"] == "fp8":
        cache = (torch.zeros((pages, H, page, D), dtype=torch.float8_e4m3fn, device=DEV),
                 torch.zeros((pages, H, page // 8, D, 8), dtype=torch.float8_e4m3fn, device=DEV),
                 torch.zeros((pages, H, page), dtype=torch.uint8, device=DEV),
                 torch.zeros((pages, H, page), dtype=torch.uint8, device=DEV))
    else:
        cache = (torch.zeros((pages, H, page, D), dtype=torch.bfloat16, device=DEV),
                 torch.zeros((pages, H, page // 8, D, 8), dtype=torch.bfloat16, device=DEV), None, None)
    return {"case": case, "q": qkv[:, :Hq], "k": qkv[:, Hq:Hq + H], "v": qkv[:, Hq + H:], "slots": slots.long(), "cache": cache,
            "rotary": _rotary(case), "positions": _positions(case, g)}


def _prepare_window(case, g, seed):
    rows, page = case["rows"], case["page"]
    order = torch.randperm(rows, generator=g, device=DEV)
    queries = torch.tensor(_queries(case), device=DEV)[order]
    past = _shuffled(_spread(case["past_lo"], case["past_hi"], rows), g)
    offsets = torch.zeros(rows + 1, dtype=torch.int32, device=DEV)
    offsets[1:] = torch.cumsum(queries, 0)
    width = max(1, -(-(case["past_hi"] + case["q_hi"]) // page))
    pages = rows * width
    table = torch.randperm(pages, generator=g, device=DEV).reshape(rows, width)
    q = _randn(g, sum(_queries(case)), case["q_heads"], case["D"]).to(torch.bfloat16)
    return {"case": case, "q": q, "cache": _cache_of(pages, case["heads"], page, case["D"], case["cache"], g), "offsets": offsets,
            "row_pages": table.to(torch.int32), "row_lens": (past + queries).to(torch.int32), "scale": case["D"] ** -0.5}


def _prepare_beam(case, g, seed):
    n, B, V = case["seqs"], case["beams"], case["V"]
    per = 8 if case["dtype"] == "bf16" else 4                        # rows start on 16 bytes
    pitch = -(-V // per) * per
    logits = torch.empty((n, B, pitch), dtype=DTYPES[case["dtype"]], device=DEV)
    for s0 in range(0, n, 8):
        m = min(8, n - s0)
        x = _randn(g, m, B, pitch).mul_(3.0)
        cols = torch.randint(0, V, (m, B, 20), generator=g, device=DEV)
        logits[s0:s0 + m] = x.scatter_(2, cols, torch.gather(x, 2, cols) + 8.0)
    scores = -20.0 - 2.0 * _rand(g, n, B)
    finished = (_rand(g, n, B) < 0.3).to(torch.uint8) if case["ends"] else None
    return {"case": case, "logits": logits[..., :V], "scores": scores, "finished": finished, "eos": 2, "tau": 0.9}


def _prepare_states(case, g, seed):
    n, B, page, H, D = case["seqs"], case["beams"], case["page"], case["heads"], case["D"]
    lens = _shuffled(_spread(case["len_lo"], case["len_hi"], n), g)[:, None].expand(n, B).reshape(-1)
    width = case["len_hi"] // page + 1
    pages = n * B * width
    table = torch.randperm(pages, generator=g, device=DEV).reshape(n * B, width)
    k = _randn(g, pages, H, page, D).to(torch.bfloat16)
    v = _randn(g, pages, H, page // 8, D, 8).to(torch.bfloat16)
    parent = torch.randint(0, B, (n, B), generator=g, device=DEV).to(torch.int32)
    return {"case": case, "parent": parent, "row_pages": table.to(torch.int32), "row_lens": lens.to(torch.int32).contiguous(),
            "cache": (k, v, None, None)}


# ---------------------------------------------------------------- one pass
def run(s):
    kind = s["case"]["kind"]
    if own:
        import paper_2505_18573_amd as e3
        if kind == "rotate":
            return {"y": e3.e3_rotate(s["x"], e3.E3Rotary(*s["rotary"], s["case"]["pairs"] == "neighbours"), s["positions"],
                                      inverse=s["case"]["inverse"])}
        if kind == "append":
            cache = e3.E3Cache(*s["cache"])
            q = e3.e3_cache_append_rotated(cache, s["q"], s["k"], s["v"], e3.E3Rotary(*s["rotary"], s["case"]["pairs"] == "neighbours"),
                                           s["positions"], s["slots"])
            k, v = e3.e3_cache_read(cache, s["slots"])
            return {"q": q, "k": k, "v": v}
        if kind == "window":
            out, lse = e3.e3_window_attention(s["q"], e3.E3Cache(*s["cache"]), s["offsets"], s["row_pages"], s["row_lens"],
                                              s["case"]["window"], s["case"]["sinks"], s["scale"])
            return {"out": out, "lse": lse}
        if kind == "beam":
            parent, token, score = e3.e3_beam_select(s["logits"], s["scores"], s["case"]["keep"], s["tau"], s["finished"], s["eos"])
            return {"parent": parent, "token": token, "score": score}
        cache = e3.E3Cache(*s["cache"])
        pages, lens, src, dst, counts = e3.e3_beam_reorder(s["parent"], s["row_pages"], s["row_lens"], s["case"]["page"])
        e3.e3_cache_copy(cache, src, dst, counts)
        return {"pages": pages, "lens": lens, "k": cache.k, "v": cache.v}
    return {"rotate": _plain_rotate, "append": _plain_append, "window": _plain_window, "beam": _plain_beam,
            "states": _plain_states}[kind](s)


def _plain_turned(s, x, inverse=False):
    """x [tokens, heads, D], rotated, in 32 bits."""
    freqs, axis = s["rotary"]
    neighbours = s["case"]["pairs"] == "neighbours"
    n = freqs.numel()
    at = s["positions"][axis.long()] if axis is not None else s["positions"][:1].expand(n, -1)      # [n, tokens]
    angle = (at.double() * freqs[:, None]).t()[:, None]
    c, d = torch.cos(angle).float(), torch.sin(angle).float()
    d = -d if inverse else d
    x = x.float()
    a, b = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if neighbours else (x[..., :n], x[..., n:2 * n])
    a, b = a * c - b * d, b * c + a * d
    turned = torch.stack([a, b], -1).flatten(-2) if neighbours else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., 2 * n:]], -1)


def _plain_rotate(s):
    return {"y": _plain_turned(s, s["x"], s["case"]["inverse"]).to(s["x"].dtype)}


def _to_fp8(x):
    """Codes and exponents of the last axis' vectors: the smallest power of two that brings the largest to at most 448."""
    a = x.abs().amax(-1)
    m, e = torch.frexp(a)                                            # a = m 2^e, m in [1/2, 1); 448 = 7/8 2^9
    e = (e - 9 + (m > 0.875)).clamp(-126, 127)
    return torch.ldexp(x, -e[..., None]).to(torch.float8_e4m3fn), e


def _plain_append(s):
    def stored(x):
        if s["case"]["cache"] == "bf16":
            return x.to(torch.bfloat16)
        y, e = _to_fp8(x)
        return torch.ldexp(y.float(), e[..., None]).to(torch.bfloat16)

    return {"q": _plain_turned(s, s["q"]).to(s["q"].dtype), "k": stored(_plain_turned(s, s["k"])), "v": stored(s["v"].float())}


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


def _plain_window(s):
    q, c = s["q"], s["case"]
    total, Hq, D = q.shape
    rows, H, T = c["rows"], c["heads"], max(1, c["q_hi"])
    R = Hq // H
    k, v = _plain_pages(s, s["row_pages"].long())
    L = k.shape[2]
    # every row's queries, filled up to the largest number of them
    n = (s["offsets"][1:] - s["offsets"][:-1]).long()
    t = torch.arange(T, device=q.device)
    source = s["offsets"][:-1, None].long() + t
    real = t < n[:, None]                                                                            # [rows, T]
    qh = q[source.clamp(max=max(0, total - 1))].float().reshape(rows, T, H, R, D).permute(0, 2, 3, 1, 4).reshape(rows, H, R * T, D)
    p = (s["row_lens"].long() - n)[:, None] + t
    j = torch.arange(L, device=q.device)
    seen = (j <= p[..., None]) & ((j > p[..., None] - c["window"]) | (j < c["sinks"]))               # [rows, T, L]
    x = torch.matmul(qh, k.transpose(-1, -2).contiguous()).mul_(s["scale"]).reshape(rows, H, R, T, L)
    x.masked_fill_(~seen[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    x = x.sub_(m).exp_()
    sums = x.sum(-1, keepdim=True)
    out = torch.matmul(x.reshape(rows, H, R * T, L), v).reshape(rows, H, R, T, D) / sums
    out = torch.where(sums > 0, out, torch.zeros_like(out)).permute(0, 3, 1, 2, 4).reshape(rows, T, Hq, D)
    lse = (m + torch.log(sums))[..., 0].permute(0, 3, 1, 2).reshape(rows, T, Hq)
    return {"out": out[real].to(torch.bfloat16), "lse": lse[real]}


def _plain_beam(s):
    """Scores in 64 bits: they are compared, and near ones must not change places."""
    z, c = s["logits"], s["case"]
    n, B, V = z.shape
    x = z.double() / s["tau"]
    m = x.amax(-1, keepdim=True)
    x = s["scores"].double()[..., None] + (x - m) - torch.log(torch.exp(x - m).sum(-1, keepdim=True))
    if s["finished"] is not None:
        only = torch.full_like(x[:1, :1], -math.inf).expand(n, B, V).clone()
        only[..., s["eos"]] = s["scores"].double()
        x = torch.where(s["finished"].bool()[..., None], only, x)
    score, index = torch.sort(x.reshape(n, B * V), dim=1, descending=True, stable=True)
    score, index = score[:, :c["keep"]], index[:, :c["keep"]]
    none = score == -math.inf                                        # fewer candidates than asked for
    return {"parent": torch.where(none, -1, index // V).to(torch.int32), "token": torch.where(none, -1, index % V).to(torch.int32),
            "score": score.float()}


def _heirs(parent):
    """Of rows [sequences, beams]: whether each is its parent's first child, and which childless row the others take a page of."""
    n, B = parent.shape
    b = torch.arange(B, device=parent.device)
    same = parent[:, :, None] == parent[:, None, :]
    first = ~(same & (b[None, None, :] < b[None, :, None])).any(-1)
    childless = ~(parent[:, :, None] == b[None, None, :]).any(1)
    # the j-th row that is no first child takes the page of the j-th row without children
    rank = torch.cumsum((~first).long(), 1) - 1
    donors = torch.sort(torch.where(childless, b, B + b), dim=1).values
    donor = torch.gather(donors, 1, rank.clamp(min=0)) % B
    return first, donor


def _plain_states(s):
    parent, c = s["parent"].long(), s["case"]
    n, B = parent.shape
    width, page = s["row_pages"].shape[1], c["page"]
    first, donor = _heirs(parent)
    base = torch.arange(n, device=parent.device)[:, None] * B
    p, d = (base + parent).reshape(-1), (base + donor).reshape(-1)
    first = first.reshape(-1)
    lens = s["row_lens"].long()
    at = lens // page                                                # the entry that the next token goes to
    pages = s["row_pages"][p]
    last = torch.where(first, s["row_pages"][p, at[p]], s["row_pages"][d, at[d]])
    pages = torch.where(torch.arange(width, device=parent.device) == at[p][:, None], last[:, None], pages)
    k, v = s["cache"][0], s["cache"][1]
    count = torch.where(first, torch.zeros_like(p), (lens[p] % page + 7) // 8 * 8)
    src, dst = s["row_pages"][p, at[p]].long(), torch.where(first, s["row_pages"][p, at[p]], last).long()
    t = torch.arange(page, device=parent.device)
    keep = t < count[:, None]                                        # [rows, page]
    k[dst] = torch.where(keep[:, None, :, None], k[src], k[dst])
    v[dst] = torch.where(keep[:, ::8][:, None, :, None, None], v[src], v[dst])
    return {"pages": pages, "lens": lens[p].to(torch.int32), "k": k, "v": v}


# ---------------------------------------------------------------- from the definition, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"rotate": _exact_rotate, "append": _exact_append, "window": _exact_window, "beam": _exact_beam,
            "states": _exact_states}[case["kind"]](s)


def _exact_turned(s, x, inverse=False):
    """Pair by pair as a product of complex numbers."""
    freqs, axis = s["rotary"]
    y = x.double().clone()
    n = freqs.numel()
    for i in range(n):
        at = s["positions"][int(axis[i]) if axis is not None else 0].double()
        turn = torch.polar(torch.ones_like(at), at * freqs[i] * (-1.0 if inverse else 1.0))[:, None]
        a, b = (2 * i, 2 * i + 1) if s["case"]["pairs"] == "neighbours" else (i, i + n)
        z = torch.complex(x[..., a].double(), x[..., b].double()) * turn
        y[..., a], y[..., b] = z.real, z.imag
    return y


def _exact_rotate(s):
    return {"y": _exact_turned(s, s["x"], s["case"]["inverse"])}


def _exact_stored(s, x):
    if s["case"]["cache"] == "bf16":
        return x
    largest = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(largest / 448.0)).clamp(-126, 127)
    e = torch.where(largest > 448.0 * torch.exp2(e), e + 1, torch.where(largest <= 448.0 * torch.exp2(e - 1), e - 1, e)).clamp(-126, 127)
    y = x / torch.exp2(e)
    # three bits behind the leading one, in steps of 2^-9 below 2^-6
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * torch.exp2(e)


def _exact_append(s):
    return {"q": _exact_turned(s, s["q"]), "k": _exact_stored(s, _exact_turned(s, s["k"])), "v": _exact_stored(s, s["v"].double())}


def _exact_window(s):
    q, (k, v, ks, vs), c = s["q"].double(), s["cache"], s["case"]
    total, Hq, D = q.shape
    H, W, S = k.shape[1], c["window"], c["sinks"]
    out = torch.zeros((total, Hq, D), dtype=torch.float64, device=q.device)
    lse = torch.full((total, Hq), -math.inf, dtype=torch.float64, device=q.device)
    offsets, lens = s["offsets"].tolist(), s["row_lens"].tolist()
    for r in range(c["rows"]):
        pages = s["row_pages"][r].long()
        a, b = (x.view(torch.uint8)[pages].view(x.dtype) if ks is not None else x[pages] for x in (k, v))
        a = a.double().transpose(0, 1).reshape(H, -1, D)
        b = b.double().permute(1, 0, 2, 4, 3).reshape(H, -1, D)
        if ks is not None:
            a, b = (x * torch.exp2(y[pages].double() - 127).transpose(0, 1).reshape(H, -1, 1) for x, y in ((a, ks), (b, vs)))
        n = offsets[r + 1] - offsets[r]
        for t0 in range(0, n, 256):                                   # a block of queries: the tokens that any of them sees
            t1 = min(n, t0 + 256)
            p = lens[r] - n + torch.arange(t0, t1, device=q.device)
            lo, hi = max(0, int(p[0]) - W + 1), int(p[-1]) + 1
            ids = torch.cat([torch.arange(0, min(S, lo), device=q.device), torch.arange(lo, hi, device=q.device)])
            gap = p[:, None] - ids[None]
            hidden = (gap < 0) | ((gap >= W) & (ids[None] >= S))
            x = q[offsets[r] + t0:offsets[r] + t1].reshape(t1 - t0, H, Hq // H, D).permute(1, 2, 0, 3).reshape(H, -1, D)
            x = torch.bmm(x, a[:, ids].transpose(1, 2).contiguous()).reshape(H, Hq // H, t1 - t0, -1) * s["scale"]
            x = x.masked_fill(hidden, -math.inf)
            lse[offsets[r] + t0:offsets[r] + t1] = torch.logsumexp(x, -1).reshape(Hq, -1).t()
            y = torch.bmm(torch.softmax(x, -1).reshape(H, -1, ids.numel()), b[:, ids].contiguous())
            out[offsets[r] + t0:offsets[r] + t1] = y.reshape(H, Hq // H, t1 - t0, D).permute(2, 0, 1, 3).reshape(t1 - t0, Hq, D)
    return {"out": out, "lse": lse}


def _exact_beam(s):
    z, c = s["logits"], s["case"]
    n, B, V = z.shape
    keep = c["keep"]
    parent, token = (torch.zeros((n, keep), dtype=torch.int32, device=z.device) for _ in range(2))
    score = torch.zeros((n, keep), dtype=torch.float64, device=z.device)
    for i in range(n):
        x = torch.log_softmax(z[i].double() / s["tau"], -1) + s["scores"][i].double()[:, None]
        if s["finished"] is not None:
            for b in torch.nonzero(s["finished"][i])[:, 0].tolist():
                x[b] = -math.inf
                x[b, s["eos"]] = s["scores"][i, b].double()
        flat = x.reshape(-1)
        border = torch.topk(flat, keep).values[-1]
        near = torch.nonzero(flat >= border)[:, 0]                   # in index order
        order = torch.sort(flat[near], descending=True, stable=True).indices[:keep]
        best = flat[near[order]]
        there = torch.isfinite(best)
        parent[i], token[i] = torch.where(there, near[order] // V, -1).int(), torch.where(there, near[order] % V, -1).int()
        score[i] = best
    return {"parent": parent, "token": token, "score": score}


def _exact_states(s):
    page, parents = s["case"]["page"], s["parent"].tolist()
    table, lens = s["row_pages"].tolist(), s["row_lens"].tolist()
    B = len(parents[0])
    k, v = (x.clone() for x in s["cache"][:2])
    pages, out_lens, moved = [], [], []
    for i, of in enumerate(parents):
        free = [b for b in range(B) if b not in of]
        had = set()
        for r in range(B):
            p = i * B + of[r]
            at = lens[p] // page
            row = list(table[p])
            if of[r] in had:
                d = i * B + free.pop(0)
                row[at] = table[d][lens[d] // page]
                moved.append((table[p][at], row[at], -(-(lens[p] % page) // 8)))
            had.add(of[r])
            pages.append(row)
            out_lens.append(lens[p])
    for a, b, blocks in moved:
        k[b, :, :8 * blocks] = s["cache"][0][a, :, :8 * blocks]
        v[b, :, :blocks] = s["cache"][1][a, :, :blocks]
    as_int = lambda x: torch.tensor(x, dtype=torch.int32, device=k.device)
    return {"pages": as_int(pages), "lens": as_int(out_lens), "k": k.double(), "v": v.double()}


# ---------------------------------------------------------------- what a pass cannot do without
def _window_rows(case):
    """(queries, tokens before them) of each row, as if both grew together."""
    return list(zip(_queries(case), _spread(case["past_lo"], case["past_hi"], case["rows"])))


def _pairs(n, past, W, S):
    """Visible (query, key) pairs of a row: sums of min(p + 1, W) and of the first tokens outside the window."""
    def upto(x, most):                                               # sum over p < x of min(p + 1, most)
        a = min(x, most)
        return a * (a + 1) // 2 + (x - a) * most

    end = past + n
    in_window = upto(end, W) - upto(past, W)
    outside = [upto(max(0, x - W), S) for x in (past, end)]          # a first token at distance W and more
    return in_window + (outside[1] - outside[0])


def _window_work(case):
    W, S = case["window"], case["sinks"]
    per = 2 * case["heads"] * (case["D"] + 1 if case["cache"] == "fp8" else 2 * case["D"])        # of a token
    kept = pairs = 0
    for n, past in _window_rows(case):
        lo = max(0, past - W + 1)
        kept += (past + n - lo + min(S, lo)) if n else 0
        pairs += _pairs(n, past, W, S)
    out = sum(_queries(case)) * case["q_heads"] * (2 * 2 * case["D"] + 4)
    return {"bytes": kept * per + out + 4 * kept / case["page"] + 8 * case["rows"], "flops": 4.0 * case["D"] * case["q_heads"] * pairs}


def _spread_out(case):
    return case["rows"] * case["q_heads"] * max(1, case["q_hi"]) * (case["past_hi"] + case["q_hi"] + case["page"])


def _held(case):
    return case["rows"] * (case["past_hi"] + case["q_hi"] + case["page"]) * case["heads"] * case["D"]


def work(case):
    size = {"bf16": 2, "f32": 4}
    if case["kind"] == "rotate":
        n = case["tokens"] * case["heads"]
        return {"bytes": 2 * n * case["D"] * size[case["dtype"]] + 8 * case["axes"] * case["tokens"], "flops": 3.0 * n * case["rot"]}
    if case["kind"] == "append":                   # queries in and out; keys and values in, into the cache, and back in bf16
        n, D, H = case["tokens"], case["D"], case["heads"]
        held = D + 1 if case["cache"] == "fp8" else 2 * D
        per = 2 * case["q_heads"] * D * size[case["dtype"]] + 2 * H * (D * (size[case["dtype"]] + 2) + 2 * held)
        return {"bytes": n * (per + 16 + 8 * case["axes"]), "flops": 3.0 * n * (case["q_heads"] + H) * case["rot"]}
    if case["kind"] == "window":
        return _window_work(case)
    rows = case["seqs"] * case["beams"]
    if case["kind"] == "beam":
        return {"bytes": rows * case["V"] * size[case["dtype"]] + 4 * rows + 12 * case["seqs"] * case["keep"], "flops": 4.0 * rows * case["V"]}
    # a table's row in and out, and for each row beyond a parent's first child (a share (1 - 1/B)^B of them) half a page in and out
    width = case["len_hi"] // case["page"] + 1
    more = rows * (1 - 1 / case["beams"]) ** case["beams"]
    return {"bytes": rows * (8 * width + 12) + more * 2 * case["page"] / 2 * 4 * case["heads"] * case["D"], "flops": 0}
