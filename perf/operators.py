"""The attention side of a decode step, measured operator by operator.

Four kinds of work, at the sizes of the models that the benchmark takes its linear layers from (LLaMA3-8B: hidden 4096, 32 query and
8 key heads of 128; LLaMA3-70B: hidden 8192, 64 and 8 of 128; Qwen3-32B: hidden 5120, 64 and 8 of 128) and at generic ones:

  tables     `torq_block_tables`: pages of a paged key-value cache handed out, and the slots of a step's new tokens
  append     `torq_cache_append`: a step's keys and values written to their slots, as bf16 or MXFP8
  attention  `torq_paged_attention`: one new token of each request over its pages
  norm       `torq_add_rms_norm`: residual addition and root-mean-square norm, to bf16 or MXFP8

Each is computed in elementary torch operations in 32 bits where `own` is false, and by the framework's call where it is true.
MXFP8 tensors are handed over as torch's float8_e4m3fn elements and float8_e8m0fnu scales, one for 32 elements.
"""
import math

import torch

own = False
DEVICE = "cuda:0"
F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
MOST_BYTES, MOST_FLOPS = 1.9e9, 2.9e10  # of a drawn attention
MOST_NORM = 8192 * 8192
MOST_APPEND = 8192 * 8 * 128
MOST_TOKENS = 1 << 18


def listed():
    return [
        # bookkeeping of a decode step: 256 running requests, a token each; one in sixteen or so needs a new page
        {"name": "tables_decode_256", "kind": "tables", "B": 256, "low": 1, "high": 32768, "new": 1, "page": 16},
        # bookkeeping of a prefill step: 61 prompts that start with an empty cache
        {"name": "tables_prefill_61", "kind": "tables", "B": 61, "low": 1, "high": 8192, "new": 0, "page": 64},
        # a decode step of sixteen sequences: their new keys and values (LLaMA3-8B or 70B) to their slots
        {"name": "append_decode_16", "kind": "append", "T": 16, "heads": 8, "head_dim": 128, "page": 16, "format": "bf16", "layout": "heads"},
        # prefill of 8192 tokens into an 8-bit cache, keys and values being columns of one projection's output
        {"name": "append_prefill_mxfp8", "kind": "append", "T": 8192, "heads": 8, "head_dim": 128, "page": 64, "format": "mxfp8", "layout": "heads"},
        # one sequence early in its answer (LLaMA3-8B): a launch or two, latency counts
        {"name": "attention_1_short", "kind": "attention", "B": 1, "heads": 32, "kv_heads": 8, "head_dim": 128, "page": 16,
         "low": 333, "high": 333, "empty": 0, "format": "bf16", "layout": "heads"},
        # sixteen sequences of ragged length (LLaMA3-70B), the decode step beside block_decode_16 of the linear layers
        {"name": "attention_16", "kind": "attention", "B": 16, "heads": 64, "kv_heads": 8, "head_dim": 128, "page": 16,
         "low": 1000, "high": 8192, "empty": 0, "format": "bf16", "layout": "heads"},
        # one sequence of 131072 tokens: eight pairs of a request and a key head for the whole GPU
        {"name": "attention_1_long", "kind": "attention", "B": 1, "heads": 64, "kv_heads": 8, "head_dim": 128, "page": 64,
         "low": 131072, "high": 131072, "empty": 0, "format": "bf16", "layout": "heads"},
        # a captured batch of 77 places, ten of them idle, every query head with a key head of its own, odd head and page sizes, tokens outermost in a page
        {"name": "attention_77_mha", "kind": "attention", "B": 77, "heads": 20, "kv_heads": 20, "head_dim": 80, "page": 48,
         "low": 1, "high": 2048, "empty": 10, "format": "bf16", "layout": "tokens"},
        # a batch of 45 (Qwen3-32B) with long contexts in an 8-bit cache: the largest
        {"name": "attention_45_mxfp8", "kind": "attention", "B": 45, "heads": 64, "kv_heads": 8, "head_dim": 128, "page": 32,
         "low": 8000, "high": 32768, "empty": 0, "format": "mxfp8", "layout": "heads"},
        # the norm ahead of a decode step's q, k, v (LLaMA3-8B): latency
        {"name": "norm_1_row", "kind": "norm", "M": 1, "d": 4096, "residual": True, "format": "bf16"},
        # the same in a prefill of 8192 tokens (LLaMA3-70B)
        {"name": "norm_prefill_70b", "kind": "norm", "M": 8192, "d": 8192, "residual": True, "format": "bf16"},
        # ahead of a layer that is kept at 8 bits, a chunk of 2048 tokens (Qwen3-32B)
        {"name": "norm_chunk_mxfp8", "kind": "norm", "M": 2048, "d": 5120, "residual": True, "format": "mxfp8"},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(["tables", "append", "attention", "attention", "attention", "norm", "norm"])
    form = rng.choice(["bf16", "bf16", "mxfp8"])
    page = 16 * _log(rng, 1, 8)
    if kind == "tables":
        B = _log(rng, 1, 2000)
        new = rng.choice([0, 1, 1, 5])
        high = _log(rng, 16, max(16, MOST_TOKENS // B))
        return {"kind": kind, "B": B, "low": rng.randint(0, min(64, high)), "high": high, "new": new, "page": page}
    dims = [32, 64, 96, 128, 192, 256] if form == "mxfp8" else [64, 72, 80, 96, 112, 128, 128, 128, 192, 256]
    layout = rng.choice(["heads", "heads", "tokens"])
    if kind == "append":
        heads, dim = rng.choice([1, 2, 4, 8, 8, 20]), rng.choice(dims)
        T = _log(rng, 1, max(1, MOST_APPEND // heads // dim))
        return {"kind": kind, "T": T, "heads": heads, "head_dim": dim, "page": page, "format": form, "layout": layout}
    if kind == "attention":
        kv = rng.choice([1, 2, 4, 8, 8, 8, 20])
        group = rng.choice([1, 2, 4, 5, 7, 8, 8, 12, 16, 24])
        dim, B = rng.choice(dims), _log(rng, 1, 256)
        high = _log(rng, 1, 131072)
        case = {"kind": kind, "B": B, "heads": kv * group, "kv_heads": kv, "head_dim": dim, "page": page,
                "low": max(1, int(high * rng.random())), "high": high, "empty": rng.choice([0, 0, B // 8]), "format": form, "layout": layout}
        while case["high"] > 1 and (work(case)["bytes"] > MOST_BYTES or work(case)["flops"] > MOST_FLOPS):
            case.update(low=max(1, case["low"] // 2), high=case["high"] // 2)
        return case
    d = rng.choice([32 * _log(rng, 2, 896), 1024 * rng.randint(1, 28)])
    M = _log(rng, 1, max(1, MOST_NORM // d))
    return {"kind": kind, "M": M, "d": d, "residual": rng.random() < 0.8, "format": form}


def _spread(n, low, high):
    """n whole numbers over [low, high] in no order, the same for every seed: what a pass has to read goes by them."""
    return [low + int((high - low + 1) * ((0.5 + 0.6180339887498949 * (i + 1)) % 1.0)) for i in range(n)]


def _requests(case):
    """Tokens that each request has in the cache and after the step."""
    if case["kind"] == "tables":
        lengths = _spread(case["B"], case["low"], case["high"])
        return [max(0, n - case["new"]) if case["new"] else 0 for n in lengths], lengths
    lengths = _spread(case["B"], case["low"], case["high"])
    for i in range(case["empty"]):
        lengths[(7 * i + 3) % case["B"]] = 0
    return None, lengths


def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _quantised(x):
    """MXFP8 of the last dimension's blocks of 32: elements, and the scales as powers of two.  The scale is the least power of two
    that leaves no element above 448, E4M3's largest value."""
    blocks = x.float().unflatten(-1, (-1, 32))
    mantissa, exponent = torch.frexp(blocks.abs().amax(-1))  # amax = mantissa 2^exponent, mantissa in [0.5, 1); 448 = 0.875 2^9
    byte = (exponent - 9 + (mantissa > 0.875) + 127).clamp(0, 254)
    elements = torch.ldexp(blocks, 127 - byte.unsqueeze(-1)).flatten(-2).to(F8)
    return elements, byte.to(torch.uint8).view(E8)


def _values(elements, scales):
    return (elements.float().unflatten(-1, (-1, 32)) * scales.float().unsqueeze(-1)).flatten(-2)


def _paged(pages, case, dtype, last):
    """An uninitialised [pages, heads, page, last], in memory in that order or with a page's tokens ahead of its heads."""
    heads = case.get("kv_heads", case["heads"])
    if case["layout"] == "heads":
        return torch.empty((pages, heads, case["page"], last), dtype=dtype, device=DEVICE)
    return torch.empty((pages, case["page"], heads, last), dtype=dtype, device=DEVICE).transpose(1, 2)


def _fill(cache, seed, outliers):
    """Normal values, a few channels of them larger (keys have such), in `cache`, in pieces."""
    g, channel = _gen(seed), torch.ones(cache.shape[-1], device=DEVICE)
    channel[:: max(1, cache.shape[-1] // outliers) if outliers else cache.shape[-1] + 1] = 3.0 if outliers else 1.0
    step = max(1, (1 << 26) // cache[0].numel())
    for i in range(0, cache.shape[0], step):
        part = cache[i : i + step]
        yield i, part, torch.randn(part.shape, generator=g, device=DEVICE) * channel


def _prepare_attention(case, seed):
    B, dim, page = case["B"], case["head_dim"], case["page"]
    _, lengths = _requests(case)
    need = [-(-n // page) for n in lengths]
    pages, width = sum(need) + 3, max(max(need), 1) + 1
    order, tables, at = torch.randperm(pages, generator=_gen(seed), device=DEVICE).tolist(), [], 0
    for n in need:
        tables.append(order[at : at + n] + [-1] * (width - n))
        at += n
    state = {"tables": _ints(tables), "lengths": _ints(lengths),
             "q": torch.randn((B, case["heads"], dim), generator=_gen(seed + 1), device=DEVICE).bfloat16(), "scale": dim ** -0.5}
    for name, outliers, s in (("k", 4, seed + 2), ("v", 0, seed + 3)):
        if case["format"] == "bf16":
            cache = _paged(pages, case, torch.bfloat16, dim)
            for _, part, x in _fill(cache, s, outliers):
                part.copy_(x)
        else:
            cache, scales = _paged(pages, case, F8, dim), _paged(pages, case, torch.uint8, dim // 32)
            for i, part, x in _fill(cache, s, outliers):
                elements, e = _quantised(x)
                part.copy_(elements)
                scales[i : i + part.shape[0]].copy_(e.view(torch.uint8))
            state[name + "_scales"] = scales.view(E8)
        state[name] = cache
    return state


def _prepare_append(case, seed):
    T, heads, dim, page = case["T"], case["heads"], case["head_dim"], case["page"]
    pages = -(-T // page) + 8
    both = torch.randn((T, 2, heads, dim), generator=_gen(seed), device=DEVICE)
    both[:, 0, :, :: max(1, dim // 4)] *= 3.0
    both = both.bfloat16()
    state = {"key": both[:, 0], "value": both[:, 1]}
    if T <= 256:  # tokens of a decode step lie wherever their requests have come to
        state["slots"] = torch.randperm(pages * page, generator=_gen(seed + 1), device=DEVICE)[:T]
    else:  # a prompt's go to whole pages, in the order in which those were handed out
        order = torch.randperm(pages, generator=_gen(seed + 1), device=DEVICE)
        token = torch.arange(T, device=DEVICE)
        state["slots"] = order[token // page] * page + token % page
    for name in ("k", "v"):
        state[name] = _paged(pages, case, torch.bfloat16 if case["format"] == "bf16" else F8, dim).zero_()
        if case["format"] == "mxfp8":
            state[name + "_scales"] = _paged(pages, case, torch.uint8, dim // 32).zero_().view(E8)
    return state


def prepare(case, seed):
    seed = 1000 * int(seed)
    kind = case["kind"]
    if kind == "tables":
        held, lengths = _requests(case)
        page = case["page"]
        width = -(-max(max(lengths), 1) // page) + 2
        pages = sum(-(-n // page) for n in lengths) + 5
        order = torch.randperm(pages, generator=_gen(seed), device=DEVICE).tolist()
        tables, at = [], 0
        for n in held:
            n = -(-n // page)
            tables.append(order[at : at + n] + [-1] * (width - n))
            at += n
        state = {"held": _ints(held), "lengths": _ints(lengths), "free": _ints(order), "cursor": _ints([at]), "page": page,
                 "tables": _ints(tables), "tokens": sum(n - m for m, n in zip(held, lengths)), "after": _ints([0])}
    elif kind == "append":
        state = _prepare_append(case, seed)
    elif kind == "attention":
        state = _prepare_attention(case, seed)
    else:
        M, d = case["M"], case["d"]
        g = _gen(seed)
        x = torch.randn((M, d), generator=g, device=DEVICE)
        x[:, :: max(1, d // 40)] *= 20.0
        state = {"x": x.bfloat16(), "residual": (torch.randn((M, d), generator=g, device=DEVICE) * 4.0).bfloat16() if case["residual"] else None,
                 "weight": (1.0 + 0.2 * torch.randn(d, generator=g, device=DEVICE)).bfloat16(), "eps": 1e-5, "format": case["format"]}
    if own and kind in ("append", "attention"):
        from paper_2605_19561_amd import binding as tq
        state["cache"] = tq.KVCache(state["k"], state["v"], state.get("k_scales"), state.get("v_scales"))
    return dict(state, kind=kind)


def _tables(s):
    page, width, tables, free, T = s["page"], s["tables"].shape[1], s["tables"], s["free"], s["tokens"]
    held, lengths = s["held"].long(), s["lengths"].long()
    had, have = ((n + page - 1).div(page, rounding_mode="floor").clamp(max=width) for n in (held, lengths))
    need = (have - had).clamp(min=0)
    base = s["cursor"].long() + need.cumsum(0) - need
    column = torch.arange(width, device=DEVICE)
    index = base[:, None] + column - had[:, None]
    page_of = torch.where(index < free.numel(), free[index.clamp(0, free.numel() - 1)], -1)
    fresh = (column >= had[:, None]) & (column < have[:, None])
    torch.where(fresh, page_of, tables, out=tables)
    new = (lengths - held).clamp(min=0)
    ends, token = new.cumsum(0), torch.arange(T, device=DEVICE)
    request = torch.searchsorted(ends, token, right=True).clamp(max=held.numel() - 1)
    position = held[request] + token - (ends - new)[request]
    at = tables[request, (position // page).clamp(max=width - 1)].long()
    real = (token < ends[-1]) & (position // page < width) & (at >= 0)
    s["after"].copy_(s["cursor"] + need.sum())
    return {"tables": tables, "slots": torch.where(real, at * page + position % page, -1), "cursor": s["after"]}


def _append(s):
    page = s["k"].shape[2]
    at = (s["slots"] // page, slice(None), s["slots"] % page)
    for name, new in (("k", s["key"]), ("v", s["value"])):
        if name + "_scales" in s:
            elements, scales = _quantised(new)
            s[name].view(torch.uint8)[at] = elements.view(torch.uint8)
            s[name + "_scales"].view(torch.uint8)[at] = scales.view(torch.uint8)
        else:
            s[name][at] = new
    return {name: s[name] for name in ("k", "v", "k_scales", "v_scales") if name in s}


def _gathered(s, name, tables):
    """[B, kv_heads, tokens, head_dim] in 32 bits, the tokens of each request in order."""
    x = s[name].view(torch.uint8)[tables].view(F8) if name + "_scales" in s else s[name][tables]  # [B, pages, kv_heads, page, head_dim]
    x = _values(x, s[name + "_scales"].view(torch.uint8)[tables].view(E8)) if name + "_scales" in s else x.float()
    return x.transpose(1, 2).flatten(2, 3)


def _attention(s):
    B, heads, dim = s["q"].shape
    tables = s["tables"].clamp(min=0)
    k = _gathered(s, "k", tables)
    q = s["q"].float().view(B, k.shape[1], -1, dim)
    scores = q @ k.transpose(-1, -2) * s["scale"]
    del k
    there = torch.arange(scores.shape[-1], device=DEVICE) < s["lengths"][:, None, None, None]
    scores = torch.where(there, scores, -1e30)
    p = torch.where(there, torch.exp(scores - scores.amax(-1, keepdim=True)), 0.0)
    del scores
    total = p.sum(-1, keepdim=True)
    out = (p @ _gathered(s, "v", tables)) / torch.where(total > 0, total, 1.0)
    return out.view(B, heads, dim).bfloat16()


def _norm(s):
    total = s["x"].float()
    if s["residual"] is not None:
        total = total + s["residual"].float()
    y = total * torch.rsqrt(total.square().mean(-1, keepdim=True) + s["eps"]) * s["weight"].float()
    got = {} if s["residual"] is None else {"residual": total.bfloat16()}
    if s["format"] == "bf16":
        return dict(got, out=y.bfloat16())
    elements, scales = _quantised(y)
    return dict(got, out=elements, scales=scales)


def run(state):
    s, kind = state, state["kind"]
    if not own:
        return {"tables": _tables, "append": _append, "attention": _attention, "norm": _norm}[kind](s)
    from paper_2605_19561_amd import binding as tq
    if kind == "tables":
        slots, cursor = tq.torq_block_tables(s["held"], s["lengths"], s["free"], s["cursor"], s["tables"], s["page"], s["tokens"], cursor_out=s["after"])
        return {"tables": s["tables"], "slots": slots, "cursor": cursor}
    if kind == "append":
        tq.torq_cache_append(s["cache"], s["key"], s["value"], s["slots"])
        return {name: s[name] for name in ("k", "v", "k_scales", "v_scales") if name in s}
    if kind == "attention":
        return tq.torq_paged_attention(s["q"], s["cache"], s["tables"], s["lengths"], s["scale"])
    form = tq.TORQ_FMT_BF16 if s["format"] == "bf16" else tq.TORQ_FMT_MXFP8
    out, scales, residual = tq.torq_add_rms_norm(s["x"], s["residual"], s["weight"], s["eps"], form)
    return {name: t for name, t in (("residual", residual), ("out", out), ("scales", scales)) if t is not None}


def work(case):
    kind = case["kind"]
    per = 2.0 if case.get("format") == "bf16" else 33 / 32
    if kind == "tables":
        held, lengths = _requests(case)
        page, B = case["page"], case["B"]
        tokens, taken = sum(n - m for m, n in zip(held, lengths)), sum(-(-n // page) + -m // page for m, n in zip(held, lengths))
        return {"bytes": 8 * B + 8 * taken + 8 * tokens + 4 * min(tokens, B) + 8, "flops": 0}
    if kind == "append":
        values = 2 * case["T"] * case["heads"] * case["head_dim"]
        return {"bytes": values * (2 + per) + 8 * case["T"], "flops": 0}
    if kind == "attention":
        tokens, rows = sum(_requests(case)[1]), case["B"] * case["heads"] * case["head_dim"]
        return {"bytes": 2 * per * tokens * case["kv_heads"] * case["head_dim"] + 4 * rows + 4 * tokens / case["page"] + 4 * case["B"],
                "flops": 4.0 * tokens * case["heads"] * case["head_dim"]}
    values = case["M"] * case["d"]
    return {"bytes": values * (2 + per + (4 if case["residual"] else 0)) + 2 * case["d"], "flops": 4.0 * values}


def _exact_blocks(x):
    """In 64 bits: scales, and the elements before they are rounded."""
    blocks = x.unflatten(-1, (-1, 32))
    scale = torch.exp2(torch.ceil(torch.log2((blocks.abs().amax(-1) / 448).clamp(min=2.0 ** -127))))
    return (blocks / scale.unsqueeze(-1)).flatten(-2), scale


def exact(case, seed):
    kind = case["kind"]
    if kind == "tables":
        return None  # whole numbers
    s = prepare(case, seed)
    if kind == "append":
        got, page = {}, case["page"]
        for name, new in (("k", s["key"]), ("v", s["value"])):
            if case["format"] == "bf16":
                got[name] = s[name].double()
                got[name][s["slots"] // page, :, s["slots"] % page] = new.double()
                continue
            elements, scales = _exact_blocks(new.double())
            cache, cache_scales = s[name].double(), s[name + "_scales"].double()
            cache[s["slots"] // page, :, s["slots"] % page] = elements
            cache_scales[s["slots"] // page, :, s["slots"] % page] = scales
            got[name], got[name + "_scales"] = cache, cache_scales
        return got
    if kind == "norm":
        total = s["x"].double() + (0 if s["residual"] is None else s["residual"].double())
        y = total / (total.pow(2).mean(-1, keepdim=True) + s["eps"]).sqrt() * s["weight"].double()
        got = {} if s["residual"] is None else {"residual": total}
        if case["format"] == "bf16":
            return dict(got, out=y)
        elements, scales = _exact_blocks(y)
        return dict(got, out=elements, scales=scales)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    group = case["heads"] // case["kv_heads"]
    for b, n in enumerate(_requests(case)[1]):
        if not n:
            continue
        pages = s["tables"][b, : -(-n // case["page"])].long()
        token = torch.arange(n, device=DEVICE)
        for h in range(case["kv_heads"]):
            k, v = (s[x].view(torch.uint8)[pages, h].view(F8).double() * s[x + "_scales"].view(torch.uint8)[pages, h].view(E8).double().repeat_interleave(32, -1)
                    if case["format"] == "mxfp8" else s[x][pages, h].double() for x in ("k", "v"))
            k, v = (x[token // case["page"], token % case["page"]] for x in (k, v))
            weights = torch.softmax(s["q"][b, h * group : (h + 1) * group].double() @ k.T * s["scale"], -1)
            out[b, h * group : (h + 1) * group] = weights @ v
    return out
