"""A key-value cache in four bits, attention over it, and attention of prompts, with the scores that models give their tokens.

Three kinds of work, at the sizes of the models that the benchmark takes its linear layers from (LLaMA3-8B: 32 query and 8 key heads
of 128; LLaMA3-70B and Qwen3-32B: 64 and 8 of 128) and at generic ones:

  append     `torq_cache_append` to a cache in MXFP4: a step's keys and values, rounded to four bits, to their slots
  attention  `torq_paged_attention`: one new token of each request over a cache in MXFP4, or over one in any format with scores that
             are capped, fall with the distance, or are taken of the last tokens (and the first few) only
  chunk      `torq_chunk_attention`: prompts, pieces of prompts and drafts, several new tokens of each request, over a cache in any format

The scores: s = scale q . k;  cap: s = cap tanh(s / cap);  slopes: s -= slope |p - t| for a query at position p and a key at t;  a query
sees the keys t <= p, with a window only those t > p - window, and the first `prefix` tokens of its request whatever its position.

Each is computed in elementary torch operations in 32 bits where `own` is false, and by the framework's call where it is true.
MXFP8 caches are torch's float8_e4m3fn elements with float8_e8m0fnu scales, one for 32 elements; MXFP4 ones are bytes of two E2M1 codes, the
first in the low half, with scales of the same kind.  What an append leaves in such a cache is returned as the elements' values (in
float8_e4m3fn, which holds all of E2M1's) and the scales.
"""
import math

import torch

own = False
DEVICE = "cuda:0"
F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
MOST_BYTES, MOST_FLOPS = 0.9e9, 2.9e10        # of a drawn attention
MOST_CHUNK_FLOPS, MOST_PAIRS, MOST_GATHERED = 5.4e11, 2.1e9, 4e9  # of a drawn chunk: its work, and what the plain form makes of it
MOST_APPEND = 8192 * 8 * 128


def listed():
    plain = {"cap": 0.0, "slopes": False, "window": 0, "prefix": 0}
    return [
        # a decode step of sixteen sequences: their new keys and values (LLaMA3-8B or 70B) to their slots, in four bits
        {"name": "append4_decode_16", "kind": "append", "T": 16, "heads": 8, "head_dim": 128, "page": 16, "layout": "heads"},
        # prefill of 8192 tokens, keys and values being columns of one projection's output
        {"name": "append4_prefill", "kind": "append", "T": 8192, "heads": 8, "head_dim": 128, "page": 64, "layout": "heads"},
        # one sequence early in its answer (LLaMA3-8B): latency counts
        {"name": "attention4_1_short", "kind": "attention", "B": 1, "heads": 32, "kv_heads": 8, "head_dim": 128, "page": 16,
         "low": 333, "high": 333, "empty": 0, "format": "mxfp4", "layout": "heads", **plain},
        # a batch of 45 (Qwen3-32B) with long contexts: the largest decode step
        {"name": "attention4_45", "kind": "attention", "B": 45, "heads": 64, "kv_heads": 8, "head_dim": 128, "page": 32,
         "low": 8000, "high": 32768, "empty": 0, "format": "mxfp4", "layout": "heads", **plain},
        # sixteen sequences of ragged length (LLaMA3-70B's heads), capped scores of the last 4096 tokens and the first 16
        {"name": "attention_16_capped", "kind": "attention", "B": 16, "heads": 64, "kv_heads": 8, "head_dim": 128, "page": 16,
         "low": 1000, "high": 16384, "empty": 0, "format": "bf16", "layout": "heads", "cap": 30.0, "slopes": False, "window": 4096, "prefix": 16},
        # a captured batch of 77 places, ten of them idle, a key head for each query head, scores that fall with the distance, tokens outermost in a page
        {"name": "attention4_77_slopes", "kind": "attention", "B": 77, "heads": 20, "kv_heads": 20, "head_dim": 96, "page": 48,
         "low": 1, "high": 4096, "empty": 10, "format": "mxfp4", "layout": "tokens", "cap": 0.0, "slopes": True, "window": 0, "prefix": 0},
        # a short prompt (LLaMA3-8B): latency counts
        {"name": "chunk_37", "kind": "chunk", "B": 1, "heads": 32, "kv_heads": 8, "head_dim": 128, "page": 16, "new_low": 37, "new_high": 37,
         "past_low": 0, "past_high": 0, "empty": 0, "format": "bf16", "layout": "heads", **plain},
        # a prompt of 8192 tokens (LLaMA3-8B)
        {"name": "chunk_prompt", "kind": "chunk", "B": 1, "heads": 32, "kv_heads": 8, "head_dim": 128, "page": 64, "new_low": 8192, "new_high": 8192,
         "past_low": 0, "past_high": 0, "empty": 0, "format": "bf16", "layout": "heads", **plain},
        # 61 prompts of ragged length, capped scores of the last 512 tokens, in an 8-bit cache
        {"name": "chunk_61_capped", "kind": "chunk", "B": 61, "heads": 32, "kv_heads": 8, "head_dim": 128, "page": 16, "new_low": 1, "new_high": 1024,
         "past_low": 0, "past_high": 0, "empty": 0, "format": "mxfp8", "layout": "heads", "cap": 30.0, "slopes": False, "window": 512, "prefix": 0},
        # a piece of 512 tokens of a long prompt (LLaMA3-70B), 60000 tokens into a 4-bit cache: the most work
        {"name": "chunk4_512_late", "kind": "chunk", "B": 1, "heads": 64, "kv_heads": 8, "head_dim": 128, "page": 64, "new_low": 512, "new_high": 512,
         "past_low": 60000, "past_high": 60000, "empty": 0, "format": "mxfp4", "layout": "heads", **plain},
        # drafts of five tokens to be checked for 32 sequences (LLaMA3-70B's heads), two places idle
        {"name": "chunk4_32_drafts", "kind": "chunk", "B": 32, "heads": 64, "kv_heads": 8, "head_dim": 128, "page": 16, "new_low": 5, "new_high": 5,
         "past_low": 1000, "past_high": 8000, "empty": 2, "format": "mxfp4", "layout": "heads", **plain},
        # seven prompts whose first 100 tokens see one another, scores that fall with the distance, odd head and page sizes
        {"name": "chunk_7_prefix", "kind": "chunk", "B": 7, "heads": 20, "kv_heads": 20, "head_dim": 80, "page": 48, "new_low": 150, "new_high": 1500,
         "past_low": 0, "past_high": 300, "empty": 0, "format": "bf16", "layout": "tokens", "cap": 0.0, "slopes": True, "window": 0, "prefix": 100},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _rule(rng, most):
    """How a drawn case gives its scores."""
    return {"cap": rng.choice([0.0, 0.0, 20.0, 50.0]), "slopes": rng.random() < 0.3,
            "window": _log(rng, 1, max(1, most)) if rng.random() < 0.4 else 0, "prefix": _log(rng, 1, max(1, most)) if rng.random() < 0.3 else 0}


def draw(rng):
    kind = rng.choice(["append", "attention", "attention", "attention", "chunk", "chunk", "chunk", "chunk"])
    form = "mxfp4" if kind == "append" else rng.choice(["mxfp4", "mxfp4", "bf16", "mxfp8"])
    page = 16 * _log(rng, 1, 8)
    dims = [64, 72, 80, 96, 112, 128, 128, 128, 192, 256] if form == "bf16" else [32, 64, 96, 128, 128, 192, 256]
    layout = rng.choice(["heads", "heads", "tokens"])
    if kind == "append":
        heads, dim = rng.choice([1, 2, 4, 8, 8, 20]), rng.choice(dims)
        T = _log(rng, 1, max(1, MOST_APPEND // heads // dim))
        return {"kind": kind, "T": T, "heads": heads, "head_dim": dim, "page": page, "layout": layout}
    kv = rng.choice([1, 2, 4, 8, 8, 8, 20])
    group = rng.choice([1, 2, 4, 5, 7, 8, 8, 12, 16])
    dim = rng.choice(dims)
    if kind == "attention":
        B = _log(rng, 1, 256)
        high = _log(rng, 1, 131072)
        case = {"kind": kind, "B": B, "heads": kv * group, "kv_heads": kv, "head_dim": dim, "page": page,
                "low": max(1, int(high * rng.random())), "high": high, "empty": rng.choice([0, 0, B // 8]), "format": form, "layout": layout}
        case.update(_rule(rng, high))
        if form != "mxfp4" and not (case["cap"] or case["slopes"] or case["window"] or case["prefix"]):
            case["cap"] = 30.0
        whole = lambda: work(dict(case, window=0))
        while case["high"] > 1 and (whole()["bytes"] > MOST_BYTES or whole()["flops"] > MOST_FLOPS):
            case.update(low=max(1, case["low"] // 2), high=case["high"] // 2)
        return case
    B, new = _log(rng, 1, 64), _log(rng, 1, 8192)
    past = rng.choice([0, _log(rng, 1, 65536)])
    case = {"kind": kind, "B": B, "heads": kv * group, "kv_heads": kv, "head_dim": dim, "page": page, "new_low": rng.randint(1, new), "new_high": new,
            "past_low": rng.randint(0, past), "past_high": past, "empty": rng.choice([0, 0, B // 8]), "format": form, "layout": layout}
    case.update(_rule(rng, new + past))
    def too_much():
        rows, keys = case["B"] * case["heads"] * case["new_high"], case["new_high"] + case["past_high"]
        return rows * keys > MOST_PAIRS or case["B"] * kv * keys * dim > MOST_GATHERED or work(dict(case, window=0))["flops"] > MOST_CHUNK_FLOPS
    while case["new_high"] + case["past_high"] > 1 and too_much():
        if case["past_high"] > 4 * case["new_high"]:
            case.update(past_low=case["past_low"] // 2, past_high=case["past_high"] // 2)
        else:
            case.update(new_low=max(1, case["new_low"] // 2), new_high=max(1, case["new_high"] // 2), past_low=case["past_low"] // 2, past_high=case["past_high"] // 2)
    return case


def _spread(n, low, high, phase=0.5):
    """n whole numbers over [low, high] in no order, the same for every seed: what a pass has to read goes by them."""
    return [low + int((high - low + 1) * ((phase + 0.6180339887498949 * (i + 1)) % 1.0)) for i in range(n)]


def _requests(case):
    """New tokens of each request, and its tokens after the step."""
    B = case["B"]
    if case["kind"] == "attention":
        lengths, new = _spread(B, case["low"], case["high"]), [1] * B
    else:
        new = _spread(B, case["new_low"], case["new_high"])
        lengths = [n + p for n, p in zip(new, _spread(B, case["past_low"], case["past_high"], 0.25))]
    for i in range(case["empty"]):
        new[(7 * i + 3) % B], lengths[(7 * i + 3) % B] = 0, 0
    return new, lengths


def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _round8(x):
    """MXFP8 of the last dimension's blocks of 32: elements, and the bytes of the scales, the least powers of two that leave no element above 448."""
    blocks = x.float().unflatten(-1, (-1, 32))
    mantissa, exponent = torch.frexp(blocks.abs().amax(-1))  # amax = mantissa 2^exponent, mantissa in [0.5, 1); 448 = 0.875 2^9
    byte = (exponent - 9 + (mantissa > 0.875) + 127).clamp(0, 254)
    return torch.ldexp(blocks, 127 - byte.unsqueeze(-1)).flatten(-2).to(F8).view(torch.uint8), byte.to(torch.uint8)


def _round4(x):
    """MXFP4 of the same blocks: codes, two to a byte, and scales 2^(floor(log2 amax) - 2).  Nearest E2M1 value, ties to the even code, at most 6."""
    blocks = x.float().unflatten(-1, (-1, 32))
    amax = blocks.abs().amax(-1)
    exponent = torch.frexp(amax)[1] - 1                      # floor(log2 amax)
    byte = torch.where(amax > 0, exponent - 2 + 127, 0).clamp(0, 254)
    z = torch.ldexp(blocks, 127 - byte.unsqueeze(-1)).flatten(-2)
    a = z.abs()
    # the number of borders below: a border itself goes to the even code, so it is passed by those above even codes only beyond it
    code = (a > 0.25).byte() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    code = code + 8 * torch.signbit(x).byte()
    return code[..., ::2] + 16 * code[..., 1::2], byte.to(torch.uint8)


def _pairs(dtype):
    """The two values of each byte of codes."""
    one = torch.tensor(E2M1 + [-x for x in E2M1], device=DEVICE)
    byte = torch.arange(256, device=DEVICE)
    return torch.stack([one[byte % 16], one[byte // 16]], -1).to(dtype)


def _elements4(codes):
    """Bytes of codes as float8_e4m3fn, two to a byte."""
    table = _pairs(F8).view(torch.uint8).view(torch.int16).flatten()
    return torch.index_select(table, 0, codes.flatten().int()).view(torch.uint8).view(*codes.shape[:-1], -1).view(F8)


def _blank(pages, case, dtype, last):
    """An uninitialised [pages, heads, page, last], in memory in that order or with a page's tokens ahead of its heads."""
    heads = case.get("kv_heads", case["heads"])
    if case["layout"] == "heads":
        return torch.empty((pages, heads, case["page"], last), dtype=dtype, device=DEVICE)
    return torch.empty((pages, case["page"], heads, last), dtype=dtype, device=DEVICE).transpose(1, 2)


def _filled(state, name, pages, case, seed, outliers):
    """A cache of normal values, a few channels of them larger (keys have such), in its format, made in pieces."""
    dim, form = case["head_dim"], case["format"]
    g, channel = _gen(seed), torch.ones(dim, device=DEVICE)
    if outliers:
        channel[:: max(1, dim // outliers)] = 3.0
    per = {"bf16": 1, "mxfp8": 1, "mxfp4": 2}[form]
    cache = _blank(pages, case, torch.bfloat16 if form == "bf16" else torch.uint8, dim // per)
    scales = None if form == "bf16" else _blank(pages, case, torch.uint8, dim // 32)
    step = max(1, (1 << 26) // (cache[0].numel() * per))
    for i in range(0, pages, step):
        part = cache[i : i + step]
        x = torch.randn((*part.shape[:3], dim), generator=g, device=DEVICE) * channel
        if form == "bf16":
            part.copy_(x)
        else:
            elements, e = (_round8 if form == "mxfp8" else _round4)(x)
            part.copy_(elements)
            scales[i : i + step].copy_(e)
    state[name] = cache.view(F8) if form == "mxfp8" else cache
    if scales is not None:
        state[name + "_scales"] = scales.view(E8)


def _prepare_attention(case, seed):
    B, heads, kv, dim, page = case["B"], case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    new, lengths = _requests(case)
    need = [-(-n // page) for n in lengths]
    pages, width = sum(need) + 3, max(max(need), 1) + 1
    order, tables, at = torch.randperm(pages, generator=_gen(seed), device=DEVICE).tolist(), [], 0
    for n in need:
        tables.append(order[at : at + n] + [-1] * (width - n))
        at += n
    T = B if case["kind"] == "attention" else sum(new)
    # columns of a projection's output; larger where scores are capped, so that some come near the cap
    qkv = torch.randn((T, heads + 2 * kv, dim), generator=_gen(seed + 1), device=DEVICE) * (4.0 if case["cap"] else 1.0)
    state = {"tables": _ints(tables), "lengths": _ints(lengths), "q": qkv.bfloat16()[:, :heads], "scale": dim ** -0.5, "cap": case["cap"],
             "window": case["window"], "slopes": None, "prefix": None}
    if case["slopes"]:
        state["slopes"] = torch.exp2(-8.0 * torch.arange(1, heads + 1, device=DEVICE) / heads)
    if case["prefix"]:
        state["prefix"] = _ints([case["prefix"]] * B)
    if case["kind"] == "chunk":
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        state.update(starts=_ints(starts), most=max(new))
    _filled(state, "k", pages, case, seed + 2, 4)
    _filled(state, "v", pages, case, seed + 3, 0)
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
        state[name] = _blank(pages, case, torch.uint8, dim // 2).zero_()
        state[name + "_scales"] = _blank(pages, case, torch.uint8, dim // 32).zero_().view(E8)
    return state


def prepare(case, seed):
    seed = 1000 * int(seed)
    state = _prepare_append(case, seed) if case["kind"] == "append" else _prepare_attention(case, seed)
    if own:
        from paper_2605_19561_amd import binding as tq
        state["cache"] = tq.KVCache(state["k"], state["v"], state.get("k_scales"), state.get("v_scales"))
        if case["kind"] != "append":
            state["scores"] = tq.Scores(cap=state["cap"], slopes=state["slopes"], window=state["window"], prefix=state["prefix"])
    return dict(state, kind=case["kind"])


def _held(s):
    return {**{name: _elements4(s[name]) for name in ("k", "v")}, **{name: s[name] for name in ("k_scales", "v_scales")}}


def _append(s):
    page = s["k"].shape[2]
    at = (s["slots"] // page, slice(None), s["slots"] % page)
    k, v = _round4(s["key"]), _round4(s["value"])
    s["k"][at], s["k_scales"].view(torch.uint8)[at] = k
    s["v"][at], s["v_scales"].view(torch.uint8)[at] = v
    return _held(s)


def _gathered(s, name, tables):
    """[B, kv_heads, tokens, head_dim] in 32 bits, the tokens of each request in order."""
    x = s[name]
    x = (x.view(torch.uint8)[tables].view(F8) if x.dtype == F8 else x[tables]).transpose(1, 2).flatten(2, 3)  # [B, pages, kv_heads, page, ...]
    if name + "_scales" not in s:
        return x.float()
    scales = s[name + "_scales"].view(torch.uint8)[tables].view(E8).transpose(1, 2).flatten(2, 3)
    if x.dtype == torch.uint8:
        x = torch.index_select(_pairs(torch.float32), 0, x.flatten().int()).view(*x.shape[:-1], -1)
    return (x.float().unflatten(-1, (-1, 32)) * scales.float().unsqueeze(-1)).flatten(-2)


def _attend(s, q, position):
    """q [B, tokens, heads, head_dim] at positions [B, tokens]: the output, in 32 bits."""
    B, n, heads, dim = q.shape
    tables = s["tables"].clamp(min=0)
    k = _gathered(s, "k", tables)
    kv, keys = k.shape[1], k.shape[2]
    rows = q.float().view(B, n, kv, heads // kv, dim).permute(0, 2, 3, 1, 4).reshape(B, kv, -1, dim)
    x = (rows @ k.transpose(-1, -2)).view(B, heads, n, keys).mul_(s["scale"])
    del k
    if s["cap"]:
        x = x.div_(s["cap"]).tanh_().mul_(s["cap"])
    t = torch.arange(keys, device=DEVICE)
    far = position[:, :, None] - t                             # [B, tokens, keys]
    if s["slopes"] is not None:
        x -= s["slopes"][:, None, None] * far.abs().float()[:, None]
    seen = far >= 0
    if s["window"]:
        seen &= far < s["window"]
    if s["prefix"] is not None:
        seen |= t < s["prefix"][:, None, None]
    seen &= t < s["lengths"][:, None, None]
    x = x.masked_fill_(~seen[:, None], -1e30)
    x = x.sub_(x.amax(-1, keepdim=True)).exp_().masked_fill_(~seen[:, None], 0.0)
    total = x.sum(-1, keepdim=True)
    out = x.view(B, kv, -1, keys) @ _gathered(s, "v", tables)
    out = out.view(B, heads, n, dim) / torch.where(total > 0, total, 1.0)
    return out.transpose(1, 2)


def _attention(s):
    return _attend(s, s["q"][:, None], s["lengths"][:, None].long() - 1)[:, 0].bfloat16()


def _chunk(s):
    starts, T = s["starts"].long(), s["q"].shape[0]
    new = starts.diff()
    i = torch.arange(s["most"], device=DEVICE)
    q = s["q"][(starts[:-1, None] + i).clamp(max=T - 1)]
    out = _attend(s, q, s["lengths"][:, None] - new[:, None] + i)
    token = torch.arange(T, device=DEVICE)
    request = torch.searchsorted(starts[1:], token, right=True)
    return out[request, token - starts[request]].bfloat16()


def run(state):
    s, kind = state, state["kind"]
    if not own:
        return {"append": _append, "attention": _attention, "chunk": _chunk}[kind](s)
    from paper_2605_19561_amd import binding as tq
    if kind == "append":
        tq.torq_cache_append(s["cache"], s["key"], s["value"], s["slots"])
        return _held(s)
    if kind == "attention":
        return tq.torq_paged_attention(s["q"], s["cache"], s["tables"], s["lengths"], s["scale"], scores=s["scores"])
    return tq.torq_chunk_attention(s["q"], s["starts"], s["cache"], s["tables"], s["lengths"], s["scale"], most=s["most"], scores=s["scores"])


def _seen(case):
    """Keys that a request's new tokens see, all of them together, and (new token, key) pairs, over all requests."""
    keys = pairs = 0
    for new, length in zip(*_requests(case)):
        if not new:
            continue
        window, prefix = case["window"] or length, min(case["prefix"], length)
        first = length - new
        keys += length - max(0, max(0, first - window + 1) - prefix)
        for p in range(first, length):
            low = max(0, p - window + 1)
            pairs += p + 1 - low + min(prefix, low) + max(0, prefix - (p + 1))
    return keys, pairs


def work(case):
    if case["kind"] == "append":
        values = 2 * case["T"] * case["heads"] * case["head_dim"]
        return {"bytes": values * (2 + 17 / 32) + 8 * case["T"], "flops": 0}
    per = {"bf16": 2.0, "mxfp8": 33 / 32, "mxfp4": 17 / 32}[case["format"]]
    keys, pairs = _seen(case)
    rows = sum(_requests(case)[0]) * case["heads"] * case["head_dim"]
    return {"bytes": 2 * per * keys * case["kv_heads"] * case["head_dim"] + 4 * rows + 4 * keys / case["page"] + 8 * case["B"],
            "flops": 4.0 * pairs * case["heads"] * case["head_dim"]}


def _exact_values(s, name, pages, head):
    """[tokens, head_dim] in 64 bits of a request's pages under a key head."""
    x = s[name].view(torch.uint8)[pages, head].view(F8) if s[name].dtype == F8 else s[name][pages, head]
    x = x.flatten(0, 1)
    if name + "_scales" not in s:
        return x.double()
    if x.dtype == torch.uint8:
        x = torch.stack([x & 15, x >> 4], -1).flatten(-2).long()
        magnitude = torch.tensor(E2M1, dtype=torch.float64, device=DEVICE)[x & 7]
        x = torch.where(x >= 8, -magnitude, magnitude)
    byte = s[name + "_scales"].view(torch.uint8)[pages, head].flatten(0, 1).double()
    return x.double() * torch.exp2(byte - 127).repeat_interleave(32, -1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "append":
        got, page = {}, case["page"]
        for name, new in (("k", s["key"]), ("v", s["value"])):
            blocks = new.double().unflatten(-1, (-1, 32))
            scale = torch.exp2(torch.floor(torch.log2(blocks.abs().amax(-1).clamp(min=2.0 ** -125))) - 2)
            elements = torch.zeros((*s[name].shape[:-1], case["head_dim"]), dtype=torch.float64, device=DEVICE)
            scales = s[name + "_scales"].double()
            z = (blocks / scale.unsqueeze(-1)).flatten(-2)
            values, code = torch.tensor(E2M1, dtype=torch.float64, device=DEVICE), torch.arange(8, device=DEVICE)
            # the nearest of the eight, of two as near the one with the even code (bf16's values are further apart than 1e-9)
            nearest = ((z.abs().unsqueeze(-1) - values).abs() + 1e-9 * (code % 2)).argmin(-1)
            elements[s["slots"] // page, :, s["slots"] % page] = torch.copysign(values[nearest], z)
            scales[s["slots"] // page, :, s["slots"] % page] = scale
            got[name], got[name + "_scales"] = elements, scales
        return got
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    group, at = case["heads"] // case["kv_heads"], 0
    for b, (new, length) in enumerate(zip(*_requests(case))):
        if case["kind"] == "attention":
            at = b
        if not new:
            continue
        pages = s["tables"][b, : -(-length // case["page"])].long()
        t, p = torch.arange(length, device=DEVICE), torch.arange(length - new, length, device=DEVICE)[:, None]
        hidden = (t > p) | (t <= p - case["window"]) if case["window"] else t > p
        hidden = hidden & (t >= case["prefix"])
        for h in range(case["kv_heads"]):
            k, v = (_exact_values(s, x, pages, h)[:length] for x in ("k", "v"))
            for g in range(h * group, (h + 1) * group):
                x = s["q"][at : at + new, g].double() @ k.T * s["scale"]
                if case["cap"]:
                    x = case["cap"] * torch.tanh(x / case["cap"])
                if case["slopes"]:
                    x = x - s["slopes"][g].double() * (p - t).abs()
                out[at : at + new, g] = torch.softmax(x.masked_fill(hidden, -math.inf), -1) @ v
        at += new
    return out
