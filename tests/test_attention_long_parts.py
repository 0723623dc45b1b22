"""Attention whose workgroups go through so many keys that the places of their pages, worked out for 32 steps at a time, are worked out three times and
more: prompts over keys in one part, 128 rows to a workgroup and 64, and single tokens in long runs.  Requests share pages, in orders of their own, and
every row's query points to a key of its own, so that nearly all of its weight lies where one page is."""
import math

import pytest
import torch

from paper_2605_19561_amd import binding
from test_chunk_attention import BF, DEV, E2M1, Rule, check, few, tq   # noqa: F401

gpu = pytest.mark.gpu
PAGE = 16


def values(cache, name):
    """[pages, heads, page_size, head_dim] float64 on the GPU."""
    t = getattr(cache, name)
    if cache.format == binding.TORQ_FMT_BF16:
        return t.double()
    byte = getattr(cache, name + "_scales").view(torch.uint8)
    scale = torch.where(byte == 255, math.nan, 2.0 ** (byte.double() - 127)).repeat_interleave(32, -1)
    if cache.format == binding.TORQ_FMT_MXFP8:
        return t.double() * scale
    codes = torch.stack([t & 15, t >> 4], -1).flatten(-2).long()
    return torch.tensor([*E2M1, *-E2M1], dtype=torch.float64, device=DEV)[codes] * scale


def batch(tq, heads, kv_heads, dim, fmt, fresh, lengths, seed):
    """Cache, q, starts, tables, lengths and the key that each (row, head) points to."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    width = -(-max(lengths) // PAGE)
    cache = tq.KVCache.empty(width + 1, kv_heads, PAGE, dim, getattr(tq, "TORQ_FMT_" + fmt.upper()), device=DEV)
    x = torch.randn(((width + 1) * PAGE, 2, kv_heads, dim), generator=g, device=DEV).to(BF)
    tq.torq_cache_append(cache, x[:, 0], x[:, 1], torch.arange(len(x), device=DEV))
    order = torch.randperm(width + 1, generator=g, device=DEV)
    tables = torch.stack([order.roll(37 * b)[:width] for b in range(len(lengths))]).int()
    starts = [0]
    for n in fresh:
        starts.append(starts[-1] + n)
    k = values(cache, "k")
    q = torch.empty((starts[-1], heads, dim), dtype=BF, device=DEV)
    each = heads // kv_heads
    for b, n in enumerate(lengths):
        rows = torch.arange(fresh[b] * heads, device=DEV)
        # all over the keys, in the rows' order turned by the request, those of the last rows' windows among them
        t = ((rows * 0.61803398875 + 0.1 * b) % 1.0 * n).long().view(fresh[b], heads)
        where = tables[b].long()[t // PAGE]
        head = (torch.arange(heads, device=DEV) // each).expand(fresh[b], heads)
        q[starts[b]:starts[b + 1]] = (20 / math.sqrt(dim) * k[where, head, t % PAGE]).to(BF)
    return cache, q, torch.tensor(starts, dtype=torch.int32, device=DEV), tables, torch.tensor(lengths, dtype=torch.int32, device=DEV)


def compare(got, cache, q, starts, tables, lengths, rule, requests, two_parts):
    """Rows of these requests against float64, not-finite values and absent pages (-1) among the keys."""
    heads, dim, each = q.shape[1], q.shape[2], q.shape[1] // cache.heads
    k, v, scale = values(cache, "k"), values(cache, "v"), dim ** -0.5
    for b in requests:
        rows, n = slice(int(starts[b]), int(starts[b + 1])), int(lengths[b])
        count = rows.stop - rows.start
        p, t = (n - count + torch.arange(count, device=DEV)).repeat_interleave(each), torch.arange(n, device=DEV)
        t = t[tables[b].long()[t // PAGE] >= 0]
        where = tables[b].long()[t // PAGE]
        seen = t[None] <= p[:, None]
        if rule.window:
            seen &= t[None] > p[:, None] - rule.window
        if rule.prefix is not None:
            seen |= t[None] < int(rule.prefix[b])
        for h in range(cache.heads):
            kk, vv = k[where, h, t % PAGE], v[where, h, t % PAGE]
            mine = q[rows, h * each:(h + 1) * each].double().reshape(-1, dim)
            s = mine @ torch.nan_to_num(kk).T.contiguous() * scale
            if rule.cap:
                s = rule.cap * torch.tanh(s / rule.cap)
            if rule.slopes is not None:
                s = s - rule.slopes.to(DEV).double()[h * each:(h + 1) * each].repeat(count)[:, None] * (p[:, None] - t[None]).abs()
            e = torch.softmax(torch.where(seen, s, -math.inf), -1)
            e = torch.where(seen.any(-1, keepdim=True), e, 0.0)
            clean = torch.nan_to_num(vv)
            bad = (seen.double() @ torch.isnan(vv).double() > 0) | (seen.double() @ torch.isnan(kk).any(-1, keepdim=True).double() > 0)
            want, weight = e @ clean, e @ clean.abs()
            here = got[rows, h * each:(h + 1) * each].reshape(-1, dim)
            assert torch.equal(torch.isnan(here), bad), (b, h)
            check(torch.where(bad, 0.0, here.double()).cpu(), torch.where(bad, 0.0, want).cpu(), weight.cpu(), two_parts)


def harmed(cache, tables, lengths, rule, fresh):
    """Absent pages in every window of 32 steps, at their ends too, and (where some rows do not see them) NaN values and keys."""
    keys = [t for t in range(0, int(lengths.max()), 1024)]
    for b in range(len(lengths)):
        for t in keys:
            for entry in ((t - 1) // PAGE, t // PAGE, (t + 1024 // 2) // PAGE):
                if 0 <= entry < tables.shape[1] and (entry + b) % 2:
                    tables[b, entry] = -1
    if rule.window:
        # (pages are shared: a key here is one somewhere else for the other requests, which see it or not)
        for b, n in enumerate(lengths.tolist()[:3]):
            low = n - fresh[b] - rule.window + 1        # the first key that the first row sees
            for t, name in ((low + fresh[b] // 2, "v"), (low - 1, "v"), (int(rule.prefix[b]), "v"), (low + 1, "k")):
                page = int(tables[b, t // PAGE])
                if page < 0 or (name == "k" and b):
                    continue
                if cache.format == binding.TORQ_FMT_BF16:
                    getattr(cache, name)[page, :, t % PAGE, 3] = math.nan
                else:
                    getattr(cache, name + "_scales").view(torch.uint8)[page, :, t % PAGE, 0] = 0xFF


def rule_of(name, heads, lengths):
    B = len(lengths)
    # (the window's and the prefix's ends lie within steps, and what lies between is left out across windows of steps)
    prefix = torch.tensor([max(1, int(n * 0.4) + 7 * b) if n > 100 else b % 5 for b, n in enumerate(lengths)], dtype=torch.int32)
    return {"plain": Rule(), "absent": Rule(), "slopes": Rule(slopes=2e-4 * torch.arange(1, heads + 1) / heads), "cap": Rule(cap=40.0),
            "first and last": Rule(window=int(max(lengths) * 0.35), prefix=prefix), "harmed": Rule(window=int(max(lengths) * 0.35), prefix=prefix)}[name]


def long_and_short(long, others, new):
    """Requests of these lengths with `new` new tokens each, and others of some tokens with one."""
    return [new] * len(long) + [1] * others, list(long) + [1 + 5 * i for i in range(others)]


CHUNKS = [
    # heads, kv_heads, head_dim, new tokens, lengths, requests of few tokens: keys in one part
    (16, 16, 128, 66, (3071, 3072, 3073, 3105, 4161), 27),      # 128 rows: four waves with the same 32 steps, 1024 keys
    (32, 16, 64, 66, (2049, 3103, 3136, 4130), 60),
    (16, 16, 96, 66, (3071, 3105, 4161), 29),
    (16, 16, 128, 40, (6143, 6144, 6145, 6209, 8257), 11),      # 64: two for each half of the keys
    (32, 16, 64, 20, (6143, 6209, 8257), 13),
    (16, 16, 256, 66, (3071, 3073, 3105, 4161), 12),
    (16, 16, 192, 40, (3072, 4161), 14),
]


@gpu
@pytest.mark.parametrize("rule", ["plain", "absent", "slopes", "cap", "first and last", "harmed"])
@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("heads,kv_heads,dim,new,long,others", CHUNKS)
def test_prompts_over_many_keys_in_one_part(tq, heads, kv_heads, dim, new, long, others, fmt, rule):
    fresh, lengths = long_and_short(long, others, new)
    cache, q, starts, tables, lens = batch(tq, heads, kv_heads, dim, fmt, fresh, lengths, 61)
    scores = rule_of(rule, heads, lengths)
    if rule in ("absent", "harmed"):
        harmed(cache, tables, lens, scores, fresh)
    assert tq.torq_chunk_attention_workspace_bytes(cache, heads, len(q), new, len(lengths), tables.shape[1]) == 0        # (one part, nothing to join)
    assert not few(heads, kv_heads, new)
    got = tq.torq_chunk_attention(q, starts, cache, tables, lens, dim ** -0.5, most=new, scores=scores.on(tq))
    compare(got, cache, q, starts, tables, lens, scores, range(len(long) + 2), False)


RUNS = [
    # heads, kv_heads, head_dim, requests, longest, new tokens
    (16, 16, 128, 32, 9700, 1), (64, 16, 128, 32, 9700, 1), (16, 16, 64, 48, 9700, 1), (16, 8, 256, 32, 9700, 1),
    (384, 16, 128, 32, 9700, 1),                                # two products side by side
    (16, 16, 128, 48, 7000, 1), (32, 16, 64, 64, 7000, 1),      # a column for each wave: 33 tiles instead of 132
    (16, 16, 96, 32, 9700, 3), (32, 16, 128, 32, 9700, 4), (64, 16, 64, 48, 9700, 7),
]


@gpu
@pytest.mark.parametrize("rule", ["plain", "absent", "slopes", "cap", "first and last", "harmed"])
@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("heads,kv_heads,dim,B,longest,new", RUNS)
def test_single_tokens_in_long_runs(tq, heads, kv_heads, dim, B, longest, new, fmt, rule):
    fresh, lengths = [new] * B, [longest - 173 * (b % 7) - b for b in range(B)]
    cache, q, starts, tables, lens = batch(tq, heads, kv_heads, dim, fmt, fresh, lengths, 62)
    scores = rule_of(rule, heads, lengths)
    if rule in ("absent", "harmed"):
        harmed(cache, tables, lens, scores, fresh)
    assert few(heads, kv_heads, new)
    if new > 1:
        got = tq.torq_chunk_attention(q, starts, cache, tables, lens, dim ** -0.5, most=new, scores=scores.on(tq))
    else:
        got = tq.torq_paged_attention(q, cache, tables, lens, dim ** -0.5, scores=scores.on(tq))
    compare(got, cache, q, starts, tables, lens, scores, range(0, B, 6), True)
