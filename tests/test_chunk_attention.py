"""Caches in MXFP4, attention with scores by a rule, and attention of several new tokens of each request on the GPU: torq_cache_append,
torq_paged_attention(scores=...) and torq_chunk_attention against plain implementations in 64 bits (or bit for bit, where values are rounded by
definition)."""
import math
import zlib

import numpy as np
import pytest
import torch

from paper_2605_19561_amd import binding

DEV = "cuda:0"
BF, F8, E8 = torch.bfloat16, torch.float8_e4m3fn, torch.float8_e8m0fnu
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def tq():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    binding.lib()
    return binding


@pytest.fixture(params=["native", "interpreted"])
def either_way(request, monkeypatch):
    """The binding's C++ module, and its own Python in the place of that."""
    if request.param == "interpreted":
        monkeypatch.setattr(binding, "_host", binding._Interpreted)
    return request.param


def rng(*seed):
    return torch.Generator().manual_seed(zlib.crc32(repr(seed).encode()))


# ---- MXFP4 from its definition -----------------------------------------------------------------

def mxfp4(x):
    """float64 [..., n] -> codes [..., n / 2] and scale bytes [..., n / 32], uint8, from the definition in the header."""
    x = np.asarray(x, dtype=np.float64)
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    bad = ~np.isfinite(blocks).all(-1)
    amax = np.abs(np.where(np.isfinite(blocks), blocks, 0.0)).max(-1)
    byte = np.where(amax > 0, np.floor(np.log2(np.maximum(amax, 2.0 ** -140))) - 2 + 127, 0).clip(0, 254)
    z = np.abs(np.where(np.isfinite(blocks), blocks, 0.0)) / 2.0 ** (byte - 127)[..., None]
    distance = np.abs(z[..., None] - E2M1)
    # of two as near the one with the even code
    code = np.where(distance == distance.min(-1, keepdims=True), np.arange(8) % 2 * 8 + np.arange(8), 99).argmin(-1)
    code = np.where(bad[..., None], 0, code + 8 * np.signbit(blocks)).reshape(x.shape)
    return (code[..., ::2] + 16 * code[..., 1::2]).astype(np.uint8), np.where(bad, 255, byte).astype(np.uint8)


def test_the_tests_own_mxfp4_rounds_to_the_nearest_and_ties_to_even():
    x = np.zeros((1, 32))
    x[0, :16] = [4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.26, 0.74, -5.01, 7.9, -0.25, 1.3, -0.0, 6.0]
    codes, scales = mxfp4(x)
    nibbles = np.stack([codes & 15, codes >> 4], -1).reshape(1, 32)[0, :16]
    assert scales.tolist() == [[127]]
    assert nibbles.tolist() == [6, 0, 2, 2, 4, 4, 6, 6, 1, 1, 15, 7, 8, 3, 8, 7]


def values4(codes, scales):
    """float64 values of codes and scale bytes on the CPU."""
    codes = codes.cpu().contiguous().numpy()
    nibbles = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)
    v = np.where(nibbles >= 8, -E2M1[nibbles & 7], E2M1[nibbles & 7])
    byte = scales.contiguous().view(torch.uint8).cpu().numpy().astype(np.float64)
    s = np.where(byte == 255, np.nan, 2.0 ** (byte - 127))
    return torch.from_numpy(v * np.repeat(s, 32, -1))


def values_of(cache, name):
    """[pages, heads, page_size, head_dim] float64 on the CPU."""
    t = getattr(cache, name)
    if cache.format == binding.TORQ_FMT_BF16:
        return t.cpu().double()
    scales = getattr(cache, name + "_scales")
    if cache.format == binding.TORQ_FMT_MXFP4:
        return values4(t, scales)
    s = scales.cpu() if scales.dtype == E8 else scales.cpu().contiguous().view(E8)
    return t.cpu().double() * s.double().repeat_interleave(32, -1)


FORMATS = {"bf16": (BF, 1), "mxfp8": (F8, 1), "mxfp4": (torch.uint8, 2)}


def make_cache(tq, pages, heads, page, dim, fmt, layout, fill=0x33):
    """Filled with bytes that no append writes where it should not."""
    elt, packed = FORMATS[fmt]

    def block(last, dtype):
        if layout == "heads":
            t = torch.empty((2, pages, heads, page, last), dtype=dtype, device=DEV)
        elif layout == "tokens":
            t = torch.empty((2, pages, page, heads, last), dtype=dtype, device=DEV).transpose(-3, -2)
        else:                                        # keys and values of a page side by side
            t = torch.empty((pages, 2, heads, page, last), dtype=dtype, device=DEV).transpose(0, 1)
        t.view(torch.int16 if dtype == BF else torch.uint8).fill_(fill)
        return t
    kv = block(dim // packed, elt)
    if fmt == "bf16":
        return tq.KVCache(kv[0], kv[1])
    sc = block(dim // 32, torch.uint8)
    return tq.KVCache(kv[0], kv[1], sc[0].view(E8), sc[1].view(E8))


def u8(t):
    return t.contiguous().view(torch.uint8).cpu().numpy()


APPEND = [
    # tokens, heads, head_dim, page, layout, packed input
    (1, 1, 32, 16, "heads", False), (33, 8, 128, 16, "tokens", True), (17, 2, 96, 32, "pairs", False), (40, 5, 256, 64, "pairs", True),
    (3000, 4, 64, 16, "heads", True), (700, 20, 160, 112, "heads", False)]


@gpu
@pytest.mark.parametrize("T,heads,dim,page,layout,packed", APPEND)
def test_cache_append_in_four_bits(tq, either_way, T, heads, dim, page, layout, packed):
    pages = -(-T // page) + 3
    g = rng(T, heads, dim)
    x = (torch.randn((T, 2 * heads + 3, dim), generator=g) * torch.exp(4 * torch.randn((T, 2 * heads + 3, 1), generator=g))).to(BF)
    x[:, :, ::7] *= 0.001
    if T > 4:                                        # zeros of both signs, ties, a maximum at the border of a scale, subnormals, the largest
        x[0] = torch.tensor([0.0, -0.0] * (dim // 2), dtype=BF)
        x[1] = torch.tensor([4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -5.0, 6.0, -7.0, 7.96875, 0.2, -0.3] * (dim // 16), dtype=BF)
        x[2, :, 0], x[2, :, 1:] = -7.96875, 1.0
        x[3] = 2.0 ** -130 * torch.tensor([1.0, -3.0, 5.0, 8.0] * (dim // 4), dtype=BF)
        x[4, :, 0], x[4, :, 1:] = torch.finfo(BF).max, -1e30
    x = x.to(DEV)
    key, value = (x[:, 3:3 + heads], x[:, 3 + heads:]) if packed else (x[:, :heads].contiguous(), x[:, heads:2 * heads].contiguous())
    slots = torch.randperm(pages * page, generator=g)[:T]
    if T > 8:
        slots[7], slots[8] = -1, pages * page        # passed over
    cache = make_cache(tq, pages, heads, page, dim, "mxfp4", layout)
    names = ["k", "v", "k_scales", "v_scales"]
    want = {n: u8(getattr(cache, n)).copy() for n in names}
    tq.torq_cache_append(cache, key, value, slots.to(DEV))
    for name, new in (("k", key), ("v", value)):
        for n, rows in zip((name, name + "_scales"), mxfp4(new.cpu().double().numpy())):
            for t, slot in enumerate(slots.tolist()):
                if 0 <= slot < pages * page:
                    want[n][slot // page, :, slot % page] = rows[t].reshape(heads, -1)
    for n in names:
        assert np.array_equal(u8(getattr(cache, n)), want[n]), n


@gpu
def test_cache_append_in_four_bits_marks_blocks_that_are_not_finite(tq):
    x = torch.ones((4, 1, 64), dtype=BF)
    x[0, 0, 5], x[1, 0, 40], x[2, 0, 63] = math.inf, math.nan, -math.inf
    cache = make_cache(tq, 1, 1, 16, 64, "mxfp4", "heads")
    x = x.to(DEV)
    tq.torq_cache_append(cache, x, x, torch.arange(4, device=DEV))
    codes, scales = mxfp4(x.cpu().double().numpy())
    assert np.array_equal(u8(cache.k)[0, 0, :4], codes[:, 0]) and np.array_equal(u8(cache.v_scales)[0, 0, :4], scales[:, 0])
    assert scales[:, 0].tolist() == [[255, 125], [125, 255], [125, 255], [125, 125]]


@gpu
def test_cache_append_in_four_bits_is_the_quantiser(tq):
    x = (torch.randn((300, 4, 128), generator=rng(3)) * torch.exp(3 * torch.randn((300, 4, 1), generator=rng(4)))).to(BF).to(DEV)
    cache = make_cache(tq, 19, 4, 16, 128, "mxfp4", "tokens")
    tq.torq_cache_append(cache, x, x, torch.arange(300, device=DEV))
    codes, scales = tq.torq_quantize_f32(x.float().view(300, 512))
    assert torch.equal(cache.k.transpose(1, 2).reshape(-1, 256)[:300], codes)
    assert torch.equal(cache.v_scales.view(torch.uint8).transpose(1, 2).reshape(-1, 16)[:300], scales)


# ---- attention ---------------------------------------------------------------------------------

class Rule:
    """The scores of a test: what tq.Scores takes, on the CPU."""

    def __init__(self, cap=0.0, slopes=None, window=0, prefix=None):
        self.cap, self.slopes, self.window, self.prefix = cap, slopes, window, prefix

    def on(self, tq):
        return tq.Scores(self.cap, None if self.slopes is None else self.slopes.to(DEV), self.window, None if self.prefix is None else self.prefix.to(DEV))


def seen_by(rule, b, p, t):
    """Which keys at t [n] the queries at p [m] see, [m, n]."""
    seen = t[None] <= p[:, None]
    if rule.window:
        seen &= t[None] > p[:, None] - rule.window
    if rule.prefix is not None:
        seen |= t[None] < int(rule.prefix[b])
    return seen


def reference(q, starts, k, v, tables, lengths, scale, pages, rule):
    """float64: out, and sum_t p_t |v_t|.  k, v [pages, heads, page, dim] float64; rows of no request are NaN."""
    T, heads, dim = q.shape
    page, group = k.shape[2], heads // k.shape[1]
    out, weight = torch.full((T, heads, dim), math.nan, dtype=torch.float64), torch.full((T, heads, dim), math.nan, dtype=torch.float64)
    for b, length in enumerate(lengths.tolist()):
        rows = torch.arange(int(starts[b]), int(starts[b + 1]))
        if not len(rows):
            continue
        p = length - len(rows) + torch.arange(len(rows))
        t = torch.arange(min(max(length, 0), tables.shape[1] * page))
        entry = tables[b].long()[t // page] if len(t) else t
        there = (entry >= 0) & (entry < pages)
        t, entry = t[there], entry[there]
        seen = seen_by(rule, b, p, t)
        for h in range(heads):
            kk, vv = k[entry, h // group, t % page], v[entry, h // group, t % page]
            s = q[rows, h].double() @ kk.T * scale
            if rule.cap:
                s = rule.cap * torch.tanh(s / rule.cap)
            if rule.slopes is not None:
                s = s - rule.slopes[h].double() * (p[:, None] - t[None]).abs()
            s = torch.where(seen, s, -math.inf)
            top = s.amax(-1, keepdim=True) if len(t) else torch.zeros((len(rows), 1), dtype=torch.float64)
            e = torch.where(seen, torch.exp(s - torch.where(top == -math.inf, 0.0, top)), 0.0)
            total = e.sum(-1, keepdim=True)
            e = e / torch.where(total == 0, 1.0, total)
            # what a query does not see takes no part, finite or not
            visible = torch.where(seen[..., None], vv[None], 0.0) if len(t) * len(rows) * dim < 1 << 24 else None
            if visible is not None:
                out[rows, h], weight[rows, h] = (e[..., None] * visible).sum(1), (e[..., None] * visible.abs()).sum(1)
            else:
                out[rows, h], weight[rows, h] = e @ vv, e @ vv.abs()
    return out, weight


def few(heads, kv_heads, most):
    return heads // kv_heads * most <= 32


def check(got, out, weight, two_parts):
    got, there = got.double().cpu(), ~torch.isnan(out)
    if two_parts:
        # the output's rounding, 2^-8 |out| <= 2^-9 (|out| + W), W = sum p |v|; fp32's part (dot products ahead of the exponential, sums) below 2^-12 of that
        bound = (2.0 ** -9 + 2.0 ** -12) * (out.abs() + weight) + 1e-38
    else:
        # weights p (1 + d), |d| <= 2^-8, divided by their own sum: off by sum p d (v - out) / sum p (1 + d), at most 2^-8 (W + |out|) / (1 - 2^-8); the
        # output's rounding 2^-8 |out| of what is then there; second orders and fp32's part below 2^-12 (W + |out|)
        bound = 2.0 ** -8 * (weight + 2 * out.abs()) + 2.0 ** -12 * (weight + out.abs()) + 1e-38
    worst = ((got - out).abs() / bound)[there].max() if there.any() else torch.zeros(())
    assert float(worst) <= 1.0, float(worst)


def case(tq, fresh, lengths, heads, kv_heads, dim, page, fmt, layout, seed, spread=1.0, ones=False, gap=0):
    """A cache whose requests hold `lengths` tokens, the last fresh[b] of them new.  ones: keys 0, values 1 at one place that goes by the token.
    gap: rows of q of no request behind the last."""
    g = rng(fresh, lengths, heads, dim, page, fmt, seed)
    need = [-(-n // page) for n in lengths]
    pages, width = sum(need) + 4, max(need + [1]) + 2
    order, at = torch.randperm(pages, generator=g).int(), 0
    tables = torch.full((len(lengths), width), -1, dtype=torch.int32)
    for b, n in enumerate(need):
        tables[b, :n] = order[at:at + n]
        at += n
    cache = make_cache(tq, pages, kv_heads, page, dim, fmt, layout)
    # what lies behind a length, in the last page or in pages of nobody, is no finite value
    for t in (cache.k, cache.v):
        if fmt == "bf16":
            t.view(torch.int16).fill_(0x7FC0)
        elif fmt == "mxfp8":
            t.view(torch.uint8).fill_(0x7F)
    if fmt == "mxfp4":
        for t in (cache.k_scales, cache.v_scales):
            t.view(torch.uint8).fill_(0xFF)
    T = sum(lengths)
    if ones:
        x = torch.zeros((T, 2, kv_heads, dim))
        token = torch.cat([torch.arange(n) for n in lengths]) if T else torch.zeros(0, dtype=torch.long)
        for h in range(kv_heads):
            x[torch.arange(T), 1, h, (token * 29 + 7 * h) % dim] = 1.0
    else:
        x = torch.randn((T, 2, kv_heads, dim), generator=g)
        x[:, 0, :, ::9] *= 3.0 * spread
    slots = [int(tables[b, p // page]) * page + p % page for b, n in enumerate(lengths) for p in range(n)]
    x = x.to(BF).to(DEV)
    if T:
        tq.torq_cache_append(cache, x[:, 0], x[:, 1], torch.tensor(slots, dtype=torch.int64, device=DEV))
    starts = torch.tensor([0] + np.cumsum(fresh).tolist(), dtype=torch.int32)
    q = (torch.randn((int(starts[-1]) + gap, heads, dim), generator=g) * spread).to(BF)
    return cache, q * 0 if ones else q, starts, tables, torch.tensor(lengths, dtype=torch.int32), pages


def slopes_of(heads):
    return 2.0 ** (-8.0 * torch.arange(1, heads + 1) / heads)


def prefix_of(*n):
    return torch.tensor(n, dtype=torch.int32)


RULES = {
    "plain": lambda heads, B: Rule(),
    "capped": lambda heads, B: Rule(cap=3.0),
    "slopes": lambda heads, B: Rule(slopes=slopes_of(heads)),
    "window 1": lambda heads, B: Rule(window=1),
    "window 50": lambda heads, B: Rule(window=50),
    "window over all": lambda heads, B: Rule(window=2 ** 31 - 1),
    "prefix": lambda heads, B: Rule(prefix=torch.tensor([(37 * b) % 90 - 3 for b in range(B)], dtype=torch.int32)),
    "first and last": lambda heads, B: Rule(window=40, prefix=torch.tensor([(5 * b) % 70 for b in range(B)], dtype=torch.int32)),
    "everything": lambda heads, B: Rule(cap=5.0, slopes=slopes_of(heads), window=64, prefix=torch.full((B,), 33, dtype=torch.int32)),
}

SHAPES = [
    # heads, kv_heads, head_dim, page, lengths, format, layout
    (1, 1, 32, 16, [1, 0, 2], "mxfp4", "heads"),
    (32, 8, 128, 16, [1, 15, 16, 17, 31, 32, 33, 0, 127, 128, 129], "mxfp4", "heads"),
    (64, 8, 128, 32, [2000, 257, 1, 511], "mxfp4", "tokens"),
    (20, 20, 96, 48, [3, 300, 0, 47, 48, 49, 95, 97], "mxfp4", "tokens"),
    (7, 1, 64, 16, [65, 130], "mxfp4", "pairs"),
    (48, 2, 128, 16, [300, 20], "mxfp4", "heads"),
    (64, 2, 64, 16, [5, 520, 0, 77] * 5, "mxfp4", "pairs"),
    (80, 2, 128, 16, [300, 45, 0, 1] * 12, "mxfp4", "heads"),
    (8, 4, 192, 16, [100, 33], "mxfp4", "tokens"),
    (16, 1, 256, 16, [400, 31], "mxfp4", "heads"),
    (8, 8, 256, 16, [40, 31] * 60, "mxfp4", "heads"),
    (8, 1, 128, 16, [33000], "mxfp4", "heads"),
]


@gpu
@pytest.mark.parametrize("heads,kv_heads,dim,page,lengths,fmt,layout", SHAPES)
def test_paged_attention_over_four_bits(tq, either_way, heads, kv_heads, dim, page, lengths, fmt, layout):
    B = len(lengths)
    cache, q, starts, tables, lens, pages = case(tq, [1] * B, lengths, heads, kv_heads, dim, page, fmt, layout, 1)
    want = reference(q, starts, values_of(cache, "k"), values_of(cache, "v"), tables, lens, dim ** -0.5, pages, Rule())
    wide = torch.zeros((B, heads + 2, dim), dtype=BF, device=DEV)
    wide[:, 1:-1] = q.to(DEV)
    got = tq.torq_paged_attention(wide[:, 1:-1], cache, tables.to(DEV), lens.to(DEV), dim ** -0.5)
    check(got, *want, True)


@gpu
@pytest.mark.parametrize("byte", [0, 1, 2, 100, 127, 200, 249, 250, 252, 255])
def test_codes_under_every_scale_as_attention_reads_them(tq, byte):
    """A request of one token: out is its value, exactly (MXFP4 is exact in bf16 but for what is 2^128 and more)."""
    cache = make_cache(tq, 1, 1, 16, 32, "mxfp4", "heads")
    codes = torch.arange(16, dtype=torch.uint8)
    cache.k.view(torch.uint8).zero_()
    cache.k_scales.view(torch.uint8).fill_(127)
    cache.v[0, 0, 0] = (codes[::2] + 16 * codes[1::2]).repeat(2).to(DEV)
    cache.v_scales.view(torch.uint8).fill_(byte)
    q = torch.ones((1, 4, 32), dtype=BF, device=DEV)
    one = torch.ones((1,), dtype=torch.int32, device=DEV)
    got = tq.torq_paged_attention(q, cache, torch.zeros((1, 1), dtype=torch.int32, device=DEV), one, 1.0).cpu()
    values = np.concatenate([E2M1, -E2M1, E2M1, -E2M1]) * 2.0 ** (byte - 127.0)
    want = torch.from_numpy(np.where(np.abs(values) >= 2.0 ** 128, np.copysign(np.inf, values), values)).to(BF)
    if byte == 255:
        assert torch.isnan(got).all()
    else:
        assert torch.equal(got[0, 2], want)


SCORED = [
    # heads, kv_heads, head_dim, page, lengths, format, layout
    (32, 8, 128, 16, [1, 31, 33, 0, 128, 129, 300], "bf16", "heads"),
    (64, 8, 128, 64, [2000, 257, 1, 511], "mxfp8", "tokens"),
    (20, 20, 96, 48, [3, 300, 0, 47, 97], "mxfp4", "tokens"),
    (48, 2, 64, 16, [300, 20, 0] * 12, "bf16", "pairs"),
    (8, 4, 200, 16, [100, 33, 1000], "bf16", "heads"),
    (4, 4, 256, 16, [100, 33, 1000], "mxfp4", "heads"),
    (5, 1, 72, 112, [113, 224, 5000], "bf16", "pairs"),
]


@gpu
@pytest.mark.parametrize("rule", sorted(RULES))
@pytest.mark.parametrize("heads,kv_heads,dim,page,lengths,fmt,layout", SCORED)
def test_paged_attention_by_a_rule(tq, heads, kv_heads, dim, page, lengths, fmt, layout, rule):
    B = len(lengths)
    rule = RULES[rule](heads, B)
    for ones in (False, True):
        cache, q, starts, tables, lens, pages = case(tq, [1] * B, lengths, heads, kv_heads, dim, page, fmt, layout, 2, spread=2.0, ones=ones)
        want = reference(q, starts, values_of(cache, "k"), values_of(cache, "v"), tables, lens, dim ** -0.5, pages, rule)
        got = tq.torq_paged_attention(q.to(DEV), cache, tables.to(DEV), lens.to(DEV), dim ** -0.5, scores=rule.on(tq))
        check(got, *want, True)


CHUNKS = [
    # heads, kv_heads, head_dim, page, new tokens, tokens after the step, format, layout
    (1, 1, 8, 16, [1], [1], "bf16", "heads"),
    (32, 8, 128, 16, [1, 3, 0, 8, 2], [1, 3, 0, 200, 77], "bf16", "heads"),             # few rows
    (64, 8, 128, 16, [4, 1, 4, 0, 3], [500, 33, 4, 60, 1029], "mxfp4", "heads"),
    (8, 1, 64, 32, [2, 4, 1], [40, 4, 700], "mxfp8", "tokens"),
    (4, 4, 256, 16, [7, 16, 30], [7, 300, 31], "mxfp4", "heads"),
    (32, 8, 128, 16, [37], [37], "bf16", "heads"),
    (32, 8, 128, 16, [70, 1, 0, 129, 33], [70, 50, 20, 129, 300], "bf16", "heads"),
    (32, 8, 128, 64, [70, 1, 0, 129, 33], [70, 50, 20, 129, 300], "mxfp8", "tokens"),
    (16, 2, 128, 32, [40, 5, 64, 65], [1000, 5, 64, 66], "mxfp4", "pairs"),
    (20, 20, 80, 48, [150, 31, 1], [400, 31, 49], "bf16", "tokens"),
    (7, 1, 64, 16, [90, 200], [91, 900], "mxfp4", "heads"),
    (5, 5, 32, 16, [130, 64], [130, 100], "mxfp8", "heads"),
    (3, 1, 40, 16, [100, 33], [100, 333], "bf16", "pairs"),
    (8, 4, 192, 16, [60, 17], [100, 17], "mxfp8", "heads"),
    (8, 2, 256, 32, [50, 90], [500, 90], "bf16", "heads"),
    (6, 2, 256, 16, [70, 3], [70, 303], "mxfp4", "tokens"),
    (2, 1, 128, 16, [300] + [1, 0, 2] * 250, [400] + [7, 3, 2] * 250, "bf16", "heads"),   # more than 512 requests
]


@gpu
@pytest.mark.parametrize("rule", sorted(RULES))
@pytest.mark.parametrize("heads,kv_heads,dim,page,fresh,lengths,fmt,layout", CHUNKS)
def test_chunk_attention(tq, heads, kv_heads, dim, page, fresh, lengths, fmt, layout, rule):
    B = len(lengths)
    rule = RULES[rule](heads, B)
    for ones in (False, True):
        cache, q, starts, tables, lens, pages = case(tq, fresh, lengths, heads, kv_heads, dim, page, fmt, layout, 3, spread=2.0, ones=ones, gap=3)
        want = reference(q, starts, values_of(cache, "k"), values_of(cache, "v"), tables, lens, dim ** -0.5, pages, rule)
        out = torch.full(q.shape, 7.0, dtype=BF, device=DEV)
        got = tq.torq_chunk_attention(q.to(DEV), starts.to(DEV), cache, tables.to(DEV), lens.to(DEV), dim ** -0.5, most=max(fresh), scores=rule.on(tq), out=out)
        assert got is out and bool((out[-3:] == 7.0).all())                             # rows of no request
        check(got, *want, few(heads, kv_heads, max(fresh)))


def lengthened(tables, page, most):
    """The same tables with room for many more tokens, in pages of nobody: what is chosen by the tables' width is chosen otherwise."""
    more = -(-(2048 + most) // page)
    return torch.cat([tables, torch.full((tables.shape[0], more), -1, dtype=torch.int32)], 1)


LONG = [c for c in CHUNKS if c[0] // c[1] * max(c[4]) > 128 and c[2] <= 128] + [
    (32, 8, 128, 16, [65, 500, 3], [65, 2800, 40], "bf16", "heads"), (16, 2, 128, 64, [100, 0, 70], [2200, 30, 71], "mxfp8", "heads"),
    (16, 2, 96, 16, [99, 64], [400, 2222], "mxfp4", "tokens"), (4, 4, 64, 32, [257, 150], [1030, 2100], "mxfp8", "pairs"),
    (4, 4, 64, 32, [256, 129], [256, 129], "mxfp4", "heads"), (6, 2, 88, 16, [70, 300], [70, 310], "bf16", "heads")]


@gpu
@pytest.mark.parametrize("rule", ["plain", "slopes", "window 1", "prefix", "first and last", "slopes and all"])
@pytest.mark.parametrize("heads,kv_heads,dim,page,fresh,lengths,fmt,layout", LONG)
def test_chunk_attention_behind_long_tables(tq, heads, kv_heads, dim, page, fresh, lengths, fmt, layout, rule):
    B = len(lengths)
    if rule == "slopes and all":
        rule = Rule(slopes=slopes_of(heads), window=2000 + max(fresh), prefix=torch.full((B,), 33, dtype=torch.int32))
    else:
        rule = RULES[rule](heads, B)
    for ones in (False, True):
        cache, q, starts, tables, lens, pages = case(tq, fresh, lengths, heads, kv_heads, dim, page, fmt, layout, 11, spread=2.0, ones=ones, gap=3)
        tables = lengthened(tables, page, max(fresh))
        want = reference(q, starts, values_of(cache, "k"), values_of(cache, "v"), tables, lens, dim ** -0.5, pages, rule)
        out = torch.full(q.shape, 7.0, dtype=BF, device=DEV)
        tq.torq_chunk_attention(q.to(DEV), starts.to(DEV), cache, tables.to(DEV), lens.to(DEV), dim ** -0.5, most=max(fresh), scores=rule.on(tq), out=out)
        assert bool((out[-3:] == 7.0).all())
        check(out, *want, False)


POISONED = [
    # heads, kv_heads, head_dim, page, new tokens, tokens, format
    (8, 2, 64, 16, [1, 1, 1], [40, 200, 33], "bf16"), (16, 1, 128, 16, [1, 1], [90, 150], "mxfp8"), (4, 4, 256, 16, [1, 1], [90, 150], "mxfp4"),
    (48, 2, 128, 16, [1, 1], [90, 150], "bf16"), (16, 2, 96, 32, [3, 1, 4], [90, 40, 4], "mxfp4"), (8, 8, 128, 16, [20, 9], [20, 100], "bf16"),
    (8, 2, 128, 16, [70, 9, 130], [70, 100, 200], "bf16"), (8, 2, 128, 16, [70, 9, 130], [70, 100, 200], "mxfp8"), (8, 2, 96, 16, [40, 9], [70, 100], "mxfp4"),
    (4, 1, 64, 48, [150], [300], "bf16"), (8, 4, 256, 16, [50, 60], [80, 60], "mxfp8"), (6, 2, 160, 16, [30, 12], [80, 60], "bf16")]


@gpu
@pytest.mark.parametrize("long", [False, True])
@pytest.mark.parametrize("rule", ["plain", "window 1", "window 50", "prefix", "first and last", "slopes", "everything"])
@pytest.mark.parametrize("heads,kv_heads,dim,page,fresh,lengths,fmt", POISONED)
def test_what_a_query_does_not_see_takes_no_part(tq, heads, kv_heads, dim, page, fresh, lengths, fmt, rule, long):
    """Tokens whose keys and values are not finite: rows that see them are not finite where those are, the others are as without."""
    B = len(lengths)
    rule = RULES[rule](heads, B)
    cache, q, starts, tables, lens, pages = case(tq, fresh, lengths, heads, kv_heads, dim, page, fmt, "heads", 5)
    if long:
        tables = lengthened(tables, page, max(fresh))
    g = rng(lengths, fresh, 9)
    for b, n in enumerate(lengths):                  # in some places of values, and in whole keys
        for t in sorted({0, n // 3, n // 2, n - 2, n - 1}):
            if t < 0:
                continue
            entry, place, what = int(tables[b, t // page]), t % page, int(torch.randint(0, 3, (1,), generator=g))
            i = int(torch.randint(0, dim, (1,), generator=g))
            if fmt == "bf16":
                cache.v[entry, :, place, i] = (math.nan, math.inf, -math.inf)[what]
                if what == 0:
                    cache.k[entry, :, place, i] = math.nan
            elif fmt == "mxfp8" and what:
                cache.v.view(torch.uint8)[entry, :, place, i] = 0x7F
            else:
                cache.v_scales.view(torch.uint8)[entry, :, place, i // 32] = 0xFF
                cache.k_scales.view(torch.uint8)[entry, :, place, i // 32] = 0xFF
    want, weight = reference(q, starts, values_of(cache, "k"), values_of(cache, "v"), tables, lens, dim ** -0.5, pages, rule)
    there = torch.cat([torch.arange(int(starts[b]), int(starts[b + 1])) for b in range(B)])
    if max(fresh) == 1:
        got = tq.torq_paged_attention(q.to(DEV), cache, tables.to(DEV), lens.to(DEV), dim ** -0.5, scores=rule.on(tq))
    else:
        got = tq.torq_chunk_attention(q.to(DEV), starts.to(DEV), cache, tables.to(DEV), lens.to(DEV), dim ** -0.5, most=max(fresh), scores=rule.on(tq))
    got, want, weight = got.cpu()[there], want[there], weight[there]
    assert torch.equal(torch.isfinite(got), torch.isfinite(want)), (torch.isfinite(got) != torch.isfinite(want)).nonzero()[:5].tolist()
    # an infinity comes through as itself, or as NaN where its weight is below 2^-126, fp32's least normal number, and so 0: 0 times infinity
    infinite, nan = torch.isinf(want), torch.isnan(want)
    assert bool(torch.isnan(got)[nan].all()) and bool(((got.double() == want) | torch.isnan(got))[infinite].all())
    if rule.slopes is None:                          # (scores of a few units: no weight is that small)
        assert torch.equal(torch.isnan(got), nan)
    fine = torch.isfinite(want)
    check(torch.where(fine, got.double(), 0.0), torch.where(fine, want, 0.0), torch.where(fine, weight, 1.0), few(heads, kv_heads, max(fresh)))


@gpu
@pytest.mark.parametrize("scale", [0.0, -0.2, 1e-30, 3.0])
@pytest.mark.parametrize("cap", [0.0, 1e-3, 2.0, 170.0, 200.0, 1e5, 1e30])
@pytest.mark.parametrize("fresh,dim", [([1, 1], 128), ([3, 2], 64), ([40, 70], 128), ([70, 80], 64), ([50, 33], 256)])
def test_scales_and_caps_of_every_size(tq, fresh, dim, cap, scale):
    lengths = [90, 100]
    cache, q, starts, tables, lens, pages = case(tq, fresh, lengths, 4, 2, dim, 16, "bf16", "heads", 7, spread=1.0)
    for slopes in (None, slopes_of(4)):
        rule = Rule(cap=cap, slopes=slopes)
        want = reference(q, starts, values_of(cache, "k"), values_of(cache, "v"), tables, lens, scale, pages, rule)
        got = tq.torq_chunk_attention(q.to(DEV), starts.to(DEV), cache, tables.to(DEV), lens.to(DEV), scale, most=max(fresh), scores=rule.on(tq))
        check(got, *want, few(4, 2, max(fresh)))
