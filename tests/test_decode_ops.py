"""The attention side of a decoder block on the GPU: torq_block_tables, torq_cache_append, torq_paged_attention and
torq_add_rms_norm against plain implementations in 64 bits (or, where values are copied or rounded by definition, bit for bit), and their
refusals, which need no GPU."""
import ctypes as C
import math
import zlib

import numpy as np
import pytest
import torch

from paper_2605_19561_amd import binding

DEV = "cuda:0"
BF, F8, E8 = torch.bfloat16, torch.float8_e4m3fn, torch.float8_e8m0fnu
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


# ---- MXFP8 from its definition -----------------------------------------------------------------

def e4m3_values():
    """The 127 magnitudes of E4M3, exactly."""
    return np.array([m / 512.0 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8) if (e, m) != (15, 7)])


def mxfp8(x):
    """float64 [..., n] -> codes and scale bytes [..., n / 32], uint8, from the definition in the header."""
    x = np.asarray(x, dtype=np.float64)
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    bad = ~np.isfinite(blocks).all(-1)
    amax = np.abs(np.where(np.isfinite(blocks), blocks, 0.0)).max(-1)
    e = np.full(amax.shape, -127)
    for k in range(-127, 128):                       # the least power of two that reaches
        e = np.where((amax > 448 * 2.0 ** (k - 1)) & (k > -127), k, e)
    z = blocks / 2.0 ** e[..., None].astype(np.float64)
    values = e4m3_values()
    mag = np.abs(np.where(np.isfinite(z), z, 0.0))
    hi = np.clip(np.searchsorted(values, mag), 1, 126)
    lo = hi - 1
    up, down = values[hi] - mag, mag - values[lo]
    code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    code = np.where(mag >= values[126], 126, code)
    code = code | np.where(np.signbit(blocks), 0x80, 0)
    code = np.where(bad[..., None], 0x7F, code)
    return code.reshape(x.shape).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def test_the_tests_own_mxfp8_agrees_with_torch():
    x = torch.randn((64, 96), generator=rng(1), dtype=torch.float64) * 10.0 ** torch.randint(-6, 6, (64, 1), generator=rng(2))
    codes, scales = mxfp8(x.numpy())
    e = scales.astype(np.float64) - 127
    z = x.reshape(64, 3, 32) / 2.0 ** torch.from_numpy(e)[..., None]
    assert float(z.abs().max()) <= 448 and float(z.abs().amax(-1).min()) > 224
    assert np.array_equal(z.float().to(F8).view(torch.uint8).reshape(64, 96).numpy(), codes)


def u8(t):
    return t.contiguous().view(torch.uint8).cpu().numpy()


def values_of(cache, name):
    """[pages, heads, page_size, head_dim] float64 on the CPU."""
    t = getattr(cache, name).cpu()
    if cache.format == binding.TORQ_FMT_BF16:
        return t.double()
    s = getattr(cache, name + "_scales").cpu()
    s = s if s.dtype == E8 else s.contiguous().view(E8)
    return t.double() * s.double().repeat_interleave(32, -1)


# ---- pages and slots ---------------------------------------------------------------------------

def tables_reference(held, lengths, free, cursor, tables, page, tokens):
    tables, slots, at = tables.copy(), [], cursor
    width = tables.shape[1]
    for b, (h, n) in enumerate(zip(held, lengths)):
        h, n = max(h, 0), max(n, 0)
        had, have = min(-(-h // page), width), min(-(-n // page), width)
        for j in range(had, have):
            tables[b, j] = free[at] if at < len(free) else -1
            at += 1
        for p in range(h, n):
            if len(slots) < tokens:
                entry = tables[b, p // page] if p // page < width else -1
                slots.append(-1 if entry < 0 else int(entry) * page + p % page)
    return tables, slots + [-1] * (tokens - len(slots)), at


TABLES = {
    # name: (held, lengths, page, width, free pages, handed out before, tokens or None for all)
    "decode": ([15, 16, 17, 0, 31], [16, 17, 18, 1, 32], 16, 4, 50, 3, None),
    "prefill": ([0, 0, 0, 0], [1, 40, 16, 700], 16, 44, 60, 0, None),
    "one token": ([0], [1], 64, 1, 1, 0, None),
    "nothing new": ([5, 0, 33], [5, 0, 33], 16, 4, 9, 2, None),
    "shorter than held, negative": ([40, -3, 5], [8, 20, -7], 16, 4, 9, 0, None),
    "list runs out": ([0, 16, 0], [40, 17, 33], 16, 5, 4, 1, None),
    "list is empty": ([0, 16], [3, 18], 16, 5, 0, 0, None),
    "wider than the table": ([30, 0], [70, 100], 16, 3, 20, 0, None),
    "more places than tokens": ([3, 9], [5, 10], 16, 2, 5, 0, 11),
    "fewer places than tokens": ([3, 9, 0], [15, 30, 8], 16, 2, 5, 0, 9),
    "no places": ([0, 3], [5, 40], 16, 4, 9, 0, 0),
    "long prompts, many workgroups": ([0, 100, 0], [20000, 9000, 3], 48, 420, 700, 5, None),
    "odd page": ([6, 7, 8], [14, 15, 30], 7, 6, 30, 0, None),
}


@gpu
@pytest.mark.parametrize("name", sorted(TABLES))
@pytest.mark.parametrize("in_place", [False, True])
def test_block_tables(tq, either_way, name, in_place):
    held, lengths, page, width, pages, cursor, tokens = TABLES[name]
    new = sum(max(0, max(n, 0) - max(h, 0)) for h, n in zip(held, lengths))
    tokens = new if tokens is None else tokens
    free = torch.randperm(pages + 7, generator=rng(name)).int()[:pages].numpy()
    base = torch.randint(0, 1000, (len(held), width + 3), generator=rng(name, 2), dtype=torch.int32)
    want, slots, after = tables_reference(held, lengths, free, cursor, base[:, :width].numpy(), page, tokens)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    whole = base.to(DEV)
    cur = ints([cursor])
    got_slots, got_after = tq.torq_block_tables(ints(held), ints(lengths), ints(free), cur, whole[:, :width], page, tokens,
                                                cursor_out=cur if in_place else None)
    assert whole[:, :width].cpu().numpy().tolist() == want.tolist()
    assert torch.equal(whole[:, width:].cpu(), base[:, width:])              # the rest of a wider table is left alone
    assert got_slots.tolist() == slots and got_slots.dtype == torch.int64 and got_after.tolist() == [after]
    assert (got_after is cur) == in_place and (in_place or cur.tolist() == [cursor])


@gpu
@pytest.mark.parametrize("B", [0, 1, 255, 1024, 1025, 2500])
def test_block_tables_of_many_requests(tq, B):
    g = np.random.default_rng(B)
    held = g.integers(0, 90, B).astype(np.int32)
    lengths = held + (g.integers(0, 5, B) * g.integers(0, 9, B)).astype(np.int32)
    page, width = 16, 9
    free = g.permutation(4 * B + 1).astype(np.int32)
    tables = g.integers(0, 500, (B, width)).astype(np.int32)
    tokens = int((lengths - held).sum()) + 3
    want, slots, after = tables_reference(held.tolist(), lengths.tolist(), free, 1, tables, page, tokens)
    dev = lambda a: torch.from_numpy(a).to(DEV)
    t = dev(tables)
    got, cur = tq.torq_block_tables(dev(held), dev(lengths), dev(free), torch.ones(1, dtype=torch.int32, device=DEV), t, page, tokens)
    assert np.array_equal(t.cpu().numpy(), want) and got.tolist() == slots and cur.tolist() == [after]


# ---- new keys and values -----------------------------------------------------------------------

def make_cache(tq, pages, heads, page, dim, fmt, layout, device=DEV):
    """Filled with bytes that no append writes where it should not."""
    mx = fmt == "mxfp8"
    elt, unit = (F8, 32) if mx else (BF, 1)

    def block(last, dtype, two):
        lead = (2,) if two else ()
        if layout == "heads":
            t = torch.empty((*lead, pages, heads, page, last), dtype=dtype, device=device)
        elif layout == "tokens":
            t = torch.empty((*lead, pages, page, heads, last), dtype=dtype, device=device).transpose(-3, -2)
        else:                                        # keys and values of a page side by side
            t = torch.empty((pages, 2, heads, page, last), dtype=dtype, device=device).transpose(0, 1)
        return t
    kv = block(dim, elt, True)
    kv.contiguous()
    sc = block(dim // 32, torch.uint8, True) if mx else (None, None)
    for t in (kv[0], kv[1], *(sc if mx else ())):
        t.view(torch.uint8 if mx else torch.int16).fill_(0x33)
    return tq.KVCache(kv[0], kv[1], sc[0].view(E8) if mx else None, sc[1].view(E8) if mx else None)


APPEND = [
    # tokens, heads, head_dim, page, format, layout, packed input
    (1, 1, 8, 16, "bf16", "heads", False), (1, 1, 32, 16, "mxfp8", "heads", False), (5, 3, 72, 48, "bf16", "tokens", True),
    (33, 8, 128, 16, "bf16", "heads", True), (33, 8, 128, 16, "mxfp8", "tokens", True), (17, 2, 96, 32, "mxfp8", "pairs", False),
    (40, 5, 256, 64, "bf16", "pairs", True), (3000, 4, 64, 16, "mxfp8", "heads", True), (700, 20, 80, 112, "bf16", "heads", False)]


@gpu
@pytest.mark.parametrize("T,heads,dim,page,fmt,layout,packed", APPEND)
def test_cache_append(tq, either_way, T, heads, dim, page, fmt, layout, packed):
    pages = -(-T // page) + 3
    g = rng(T, heads, dim)
    x = (torch.randn((T, 2 * heads + 3, dim), generator=g) * torch.exp(4 * torch.randn((T, 2 * heads + 3, 1), generator=g))).to(BF)
    x[:, :, ::7] *= 0.001
    if T > 2:                                        # blocks whose maximum lies at the border of a scale, zeros, subnormals
        x[0, :, :] = 0.0
        x[1, :, 0], x[1, :, 1:] = 448.0, 1.0
        x[2, :, 0], x[2, :, 1:] = -450.0, 2.0 ** -126
    x = x.to(DEV)
    key, value = (x[:, 3:3 + heads], x[:, 3 + heads:]) if packed else (x[:, :heads].contiguous(), x[:, heads:2 * heads].contiguous())
    slots = torch.randperm(pages * page, generator=g)[:T]
    if T > 4:
        slots[3], slots[4] = -1, pages * page        # passed over
    cache = make_cache(tq, pages, heads, page, dim, fmt, layout)
    names = ["k", "v"] + (["k_scales", "v_scales"] if fmt == "mxfp8" else [])
    before = {n: u8(getattr(cache, n)).copy() for n in names}
    tq.torq_cache_append(cache, key, value, slots.to(DEV))
    want = before
    for name, new in (("k", key), ("v", value)):
        new = new.cpu()
        if fmt == "bf16":
            parts = [(name, new.contiguous().view(torch.uint8).numpy())]
        else:
            parts = list(zip((name, name + "_scales"), mxfp8(new.double().numpy())))
        for n, rows in parts:
            for t, slot in enumerate(slots.tolist()):
                if 0 <= slot < pages * page:
                    want[n][slot // page, :, slot % page] = rows[t].reshape(heads, -1)
    for n in names:
        assert np.array_equal(u8(getattr(cache, n)), want[n]), n


@gpu
def test_cache_append_marks_blocks_that_are_not_finite(tq):
    x = torch.ones((4, 1, 64), dtype=BF)
    x[0, 0, 5], x[1, 0, 40], x[2, 0, 63] = math.inf, math.nan, -math.inf
    cache = make_cache(tq, 1, 1, 16, 64, "mxfp8", "heads")
    x = x.to(DEV)
    tq.torq_cache_append(cache, x, x, torch.arange(4, device=DEV))
    codes, scales = mxfp8(x.cpu().double().numpy())
    assert np.array_equal(u8(cache.k)[0, 0, :4], codes[:, 0]) and np.array_equal(u8(cache.v_scales)[0, 0, :4], scales[:, 0])
    assert scales[:, 0].tolist() == [[255, 119], [119, 255], [119, 255], [119, 119]]
    assert torch.isnan(cache.k[0, 0, 0, :32].float()).all() and not torch.isnan(cache.k[0, 0, 0, 32:].float()).any()


# ---- attention ---------------------------------------------------------------------------------

def attention_reference(q, k, v, tables, lengths, scale, pages):
    """float64: out, and sum_t p_t |v_t|, which errors of the weights are relative to.  k, v [pages, heads, page, dim] float64."""
    B, heads, dim = q.shape
    kv_heads, page = k.shape[1], k.shape[2]
    group = heads // kv_heads
    out, weight = torch.zeros((B, heads, dim), dtype=torch.float64), torch.zeros((B, heads, dim), dtype=torch.float64)
    for b in range(B):
        n = min(max(int(lengths[b]), 0), tables.shape[1] * page)
        token = torch.arange(n)
        entry = tables[b].long()[token // page] if n else token
        token, entry = token[(entry >= 0) & (entry < pages)], entry[(entry >= 0) & (entry < pages)]
        if not len(token):
            continue
        for h in range(kv_heads):
            kk, vv = k[entry, h, token % page], v[entry, h, token % page]
            s = q[b, h * group:(h + 1) * group].double() @ kk.T * scale
            p = torch.softmax(s, -1)
            out[b, h * group:(h + 1) * group], weight[b, h * group:(h + 1) * group] = p @ vv, p @ vv.abs()
    return out, weight


def check_attention(got, out, weight):
    # the output's rounding to bf16, 2^-8 |out| <= 2^-9 (|out| + sum p |v|), which one rounding of the weights p to bf16 would pass;
    # fp32's part (a dot product of up to 256 terms before the exponential, sums over the tokens) is below 2^-12 of the same for the
    # values drawn here
    bound = (2.0 ** -9 + 2.0 ** -12) * (out.abs() + weight) + 1e-38
    worst = ((got.double().cpu() - out).abs() / bound).max()
    assert float(worst) <= 1.0, float(worst)


def attention_case(tq, B, heads, kv_heads, dim, page, lengths, fmt, layout, seed, spread=1.0, poison=True):
    g = rng(B, heads, dim, page, fmt, seed)
    need = [-(-n // page) for n in lengths]
    pages, width = sum(need) + 4, max(need + [1]) + 2
    cache = make_cache(tq, pages, kv_heads, page, dim, fmt, layout)
    order, at = torch.randperm(pages, generator=g).int(), 0
    tables = torch.full((B, width), -1, dtype=torch.int32)
    for b, n in enumerate(need):
        tables[b, :n] = order[at:at + n]
        at += n
    # what lies behind a length, in the last page or in pages of nobody, is no finite value
    for t in (cache.k, cache.v):
        t.view(torch.uint8 if fmt == "mxfp8" else torch.int16).fill_((0x7F if fmt == "mxfp8" else 0x7FC0) if poison else 0)
    T = sum(lengths)
    x = torch.randn((T, 2, kv_heads, dim), generator=g)
    x[:, 0, :, ::9] *= 3.0 * spread
    slots = [int(tables[b, p // page]) * page + p % page for b, n in enumerate(lengths) for p in range(n)]
    x = x.to(BF).to(DEV)
    if T:
        tq.torq_cache_append(cache, x[:, 0], x[:, 1], torch.tensor(slots, dtype=torch.int64, device=DEV))
    q = (torch.randn((B, heads, dim), generator=g) * spread).to(BF)
    return cache, q, tables, torch.tensor(lengths, dtype=torch.int32), pages


ATTENTION = [
    # heads, kv_heads, head_dim, page, lengths, format, layout
    (1, 1, 8, 16, [1], "bf16", "heads"),
    (1, 1, 32, 16, [1, 0, 2], "mxfp8", "heads"),
    (32, 8, 128, 16, [1, 15, 16, 17, 31, 32, 33, 0, 127, 128, 129], "bf16", "heads"),
    (32, 8, 128, 16, [1, 15, 16, 17, 31, 32, 33, 0, 127, 128, 129], "mxfp8", "heads"),
    (64, 8, 128, 64, [2000, 257, 1, 511], "bf16", "tokens"),
    (64, 8, 128, 32, [2000, 257, 1, 511], "mxfp8", "tokens"),
    (20, 20, 80, 48, [3, 300, 0, 47, 48, 49, 95, 97], "bf16", "tokens"),
    (5, 1, 72, 112, [113, 224, 700], "bf16", "pairs"),
    (7, 1, 64, 16, [65, 130], "bf16", "heads"), (7, 1, 64, 16, [65, 130], "mxfp8", "pairs"),
    (12, 1, 96, 16, [77, 200], "mxfp8", "heads"), (12, 1, 96, 16, [77, 200], "bf16", "heads"),
    (17, 1, 112, 32, [90, 1], "bf16", "heads"), (48, 2, 128, 16, [300, 20], "mxfp8", "heads"), (71, 1, 64, 16, [300, 20], "bf16", "heads"),
    # more than 16 query heads for a key head, few and many of those
    (24, 1, 128, 16, [1, 0, 2, 33, 700] * 8, "bf16", "heads"), (68, 4, 96, 32, [31, 257, 0, 64, 129, 1] * 3, "mxfp8", "tokens"),
    (64, 2, 64, 16, [5, 520, 0, 77] * 5, "bf16", "pairs"), (33, 1, 80, 16, [90, 1, 200, 16] * 9, "bf16", "heads"),
    (80, 2, 128, 16, [300, 45, 0, 1] * 12, "mxfp8", "heads"), (40, 2, 40, 16, [3, 0, 40, 33] * 70, "bf16", "heads"),
    (8, 4, 192, 16, [100, 33], "bf16", "heads"), (8, 4, 192, 16, [100, 33], "mxfp8", "tokens"),
    (16, 1, 256, 16, [400, 31], "bf16", "tokens"), (16, 1, 256, 16, [400, 31], "mxfp8", "heads"),
    (4, 2, 16, 16, [40], "bf16", "heads"), (4, 2, 24, 16, [40], "bf16", "heads"), (4, 4, 40, 16, [40, 3], "bf16", "heads"),
    (8, 1, 128, 1024, [5000], "bf16", "heads"), (8, 1, 128, 16, [33000], "mxfp8", "heads"), (2, 1, 64, 16, [20000, 5], "bf16", "heads")]


@gpu
@pytest.mark.parametrize("heads,kv_heads,dim,page,lengths,fmt,layout", ATTENTION)
def test_paged_attention(tq, either_way, heads, kv_heads, dim, page, lengths, fmt, layout):
    cache, q, tables, lens, pages = attention_case(tq, len(lengths), heads, kv_heads, dim, page, lengths, fmt, layout, 1)
    want = attention_reference(q, values_of(cache, "k"), values_of(cache, "v"), tables, lens, dim ** -0.5, pages)
    # q as columns of a wider product
    wide = torch.zeros((len(lengths), heads + 2, dim), dtype=BF, device=DEV)
    wide[:, 1:-1] = q.to(DEV)
    got = tq.torq_paged_attention(wide[:, 1:-1], cache, tables.to(DEV), lens.to(DEV), dim ** -0.5)
    check_attention(got, *want)
    for b, n in enumerate(lengths):
        if n == 0:
            assert not got[b].any()
    again = tq.torq_paged_attention(q.to(DEV), cache, tables.to(DEV), lens.to(DEV), dim ** -0.5)
    assert torch.equal(again.view(torch.int16), got.view(torch.int16))


@gpu
@pytest.mark.parametrize("heads,kv_heads,dim,page,lengths,fmt,layout", ATTENTION)
def test_paged_attention_with_tables_for_long_requests(tq, heads, kv_heads, dim, page, lengths, fmt, layout):
    # the same requests where the tables would hold long ones: the tokens are cut into runs by the lengths
    cache, q, tables, lens, pages = attention_case(tq, len(lengths), heads, kv_heads, dim, page, lengths, fmt, layout, 1)
    want = attention_reference(q, values_of(cache, "k"), values_of(cache, "v"), tables, lens, dim ** -0.5, pages)
    tables = torch.cat([tables, torch.full((len(lengths), 8192 // page + 1), -1, dtype=torch.int32)], 1)
    got = tq.torq_paged_attention(q.to(DEV), cache, tables.to(DEV), lens.to(DEV), dim ** -0.5)
    check_attention(got, *want)


@gpu
@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
def test_paged_attention_of_many_ragged_requests(tq, fmt):
    g = np.random.default_rng(5)
    lengths = [int(n) for n in g.integers(0, 400, 150)]
    cache, q, tables, lens, pages = attention_case(tq, 150, 4, 2, 64, 16, lengths, fmt, "heads", 2)
    want = attention_reference(q, values_of(cache, "k"), values_of(cache, "v"), tables, lens, 0.125, pages)
    # the table as part of a wider one whose other columns are no pages
    wide = torch.full((150, tables.shape[1] + 5), 1 << 30, dtype=torch.int32)
    wide[:, :tables.shape[1]] = tables
    wide = wide.to(DEV)
    check_attention(tq.torq_paged_attention(q.to(DEV), cache, wide[:, :tables.shape[1]], lens.to(DEV), 0.125), *want)


@gpu
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("heads,kv_heads,dim,fmt,layout", [
    (8, 4, 64, "bf16", "tokens"), (4, 4, 80, "bf16", "tokens"), (16, 4, 128, "bf16", "heads"), (16, 4, 128, "mxfp8", "heads"), (12, 4, 96, "mxfp8", "tokens"),
    (4, 4, 64, "mxfp8", "heads"), (8, 4, 256, "bf16", "heads"), (8, 4, 192, "mxfp8", "heads"), (40, 2, 64, "bf16", "heads"), (72, 4, 32, "mxfp8", "heads")])
def test_paged_attention_of_a_large_batch(tq, heads, kv_heads, dim, fmt, layout, wide):
    # so many (request, key head)s that a wave takes one for itself
    g = np.random.default_rng(dim)
    lengths = [int(n) for n in g.integers(0, 90, 200)]
    lengths[3], lengths[77], lengths[199] = 400, 0, 300
    cache, q, tables, lens, pages = attention_case(tq, 200, heads, kv_heads, dim, 16, lengths, fmt, layout, 7)
    want = attention_reference(q, values_of(cache, "k"), values_of(cache, "v"), tables, lens, dim ** -0.5, pages)
    if wide:
        tables = torch.cat([tables, torch.full((200, 100), -1, dtype=torch.int32)], 1)
    check_attention(tq.torq_paged_attention(q.to(DEV), cache, tables.to(DEV), lens.to(DEV), dim ** -0.5), *want)


@gpu
@pytest.mark.parametrize("long", [False, True])
@pytest.mark.parametrize("heads,kv_heads,dim,fmt", [(8, 8, 64, "bf16"), (16, 2, 64, "bf16"), (8, 8, 128, "bf16"), (16, 2, 128, "bf16"), (8, 8, 128, "mxfp8"),
                                                    (16, 2, 128, "mxfp8"), (4, 4, 256, "bf16"), (16, 2, 256, "bf16"), (4, 4, 256, "mxfp8"), (16, 2, 256, "mxfp8")])
def test_paged_attention_past_the_cache(tq, heads, kv_heads, dim, fmt, long):
    # tables that could name more than 96 MiB of whole lines: read with the non-temporal hint, however little there is
    B = 200 if heads == kv_heads else 3
    g = np.random.default_rng(dim)
    lengths = [int(n) for n in g.integers(0, 120, B)]
    lengths[0], lengths[2] = 0, 450
    cache, q, tables, lens, pages = attention_case(tq, B, heads, kv_heads, dim, 16, lengths, fmt, "heads", 8)
    want = attention_reference(q, values_of(cache, "k"), values_of(cache, "v"), tables, lens, dim ** -0.5, pages)
    # the same pages at the front of a large pool
    size = (1 if fmt == "mxfp8" else 2) * kv_heads * 16 * dim
    pool = 60 * 2 ** 20 // size
    parts = []
    for n in ("k", "v") + (("k_scales", "v_scales") if fmt == "mxfp8" else ()):
        t = getattr(cache, n)
        big = torch.empty((pool, *t.shape[1:]), dtype=torch.uint8 if fmt == "mxfp8" else BF, device=DEV)
        big[:pages] = t.view(torch.uint8) if fmt == "mxfp8" else t
        parts.append(big.view(t.dtype))
    if long or B < 200:                              # (else 32 pages a request, one launch; B requests of them are enough)
        tables = torch.cat([tables, torch.full((B, 40000), -1, dtype=torch.int32)], 1)
    big = tq.KVCache(*parts)
    check_attention(tq.torq_paged_attention(q.to(DEV), big, tables.to(DEV), lens.to(DEV), dim ** -0.5), *want)


@gpu
@pytest.mark.parametrize("heads,kv_heads,dim,fmt,page", [(20, 20, 80, "bf16", 16), (40, 8, 128, "bf16", 32), (16, 8, 64, "mxfp8", 16), (32, 4, 256, "mxfp8", 64), (51, 3, 96, "bf16", 16)])
def test_paged_attention_of_many_tiny_requests(tq, heads, kv_heads, dim, fmt, page):
    # tables for at most 128 tokens
    g = np.random.default_rng(dim)
    lengths = [int(n) for n in g.integers(0, 64 - page + 1, 190)]
    lengths[5], lengths[6] = 64, 0
    cache, q, tables, lens, pages = attention_case(tq, 190, heads, kv_heads, dim, page, lengths, fmt, "tokens", 9)
    assert tables.shape[1] * page <= 192
    tables = tables[:, : 128 // page].contiguous()
    want = attention_reference(q, values_of(cache, "k"), values_of(cache, "v"), tables, lens, dim ** -0.5, pages)
    check_attention(tq.torq_paged_attention(q.to(DEV), cache, tables.to(DEV), lens.to(DEV), dim ** -0.5), *want)


@gpu
@pytest.mark.parametrize("B,heads,kv_heads", [(64, 4, 2), (65, 4, 2), (513, 4, 2), (5000, 2, 1), (5000, 4, 4)])
def test_paged_attention_of_very_many_requests(tq, B, heads, kv_heads):
    # more requests than a wave has lanes, most of them empty or short, a few long, wide tables
    g = np.random.default_rng(B)
    lengths = [int(n) for n in g.integers(0, 40, B) * (g.random(B) < 0.3)]
    lengths[B // 2], lengths[B - 1], lengths[63] = 700, 333, 90
    cache, q, tables, lens, pages = attention_case(tq, B, heads, kv_heads, 32, 16, lengths, "bf16", "heads", 10)
    want = attention_reference(q, values_of(cache, "k"), values_of(cache, "v"), tables, lens, 0.2, pages)
    check_attention(tq.torq_paged_attention(q.to(DEV), cache, tables.to(DEV), lens.to(DEV), 0.2), *want)


@gpu
@pytest.mark.parametrize("native", [True, False])
def test_decode_calls_without_requests_or_tokens(tq, native, monkeypatch):
    if not native:
        monkeypatch.setattr(binding, "_host", binding._Interpreted)
    cache = make_cache(tq, 2, 2, 16, 64, "bf16", "heads")
    before = u8(cache.k).copy()
    none = torch.empty((0, 2, 64), dtype=BF, device=DEV)
    tq.torq_cache_append(cache, none, none, torch.empty(0, dtype=torch.int64, device=DEV))
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=DEV)
    assert np.array_equal(u8(cache.k), before)
    assert tq.torq_paged_attention(none, cache, i32(0, 3), i32(0), 1.0).shape == (0, 2, 64)
    slots, cursor = tq.torq_block_tables(i32(0), i32(0), i32(0), i32(1), i32(0, 0), 16, 3)
    assert slots.tolist() == [-1] * 3 and cursor.tolist() == [0]
    assert tq.torq_add_rms_norm(none[:, 0].contiguous(), none[:, 0].contiguous(), torch.ones(64, dtype=BF, device=DEV), 1e-5, tq.TORQ_FMT_MXFP8)[1].shape == (0, 2)


@gpu
def test_paged_attention_with_one_weight_near_one(tq):
    # scores of hundreds: maxima that move from tile to tile, weights that underflow
    cache, q, tables, lens, pages = attention_case(tq, 3, 8, 2, 128, 16, [500, 64, 1], "bf16", "heads", 3, spread=6.0)
    want = attention_reference(q, values_of(cache, "k"), values_of(cache, "v"), tables, lens, 0.3, pages)
    got = tq.torq_paged_attention(q.to(DEV), cache, tables.to(DEV), lens.to(DEV), 0.3)
    # scores here have an absolute error of up to 136 * 2^-24 * sum |q k| * scale, and it multiplies a weight
    s_err = 136 * 2.0 ** -24 * 0.3 * float(q.double().abs().max()) * 128 * float(values_of(cache, "k").nan_to_num(0).abs().max())
    out, weight = want
    bound = (2.0 ** -9 + 2.0 ** -12) * (out.abs() + weight) + 2 * s_err * weight
    assert ((got.double().cpu() - out).abs() <= bound).all()


@gpu
@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
def test_paged_attention_leaves_out_what_is_no_token(tq, fmt):
    # entries that are no pages within the length, lengths past the table and below zero, a table of no columns
    lengths = [100, 100, 40, 64]
    cache, q, tables, lens, pages = attention_case(tq, 4, 4, 2, 64, 16, lengths, fmt, "heads", 4)
    tables[0, 2], tables[1, :] = -1, pages
    lens[2], lens[3] = -5, 1 << 30
    narrow = tables[:, :4].contiguous()
    want = attention_reference(q, values_of(cache, "k"), values_of(cache, "v"), narrow, lens, 0.125, pages)
    got = tq.torq_paged_attention(q.to(DEV), cache, narrow.to(DEV), lens.to(DEV), 0.125)
    check_attention(got, *want)
    assert not got[1].any() and not got[2].any() and got[3].any()
    none = tq.torq_paged_attention(q.to(DEV), cache, torch.empty((4, 0), dtype=torch.int32, device=DEV), lens.to(DEV), 0.125)
    assert none.shape == q.shape and not none.any()


@gpu
def test_a_cache_without_pages_holds_nothing(tq, either_way):
    k = torch.empty((0, 2, 16, 64), dtype=BF, device=DEV)
    cache = tq.KVCache(k, k)
    x = torch.ones((3, 2, 64), dtype=BF, device=DEV)
    tq.torq_cache_append(cache, x, x, torch.arange(3, device=DEV))
    ones = torch.ones((3, 1), dtype=torch.int32, device=DEV)
    assert not tq.torq_paged_attention(x, cache, 0 * ones, ones[:, 0].contiguous(), 1.0).any()


@gpu
def test_paged_attention_passes_on_what_is_not_finite(tq):
    cache, q, tables, lens, pages = attention_case(tq, 3, 2, 1, 64, 16, [50, 50, 50], "bf16", "heads", 5)
    cache.k[int(tables[0, 1]), 0, 3, 7] = math.nan
    cache.v[int(tables[1, 0]), 0, 2, 9] = math.inf
    got = tq.torq_paged_attention(q.to(DEV), cache, tables.to(DEV), lens.to(DEV), 0.125).float().cpu()
    assert torch.isnan(got[0]).all() and torch.isinf(got[1, :, 9]).all()
    assert torch.isfinite(got[1, :, :9]).all() and torch.isfinite(got[2]).all()


@gpu
def test_paged_attention_of_tiny_mxfp8_values(tq):
    # blocks of zeros and blocks at the least scale, 2^-127: next to nothing, and nothing else
    cache = make_cache(tq, 1, 1, 16, 32, "mxfp8", "heads")
    x = torch.zeros((2, 1, 32), dtype=BF)
    x[1] = 2.0 ** -125
    x = x.to(DEV)
    tq.torq_cache_append(cache, x, x, torch.arange(2, device=DEV))
    assert u8(cache.k_scales)[0, 0, :2].tolist() == [[0], [0]]
    q = torch.ones((1, 1, 32), dtype=BF, device=DEV)
    got = tq.torq_paged_attention(q, cache, torch.zeros((1, 1), dtype=torch.int32, device=DEV), torch.tensor([2], dtype=torch.int32, device=DEV), 1.0)
    assert float(got.abs().max()) <= 2.0 ** -125


@gpu
def test_paged_attention_past_32_bits(tq):
    # pages whose places, in bytes and in elements, do not fit 32 bits
    dim, page, heads = 128, 16, 1
    pages = (1 << 32) // (page * dim) + 40
    k = torch.empty((pages, heads, page, dim), dtype=BF, device=DEV)
    cache = tq.KVCache(k, torch.empty_like(k))
    at = [pages - 1, 7, pages - 20, (1 << 31) // (page * dim) + 3]
    tables = torch.tensor([at], dtype=torch.int32, device=DEV)
    n = 60
    x = torch.randn((n, 2, heads, dim), generator=rng(77)).to(BF).to(DEV)
    slots = torch.tensor([at[p // page] * page + p % page for p in range(n)], dtype=torch.int64, device=DEV)
    tq.torq_cache_append(cache, x[:, 0], x[:, 1], slots)
    q = torch.randn((1, 4, dim), generator=rng(78)).to(BF)
    got = tq.torq_paged_attention(q.to(DEV), cache, tables, torch.tensor([n], dtype=torch.int32, device=DEV), dim ** -0.5)
    rows = x.cpu().double()
    small_k, small_v = (torch.zeros((4, heads, page, dim), dtype=torch.float64) for _ in "kv")
    for p in range(n):
        small_k[p // page, :, p % page], small_v[p // page, :, p % page] = rows[p, 0], rows[p, 1]
    check_attention(got, *attention_reference(q, small_k, small_v, torch.arange(4)[None], torch.tensor([n]), dim ** -0.5, 4))


@gpu
def test_decode_calls_on_another_stream_and_in_a_graph(tq):
    lengths = [200, 3, 90]
    cache, q, tables, lens, pages = attention_case(tq, 3, 8, 2, 64, 16, lengths, "mxfp8", "heads", 6)
    q, tables, lens = q.to(DEV), tables.to(DEV), lens.to(DEV)
    weight = torch.ones(512, dtype=BF, device=DEV)
    x = torch.randn((3, 512), generator=rng(9)).to(BF).to(DEV)
    want = tq.torq_paged_attention(q, cache, tables, lens, 0.125)
    want_norm = tq.torq_add_rms_norm(x, want.view(3, 512), weight, 1e-5)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = tq.torq_paged_attention(q, cache, tables, lens, 0.125, stream=stream)
    got.record_stream(stream)
    norm = tq.torq_add_rms_norm(x, got.view(3, 512), weight, 1e-5, stream=stream)
    stream.synchronize()
    assert torch.equal(got, want) and torch.equal(norm[0], want_norm[0]) and torch.equal(norm[2], want_norm[2])

    # a step with kept buffers, captured: each replay goes on from the state that the last one left
    held, free = lens.clone(), torch.arange(pages - 4, pages, dtype=torch.int32, device=DEV)
    cursor, ws = torch.zeros(1, dtype=torch.int32, device=DEV), torch.empty(tq.torq_paged_attention_workspace_bytes(cache, 8, 3, tables.shape[1]) + 16, dtype=torch.uint8, device=DEV)
    slots, out, now = torch.empty(3, dtype=torch.int64, device=DEV), torch.empty_like(q), held.clone()
    new = torch.randn((3, 2, 2, 64), generator=rng(10)).to(BF).to(DEV)

    def step():
        now.copy_(held + 1)
        tq.torq_block_tables(held, now, free, cursor, tables, 16, 3, slots=slots, cursor_out=cursor)
        tq.torq_cache_append(cache, new[:, 0], new[:, 1], slots)
        tq.torq_paged_attention(q, cache, tables, now, 0.125, out=out, workspace=ws)
        held.copy_(now)

    state = [t.clone() for t in (held, cursor, tables, cache.k.view(torch.uint8), cache.v.view(torch.uint8), cache.k_scales.view(torch.uint8), cache.v_scales.view(torch.uint8))]
    restore = lambda: [a.copy_(b) for a, b in zip((held, cursor, tables, cache.k.view(torch.uint8), cache.v.view(torch.uint8), cache.k_scales.view(torch.uint8), cache.v_scales.view(torch.uint8)), state)]
    eager = []
    for _ in range(4):
        step()
        eager.append((out.clone(), slots.clone(), tables.clone(), cursor.clone()))
    restore()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    restore()
    for o, s, t, c in eager:
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, o) and torch.equal(slots, s) and torch.equal(tables, t) and torch.equal(cursor, c)
        (q.float() @ q.float().transpose(1, 2)).sum().item()                  # the program's own work between replays


# ---- norm --------------------------------------------------------------------------------------

NORM = [(1, 32), (3, 64), (5, 96), (64, 128), (2, 2048), (3, 2080), (1, 4096), (7, 5120), (2, 8192), (3, 8224), (2, 14336), (2, 25600), (1, 28672), (2, 32768)]


def norm_reference(x, r, w, eps):
    s = x.double() if r is None else x.double() + r.double()
    return s, s / (s.pow(2).mean(-1, keepdim=True) + eps).sqrt() * w.double()


@gpu
@pytest.mark.parametrize("M,d", NORM)
@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
@pytest.mark.parametrize("with_residual", [True, False])
def test_add_rms_norm(tq, either_way, M, d, fmt, with_residual):
    g = rng(M, d)
    x = (torch.randn((M, d), generator=g) * 3).to(BF)
    x[:, ::17] *= 30
    r = torch.randn((M, d), generator=g).to(BF) if with_residual else None
    w = (1 + 0.3 * torch.randn(d, generator=g)).to(BF)
    s, y = norm_reference(x, r, w, 1e-5)
    form = tq.TORQ_FMT_BF16 if fmt == "bf16" else tq.TORQ_FMT_MXFP8
    out, scales, total = tq.torq_add_rms_norm(x.to(DEV), None if r is None else r.to(DEV), w.to(DEV), 1e-5, form)
    if r is None:
        assert total is None
    else:                                            # bf16 + bf16 in fp32, then rounded: fp32's rounding first, 2^-24
        assert ((total.double().cpu() - s).abs() <= (2.0 ** -8 + 2.0 ** -23) * s.abs()).all()
    # fp32's part of y: a sum of d squares in pieces of at most 128 and a tree (2^-17), a root, a quotient, two products
    part = 2.0 ** -16
    if fmt == "bf16":
        assert scales is None and out.dtype == BF
        assert ((out.double().cpu() - y).abs() <= (2.0 ** -8 + part) * y.abs() + 1e-38).all()
        return
    assert out.dtype == F8 and scales.dtype == E8 and scales.shape == (M, d // 32)
    # the scale is the definition's for some value within fp32's part of the largest
    amax = y.abs().reshape(M, -1, 32).amax(-1)
    byte = scales.view(torch.uint8).cpu().double()
    assert (amax * (1 - part) <= 448 * 2.0 ** (byte - 127)).all() and (amax * (1 + part) > 224 * 2.0 ** (byte - 127)).all()
    # E4M3: half a unit in the last of four significant bits, and of the least ones' spacing 2^-9
    back = out.double().cpu() * (2.0 ** (byte - 127)).repeat_interleave(32, -1)
    spacing = (2.0 ** (byte - 127 - 9)).repeat_interleave(32, -1)
    assert ((back - y).abs() <= (2.0 ** -4 + 2 * part) * y.abs() + spacing / 2).all()


@gpu
@pytest.mark.parametrize("M,d", [(1000, 32), (999, 128), (777, 160), (501, 256), (333, 288), (130, 1024), (70, 1056)])
@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
def test_add_rms_norm_of_many_short_rows(tq, M, d, fmt):
    # rows that share a wave or a workgroup, the last of them not full
    g = rng(M, d)
    x, w = torch.randn((M, d), generator=g).to(BF), (1 + 0.1 * torch.randn(d, generator=g)).to(BF)
    _, y = norm_reference(x, None, w, 1e-6)
    form = tq.TORQ_FMT_BF16 if fmt == "bf16" else tq.TORQ_FMT_MXFP8
    out, scales, _ = tq.torq_add_rms_norm(x.to(DEV), None, w.to(DEV), 1e-6, form)
    if fmt == "bf16":
        assert ((out.double().cpu() - y).abs() <= (2.0 ** -8 + 2.0 ** -16) * y.abs() + 1e-38).all()
        return
    step = (2.0 ** (scales.view(torch.uint8).cpu().double() - 127)).repeat_interleave(32, -1)
    assert ((out.double().cpu() * step - y).abs() <= (2.0 ** -4 + 2.0 ** -15) * y.abs() + step * 2.0 ** -10).all()


@gpu
def test_add_rms_norm_in_place_and_at_the_edges(tq):
    g = rng(8)
    x, r, w = torch.randn((5, 256), generator=g).to(BF), torch.randn((5, 256), generator=g).to(BF), torch.ones(256, dtype=BF)
    x[1], r[1] = 0, 0                                # a row of zeros: eps carries it
    x[2] = 2.0 ** 59                                 # squares of 2^118, the sum of 256 fits fp32
    r[2] = 0
    x[3, 7] = math.nan
    x[4] = 2.0 ** -70                                # squares of 2^-140 against eps = 0: subnormal sums
    r[4] = 0
    a, b = x.to(DEV), r.to(DEV)
    want = tq.torq_add_rms_norm(a, b, w.to(DEV), 1e-6)
    assert not want[0][1].any() and torch.isnan(want[0][3]).all() and not want[2][1].any()
    assert ((want[0][2].double().cpu() - 1).abs() <= 2.0 ** -8 + 2.0 ** -16).all() and float(want[0][4].abs().max()) < 1e-15
    for residual_out, out in ((b, None), (a, None), (b, a)):
        p, q = a.clone(), b.clone()
        ro, o = (q if residual_out is b else p), (p if out is a else None)
        got = tq.torq_add_rms_norm(p, q, w.to(DEV), 1e-6, residual_out=ro, out=o)
        assert got[2] is ro and torch.equal(got[0].view(torch.int16), want[0].view(torch.int16)) and torch.equal(got[2].view(torch.int16), want[2].view(torch.int16))
    none = tq.torq_add_rms_norm(torch.empty((0, 64), dtype=BF, device=DEV), None, w[:64].to(DEV), 1e-6)
    assert none[0].shape == (0, 64)
    codes, scales, _ = tq.torq_add_rms_norm(a, b, w.to(DEV), 1e-6, tq.TORQ_FMT_MXFP8)
    assert (scales.view(torch.uint8)[3] == 255).all() and (codes.view(torch.uint8)[3] == 0x7F).all() and (scales.view(torch.uint8)[1] == 0).all()


# ---- refusals, on the host ---------------------------------------------------------------------

def cache_struct(**changed):
    at = dict(k=0x1000, v=0x2000, k_scales=None, v_scales=None, pages=10, page_stride=8 * 16 * 128, head_stride=16 * 128, token_stride=128,
              format=binding.TORQ_FMT_BF16, heads=8, head_dim=128, page_size=16)
    at.update(changed)
    return binding._KVCacheStruct(*at.values())


BAD_CACHES = [dict(format=0), dict(format=3), dict(heads=0), dict(head_dim=0), dict(head_dim=12), dict(head_dim=264), dict(page_size=0), dict(page_size=8),
              dict(page_size=24), dict(page_size=1 << 17), dict(pages=-1), dict(pages=1 << 31), dict(page_stride=-8), dict(head_stride=4), dict(token_stride=12),
              dict(token_stride=1 << 26), dict(format=9, head_dim=72, k_scales=16, v_scales=16), dict(format=9, token_stride=8, k_scales=16, v_scales=16)]


@pytest.mark.parametrize("changed", BAD_CACHES, ids=str)
def test_caches_that_are_refused(changed):
    L, p = binding.lib(), C.c_void_p(0x1000)         # never dereferenced: every call below fails validation first
    bad = C.byref(cache_struct(**changed))
    assert L.torq_cache_append(bad, p, 128, 128, p, 128, 128, p, 4, None) == binding.TORQ_EINVAL
    assert L.torq_paged_attention(bad, p, 128, 128, 8, p, 4, 4, p, 2, 1.0, p, p, 1 << 30, None) == binding.TORQ_EINVAL
    assert L.torq_paged_attention_workspace_bytes(bad, 8, 2, 4) == 0


def test_attention_workspace_stays_within_its_documented_bound():
    need = binding.lib().torq_paged_attention_workspace_bytes
    sizes = [need(C.byref(cache_struct(heads=kv, head_dim=dim)), kv * group, B, width)
             for kv in (1, 3, 8, 20, 64) for dim in (8, 64, 72, 128, 136, 256) for group in (1, 2, 3, 16, 17, 32, 33, 71)
             for B in (0, 1, 5, 31, 32, 77, 300) for width in (0, 1, 32, 33, 64, 65, 999, 2000)]
    assert 0 < max(sizes) <= 66 << 20 and all(n % 16 == 0 for n in sizes)


def test_decode_calls_reject_bad_arguments_without_launching():
    L, p, odd, odd2 = binding.lib(), C.c_void_p(0x1000), C.c_void_p(0x1004), C.c_void_p(0x1002)
    E, A, OK = binding.TORQ_EINVAL, binding.TORQ_EALIGN, binding.TORQ_OK
    good = C.byref(cache_struct())
    mx = dict(format=9, k_scales=0x3000, v_scales=0x4000)

    def append(cache=good, key=p, kt=1024, kh=128, value=p, vt=1024, vh=128, slots=p, tokens=4):
        return L.torq_cache_append(cache, key, kt, kh, value, vt, vh, slots, tokens, None)
    assert [append(cache=None), append(key=None), append(value=None), append(slots=None), append(tokens=-1), append(kt=4), append(vh=-8)] == [E] * 7
    assert [append(cache=C.byref(cache_struct(k=None))), append(cache=C.byref(cache_struct(**dict(mx, v_scales=None))))] == [E] * 2
    assert [append(key=odd), append(value=odd), append(slots=odd), append(cache=C.byref(cache_struct(v=0x1008)))] == [A] * 4
    assert append(key=None, value=None, slots=None, tokens=0) == OK

    def attention(cache=good, q=p, qs=1024, qh=128, heads=32, tables=p, ts=4, width=4, lengths=p, B=2, scale=1.0, out=p, ws=p, n=1 << 30):
        return L.torq_paged_attention(cache, q, qs, qh, heads, tables, ts, width, lengths, B, scale, out, ws, n, None)
    assert [attention(cache=None), attention(q=None), attention(tables=None), attention(lengths=None), attention(out=None), attention(heads=0),
            attention(heads=12), attention(ts=3), attention(width=-1), attention(B=-1), attention(qs=4), attention(qh=-8),
            attention(scale=math.inf), attention(scale=math.nan), attention(width=1 << 27, ts=1 << 27), attention(B=1 << 40)] == [E] * 16
    assert [attention(q=odd), attention(out=odd), attention(ws=odd), attention(tables=odd2), attention(lengths=odd2)] == [A] * 5
    assert attention(B=0, q=None, tables=None, lengths=None, out=None, ws=None, n=0) == OK
    need = binding.lib().torq_paged_attention_workspace_bytes(good, 32, 2, 4000)
    assert need > 0
    assert attention(width=4000, ts=4000, n=need - 1) == binding.TORQ_EWORKSPACE and attention(width=4000, ts=4000, ws=None, n=0) == E

    def tables(held=p, lengths=p, B=2, free=p, n=9, cursor=p, after=p, table=p, ts=4, width=4, page=16, slots=p, tokens=3):
        return L.torq_block_tables(held, lengths, B, free, n, cursor, after, table, ts, width, page, slots, tokens, None)
    assert [tables(held=None), tables(lengths=None), tables(B=-1), tables(free=None), tables(n=-1), tables(cursor=None), tables(after=None),
            tables(table=None), tables(ts=3), tables(width=-1), tables(page=0), tables(slots=None), tables(tokens=-1)] == [E] * 13
    assert [tables(held=odd2), tables(lengths=odd2), tables(free=odd2), tables(cursor=odd2), tables(after=odd2), tables(table=odd2), tables(slots=odd)] == [A] * 7

    def norm(x=p, r=p, w=p, M=4, d=256, eps=1e-5, fmt=8, ro=p, out=p, scales=p):
        return L.torq_add_rms_norm(x, r, w, M, d, eps, fmt, ro, out, scales, None)
    assert [norm(x=None), norm(w=None), norm(out=None), norm(ro=None), norm(r=None), norm(M=-1), norm(d=0), norm(d=40), norm(d=32800),
            norm(eps=-1.0), norm(eps=math.nan), norm(eps=math.inf), norm(fmt=0), norm(fmt=10), norm(fmt=9, scales=None)] == [E] * 15
    assert [norm(x=odd), norm(r=odd), norm(w=odd), norm(ro=odd), norm(out=odd)] == [A] * 5
    assert norm(M=0, x=None, r=None, w=None, ro=None, out=None, scales=None) == OK
    # the 4-bit quantisers take none of these formats
    assert all(L.torq_quantize_f32_fmt(p, 4, 64, f, C.c_float(1.0), p, p, None) == E for f in (8, 9))


def test_kv_cache_refuses_what_does_not_fit():
    t = lambda *shape, dtype=BF: torch.empty(shape, dtype=dtype)
    k = t(4, 2, 16, 64)
    assert binding.KVCache(k, k.clone()).format == binding.TORQ_FMT_BF16
    f, s = t(4, 2, 16, 64, dtype=F8), t(4, 2, 16, 2, dtype=E8)
    assert binding.KVCache(f, f.clone(), s, s.clone()).format == binding.TORQ_FMT_MXFP8
    assert binding.KVCache(f, f.clone(), s.view(torch.uint8), s.view(torch.uint8)).page_size == 16
    one = t(1, 1, 16, 64)
    assert binding.KVCache(one, t(1, 16, 1, 64).transpose(1, 2)).heads == 1           # strides of dimensions of one entry say nothing
    for bad in [(k, t(4, 2, 16, 72)), (k, f), (k.half(), k.half()), (k[0], k[0]), (k, k, s, s), (f, f), (f, f, s, None), (f, f, s, t(4, 2, 16, 4, dtype=E8)),
                (k, t(4, 16, 2, 64).transpose(1, 2)), (t(4, 2, 64, 16).transpose(2, 3), t(4, 2, 64, 16).transpose(2, 3)),
                (f, f, s, t(4, 16, 2, 2, dtype=E8).transpose(1, 2)), (f, f, s, s.float())]:
        with pytest.raises(ValueError):
            binding.KVCache(*bad)
    with pytest.raises(ValueError):
        binding.KVCache.empty(2, 2, 16, 72, binding.TORQ_FMT_MXFP8, device="cpu")
    with pytest.raises(ValueError):
        binding.KVCache.empty(2, 2, 16, 64, binding.TORQ_FMT_NVFP4, device="cpu")


def test_decode_calls_refuse_host_tensors_and_wrong_shapes(either_way):
    k = torch.zeros((4, 2, 16, 64), dtype=BF)
    cache = binding.KVCache(k, k.clone())
    i = lambda *shape: torch.zeros(shape, dtype=torch.int32)
    x = torch.zeros((3, 2, 64), dtype=BF)
    slots = torch.zeros(3, dtype=torch.int64)
    for call in (lambda: binding.torq_block_tables(i(3), i(3), i(5), i(1), i(3, 4), 16, 3), lambda: binding.torq_block_tables(i(2), i(3), i(5), i(1), i(3, 4), 16, 3),
                 lambda: binding.torq_block_tables(i(3), i(3), i(5), i(2), i(3, 4), 16, 3), lambda: binding.torq_block_tables(i(3), i(3), i(5), i(1), i(3, 4), 16, 3, slots=slots[:2]),
                 lambda: binding.torq_cache_append(cache, x, x, slots), lambda: binding.torq_cache_append(cache, x, x[:, :1], slots),
                 lambda: binding.torq_cache_append(cache, x, x, slots[:2]),
                 lambda: binding.torq_paged_attention(x, cache, i(3, 2), i(3), 1.0, workspace=torch.zeros(1 << 20, dtype=torch.uint8)),
                 lambda: binding.torq_paged_attention(x, cache, i(2, 2), i(3), 1.0), lambda: binding.torq_paged_attention(x, cache, i(3, 2), i(2), 1.0),
                 lambda: binding.torq_paged_attention(x[:, :, :32], cache, i(3, 2), i(3), 1.0), lambda: binding.torq_paged_attention(x, cache, i(3, 2), i(3), 1.0, out=x[:2]),
                 lambda: binding.torq_add_rms_norm(x[0], None, x[0, 0], 1e-5), lambda: binding.torq_add_rms_norm(x[0], x[0, :1], x[0, 0], 1e-5),
                 lambda: binding.torq_add_rms_norm(x[0], None, x[0, 0, :32], 1e-5), lambda: binding.torq_add_rms_norm(x[0], None, x[0, 0], 1e-5, residual_out=x[0])):
        with pytest.raises(ValueError):
            call()
