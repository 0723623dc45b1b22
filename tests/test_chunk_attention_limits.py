"""The sizes that torq_chunk_attention takes and refuses, and calls of sizes that only many requests or long tables have."""
import ctypes as C

import pytest
import torch

from paper_2605_19561_amd import binding
from test_chunk_attention import DEV, Rule, case, check, either_way, reference, tq, values_of   # noqa: F401

gpu = pytest.mark.gpu


def answer(heads, kv_heads, tokens, most, B, keys, page=16):
    """What the call says to such sizes, with a query that is not aligned (looked at behind the sizes), so that nothing runs."""
    L, p, odd = binding.lib(), C.c_void_p(0x1000), C.c_void_p(0x1004)
    cache = C.byref(binding._KVCacheStruct(0x1000, 0x2000, 0x3000, 0x4000, 10, kv_heads * page * 128, page * 128, 128, binding.TORQ_FMT_MXFP4, kv_heads, 128, page))
    width = keys // page
    return L.torq_chunk_attention(cache, odd, heads * 128, 128, heads, tokens, p, most, p, width, width, p, B, 1.0, None, p, p, 1 << 40, None)


TAKEN = [
    # heads, kv_heads, new tokens, of a request at most, requests, tokens that the tables hold
    (64, 8, 8192, 8192, 32, 131072), (64, 8, 8192, 8192, 16, 131072), (64, 8, 8192 + 31, 8192, 32, 65536), (64, 8, 4096, 4096, 64, 32768),
    (64, 8, 2048, 2048, 256, 32768), (32, 8, 1 << 20, 1 << 20, 1024, 1 << 20), (8, 8, 1 << 16, 33, 1 << 16, 1 << 30),
    # up to 32 rows: tiles of 32 tokens below 2^31
    (64, 8, 128, 4, 16368, 1 << 18), (64, 8, 128, 2, 65408, 1 << 17),
    # workgroups of 64 rows below 2^24
    (64, 64, (1 << 24) - 65, 33, 1, 64), (64, 64, 1 << 17, 33, 1 << 17, 64), (8, 8, 99, 1 << 24, 1 << 30, 16), (1, 1, 99, 2 ** 31 - 1, 5, 16)]
REFUSED = [
    (64, 8, 128, 4, 16369, 1 << 18), (64, 8, 128, 2, 65409, 1 << 17), (64, 8, 128, 4, 1 << 30, 1 << 18), (64, 64, (1 << 24) - 64, 33, 1, 64), (64, 64, 1 << 18, 33, 1 << 18, 64),
    (8, 8, 99, 33, (1 << 30) + 1, 16), (64, 8, 8192, 8192, 32, (1 << 30) + 16), (64, 1, 99, 1 << 26, 5, 16), (64, 8, 1 << 25, 99, 1, 64)]


@pytest.mark.parametrize("heads,kv_heads,tokens,most,B,keys", TAKEN)
def test_sizes_that_are_taken(heads, kv_heads, tokens, most, B, keys):
    assert answer(heads, kv_heads, tokens, most, B, keys) == binding.TORQ_EALIGN


@pytest.mark.parametrize("heads,kv_heads,tokens,most,B,keys", REFUSED)
def test_sizes_that_are_refused(heads, kv_heads, tokens, most, B, keys):
    assert answer(heads, kv_heads, tokens, most, B, keys) == binding.TORQ_EINVAL


@gpu
@pytest.mark.parametrize("fmt,dim", [("bf16", 128), ("mxfp4", 64), ("mxfp8", 256)])
def test_places_for_long_prompts_behind_long_tables(tq, fmt, dim):
    """32 requests that might bring 8192 tokens each over tables for 131072: what a batch is laid out for, not what it has."""
    fresh, lengths = [3, 0, 70, 1] * 8, [300, 20, 70, 45] * 8
    cache, q, starts, tables, lens, pages = case(tq, fresh, lengths, 64, 8, dim, 16, fmt, "heads", 51)
    want = reference(q, starts, values_of(cache, "k"), values_of(cache, "v"), tables, lens, 0.1, pages, Rule())
    wide = torch.full((32, 131072 // 16), -1, dtype=torch.int32)
    wide[:, :tables.shape[1]] = tables
    got = tq.torq_chunk_attention(q.to(DEV), starts.to(DEV), cache, wide.to(DEV), lens.to(DEV), 0.1, most=8192)
    check(got, *want, False)


def test_a_cap_that_fp32_does_not_hold_is_refused():
    """Not taken for 0, which is none."""
    for cap in (1e-46, 5e-324, 7e-46):               # (2^-150, half of fp32's least number, and what is below: 0 in fp32)
        with pytest.raises(ValueError):
            binding.Scores(cap=cap)
    assert binding.Scores(cap=1e-45).cap == 2.0 ** -149 and binding.Scores(cap=0.0).cap == 0.0 and binding.Scores(cap=1e30).cap > 0


@gpu
@pytest.mark.parametrize("fresh", [[1, 1], [3, 2], [20, 9], [70, 33]])
@pytest.mark.parametrize("cap", [2.0 ** -149, 1e-40, 1e-30])
def test_the_least_caps_weigh_all_keys_alike(tq, fresh, cap):
    cache, q, starts, tables, lens, pages = case(tq, fresh, [90, 100], 4, 2, 128, 16, "bf16", "heads", 52)
    for scale in (1.0, -1e30):
        rule = Rule(cap=cap)
        want = reference(q, starts, values_of(cache, "k"), values_of(cache, "v"), tables, lens, scale, pages, rule)
        got = tq.torq_chunk_attention(q.to(DEV), starts.to(DEV), cache, tables.to(DEV), lens.to(DEV), scale, most=max(fresh), scores=rule.on(tq))
        check(got, *want, 2 * max(fresh) <= 32)


@pytest.mark.parametrize("most", [1 << 31, (1 << 32) + 1, (1 << 32) + 40, -(1 << 32) + 3])
def test_a_most_that_is_no_int_of_the_library_is_refused(most):
    """Not taken for what is left of it in 32 bits."""
    t = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)
    cache = binding.KVCache(t, t.clone())
    with pytest.raises(ValueError):
        binding.torq_chunk_attention_workspace_bytes(cache, 4, 99, most, 2, 4000)


@gpu
def test_a_call_with_a_most_that_is_no_int_of_the_library_is_refused(tq, either_way):
    cache, q, starts, tables, lens, _ = case(tq, [3, 2], [30, 20], 4, 2, 64, 16, "mxfp4", "heads", 53)
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device=DEV)
    for most in (1 << 31, (1 << 32) + 1):
        with pytest.raises(ValueError):
            tq.torq_chunk_attention(q.to(DEV), starts.to(DEV), cache, tables.to(DEV), lens.to(DEV), 0.1, most=most, out=out)
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())


@gpu
@pytest.mark.parametrize("heads,kv_heads,dim,fresh,fmt", [(4, 2, 64, [1, 1], "bf16"), (8, 2, 128, [1, 1], "mxfp4"), (4, 2, 64, [3, 2], "mxfp8"), (4, 2, 128, [20, 9], "bf16"),
                                                          (4, 2, 96, [70, 33], "mxfp4"), (4, 2, 256, [70, 33], "bf16")])
@pytest.mark.parametrize("prefix,cap", [(0, 0.0), (77, 0.0), (0, 5.0)])
def test_slopes_of_any_finite_size(tq, heads, kv_heads, dim, fresh, fmt, prefix, cap):
    """Whose product with a distance fp32 does not hold: the nearest key, or the farthest, has all of the weight."""
    cache, q, starts, tables, lens, pages = case(tq, fresh, [90, 100], heads, kv_heads, dim, 16, fmt, "heads", 54)
    slopes = torch.tensor(([3.4e38, -3.4e38, 2.4e38, -1e38, 1e30, -1e36, 0.0, 1e-38])[:heads])
    rule = Rule(cap=cap, slopes=slopes, prefix=torch.full((2,), prefix, dtype=torch.int32))
    want = reference(q, starts, values_of(cache, "k"), values_of(cache, "v"), tables, lens, 0.1, pages, rule)
    got = tq.torq_chunk_attention(q.to(DEV), starts.to(DEV), cache, tables.to(DEV), lens.to(DEV), 0.1, most=max(fresh), scores=rule.on(tq))
    check(got, *want, heads // kv_heads * max(fresh) <= 32)


@gpu
@pytest.mark.parametrize("fmt", ["bf16", "mxfp4"])
def test_prompts_whose_rows_pass_4_gib(tq, fmt):
    """34 prompts of 8192 tokens at once: q and out of 4.6 GB each.  (The requests share their pages, each in an order of its own, and see 70 tokens.)"""
    B, n, heads, kv_heads, dim, page = 34, 8192, 64, 8, 128, 16
    cache = tq.KVCache.empty(n // page, kv_heads, page, dim, getattr(tq, "TORQ_FMT_" + fmt.upper()), device=DEV)
    g = torch.Generator(device=DEV).manual_seed(55)
    x = torch.randn((n, 2, kv_heads, dim), generator=g, device=DEV).to(torch.bfloat16)
    tq.torq_cache_append(cache, x[:, 0], x[:, 1], torch.arange(n, device=DEV))
    tables = torch.stack([torch.randperm(n // page, generator=g, device=DEV) for _ in range(B)]).int()
    q = torch.randn((B * n, heads, dim), generator=g, device=DEV, dtype=torch.bfloat16)
    starts, lens = torch.arange(B + 1, dtype=torch.int32, device=DEV) * n, torch.full((B,), n, dtype=torch.int32, device=DEV)
    rule = Rule(window=70)
    out = tq.torq_chunk_attention(q, starts, cache, tables, lens, 0.1, most=n, scores=rule.on(tq))
    assert q.numel() * 2 > 1 << 32
    k, v = values_of(cache, "k"), values_of(cache, "v")
    for b in (0, 15, 16, 31, 32, B - 1):
        rows = slice(b * n, (b + 1) * n)
        alone = tq.torq_chunk_attention(q[rows], starts[:2], cache, tables[b:b + 1], lens[:1], 0.1, most=n, scores=rule.on(tq))
        assert torch.equal(out[rows], alone)
        # its last rows, as the last of a request that has no others
        want = reference(q[rows][-3:].cpu(), torch.tensor([0, 3]), k, v, tables[b:b + 1].cpu(), lens[:1].cpu(), 0.1, n // page, rule)
        check(out[rows][-3:], *want, False)
