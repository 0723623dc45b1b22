"""Calls of the 4-bit cache, of scores by a rule and of attention of several new tokens as programs make them, and those that are refused."""
import ctypes as C
import math

import pytest
import torch

from paper_2605_19561_amd import binding
from test_chunk_attention import BF, DEV, E8, Rule, case, check, either_way, few, lengthened, make_cache, reference, rng, slopes_of, tq, values_of   # noqa: F401

gpu = pytest.mark.gpu
i32 = lambda *n: torch.tensor(n, dtype=torch.int32)


# ---- refusals, on the host ---------------------------------------------------------------------

def cache_struct(**changed):
    at = dict(k=0x1000, v=0x2000, k_scales=0x3000, v_scales=0x4000, pages=10, page_stride=8 * 16 * 128, head_stride=16 * 128, token_stride=128,
              format=binding.TORQ_FMT_MXFP4, heads=8, head_dim=128, page_size=16)
    at.update(changed)
    return binding._KVCacheStruct(*at.values())


def scores_struct(cap=0.0, window=0, slopes=None, prefix=None):
    return C.byref(binding._ScoresStruct(cap, window, slopes, prefix))


@pytest.mark.parametrize("changed", [dict(head_dim=72), dict(head_dim=16), dict(head_dim=288), dict(token_stride=72), dict(head_stride=16), dict(page_stride=-32),
                                     dict(format=1), dict(page_size=24), dict(pages=-1), dict(heads=0)], ids=str)
def test_four_bit_caches_that_are_refused(changed):
    L, p = binding.lib(), C.c_void_p(0x1000)         # never dereferenced: every call fails validation first
    bad = C.byref(cache_struct(**changed))
    E = binding.TORQ_EINVAL
    assert L.torq_cache_append(bad, p, 128, 128, p, 128, 128, p, 4, None) == E
    assert L.torq_paged_attention_scores(bad, p, 128, 128, 8, p, 4, 4, p, 2, 1.0, None, p, p, 1 << 30, None) == E
    assert L.torq_chunk_attention(bad, p, 128, 128, 8, 9, p, 5, p, 4, 4, p, 2, 1.0, None, p, p, 1 << 30, None) == E
    assert L.torq_chunk_attention_workspace_bytes(bad, 8, 9, 5, 2, 4) == 0


def test_calls_reject_bad_arguments_without_launching():
    L, p, odd, odd2 = binding.lib(), C.c_void_p(0x1000), C.c_void_p(0x1004), C.c_void_p(0x1002)
    E, A, OK = binding.TORQ_EINVAL, binding.TORQ_EALIGN, binding.TORQ_OK
    good = C.byref(cache_struct())
    bad_scores = [scores_struct(cap=-1.0), scores_struct(cap=math.nan), scores_struct(cap=2e30), scores_struct(cap=math.inf), scores_struct(window=-1)]
    misaligned = [scores_struct(slopes=0x1002), scores_struct(prefix=0x1001)]

    def scored(cache=good, q=p, qs=1024, qh=128, heads=32, tables=p, ts=4, width=4, lengths=p, B=2, scale=1.0, scores=None, out=p, ws=p, n=1 << 30):
        return L.torq_paged_attention_scores(cache, q, qs, qh, heads, tables, ts, width, lengths, B, scale, scores, out, ws, n, None)
    assert [scored(scores=s) for s in bad_scores] == [E] * 5 and [scored(scores=s) for s in misaligned] == [A] * 2
    assert [scored(cache=C.byref(cache_struct(k_scales=None))), scored(heads=12), scored(scale=math.nan), scored(ts=3)] == [E] * 4
    assert scored(cache=C.byref(cache_struct(v=0x2008))) == A
    assert scored(B=0, q=None, tables=None, lengths=None, out=None, ws=None, n=0) == OK

    def chunk(cache=good, q=p, qs=4096, qh=128, heads=32, tokens=50, starts=p, most=40, tables=p, ts=4, width=4, lengths=p, B=2, scale=1.0, scores=None, out=p,
              ws=p, n=1 << 30):
        return L.torq_chunk_attention(cache, q, qs, qh, heads, tokens, starts, most, tables, ts, width, lengths, B, scale, scores, out, ws, n, None)
    assert [chunk(cache=None), chunk(q=None), chunk(starts=None), chunk(tables=None), chunk(lengths=None), chunk(out=None), chunk(heads=0), chunk(heads=12),
            chunk(tokens=-1), chunk(most=0), chunk(most=-3), chunk(ts=3), chunk(width=-1), chunk(B=-1), chunk(qs=4), chunk(qh=-8), chunk(scale=math.inf),
            chunk(scale=math.nan), chunk(width=1 << 27, ts=1 << 27), chunk(B=1 << 40), chunk(tokens=1 << 27), chunk(most=1 << 30),
            chunk(tokens=1 << 25, heads=48, B=1 << 22), chunk(cache=C.byref(cache_struct(v_scales=None)))] == [E] * 24
    assert [chunk(scores=s) for s in bad_scores] == [E] * 5 and [chunk(scores=s) for s in misaligned] == [A] * 2
    assert [chunk(q=odd), chunk(out=odd), chunk(ws=odd), chunk(tables=odd2), chunk(lengths=odd2), chunk(starts=odd2)] == [A] * 6
    assert chunk(B=0, q=None, starts=None, tables=None, lengths=None, out=None, ws=None, n=0) == OK
    assert chunk(tokens=0, q=None, starts=None, tables=None, lengths=None, out=None, ws=None, n=0) == OK
    for most in (1, 5, 40, 300):                     # each kind of kernel
        need = L.torq_chunk_attention_workspace_bytes(good, 32, 50, most, 2, 4000)
        assert need > 0 and need % 16 == 0
        assert chunk(most=most, width=4000, ts=4000, n=need - 1) == binding.TORQ_EWORKSPACE and chunk(most=most, width=4000, ts=4000, ws=None, n=0) == E


def test_scores_that_are_refused():
    S = binding.Scores
    x = torch.ones(8)
    for bad in (dict(cap=-1.0), dict(cap=math.nan), dict(cap=2e30), dict(window=-1), dict(window=1 << 31), dict(slopes=x.double()), dict(slopes=x[None]), dict(slopes=x[::2]),
                dict(prefix=x), dict(prefix=torch.zeros(8, dtype=torch.int64))):
        with pytest.raises(ValueError):
            S(**bad)
    s = S(cap=30.0, window=7, slopes=x, prefix=i32(1, 2))
    assert (s.cap, s.window) == (30.0, 7) and s.slopes is x and s.prefix.tolist() == [1, 2]
    s.check(8, 2, x.device)
    for heads, B in ((9, 2), (8, 3)):
        with pytest.raises(ValueError):
            s.check(heads, B, x.device)
    with pytest.raises(ValueError):
        s.check(8, 2, torch.device("cuda:0"))


def test_python_calls_refuse_host_tensors_and_wrong_shapes(either_way):
    t = torch.zeros((4, 2, 16, 32), dtype=torch.uint8)
    s = torch.zeros((4, 2, 16, 2), dtype=torch.uint8)
    cache = binding.KVCache(t, t.clone(), s.view(E8), s.clone().view(E8))
    assert cache.format == binding.TORQ_FMT_MXFP4 and cache.head_dim == 64 and cache.heads == 2 and cache.page_size == 16
    for bad in ((t, t), (t, t, s.view(E8), None), (t, t, s[..., :1].contiguous(), s[..., :1].contiguous()), (t[..., :24].contiguous(),) * 2 + (s.view(E8),) * 2):
        with pytest.raises(ValueError):
            binding.KVCache(*bad)
    with pytest.raises(ValueError):
        binding.KVCache.empty(2, 2, 16, 72, binding.TORQ_FMT_MXFP4, device="cpu")
    i = lambda *n: torch.zeros(n, dtype=torch.int32)
    x = torch.zeros((3, 2, 64), dtype=BF)
    for call in (lambda: binding.torq_cache_append(cache, x, x, torch.zeros(3, dtype=torch.int64)),
                 lambda: binding.torq_paged_attention(x, cache, i(3, 2), i(3), 1.0, scores=binding.Scores(cap=1.0)),
                 lambda: binding.torq_paged_attention(x, cache, i(3, 2), i(3), 1.0, scores=30.0),
                 lambda: binding.torq_chunk_attention(x, i(2), cache, i(1, 2), i(1), 1.0), lambda: binding.torq_chunk_attention(x, i(3), cache, i(1, 2), i(1), 1.0),
                 lambda: binding.torq_chunk_attention(x, i(2), cache, i(2, 2), i(1), 1.0), lambda: binding.torq_chunk_attention(x[..., :32], i(2), cache, i(1, 2), i(1), 1.0),
                 lambda: binding.torq_chunk_attention(x, i(2), cache, i(1, 2), i(1), 1.0, out=x[:2])):
        with pytest.raises(ValueError):
            call()


@gpu
def test_python_calls_refuse_what_does_not_go_together(tq, either_way):
    cache, q, starts, tables, lens, _ = case(tq, [3, 2], [30, 20], 4, 2, 64, 16, "mxfp4", "heads", 21)
    q, starts, tables, lens = q.to(DEV), starts.to(DEV), tables.to(DEV), lens.to(DEV)
    x = torch.ones(4, device=DEV)
    chunk = lambda **kw: tq.torq_chunk_attention(*[kw.get(n, v) for n, v in (("q", q), ("starts", starts), ("cache", cache), ("tables", tables), ("lens", lens), ("scale", 0.1))],
                                                 **{n: v for n, v in kw.items() if n not in ("q", "starts", "cache", "tables", "lens", "scale")})
    for bad in (dict(scores=tq.Scores(slopes=x[:3])), dict(scores=tq.Scores(slopes=x.cpu())), dict(scores=tq.Scores(prefix=i32(1, 2, 3).to(DEV))), dict(scores=2.0),
                dict(starts=starts.long()), dict(starts=starts[:2]), dict(q=q.float()), dict(q=q[..., :32]), dict(lens=lens.cpu()), dict(out=q[:2].clone()),
                dict(out=q.float()), dict(tables=tables.long())):
        with pytest.raises(ValueError):
            chunk(**bad)
    for bad in (dict(most=0), dict(scale=math.inf), dict(most=40, tables=tables.repeat(1, 900), workspace=torch.empty(16, dtype=torch.uint8, device=DEV))):
        with pytest.raises((ValueError, RuntimeError)):
            chunk(**bad)
    with pytest.raises(ValueError):
        tq.torq_paged_attention(q[:2], cache, tables, lens, 0.1, scores=tq.Scores(slopes=x[:3]))


# ---- what tables, lengths and starts may hold ---------------------------------------------------

# heads, kv_heads, head_dim, new tokens, tokens, format: few rows, 64, 128 and 256 of them to a workgroup
KINDS = [(4, 2, 64, [2, 5], [70, 40], "mxfp4"), (8, 2, 128, [16, 9], [100, 40], "bf16"), (8, 2, 128, [30, 25], [300, 70], "mxfp8"), (8, 2, 96, [70, 33], [90, 60], "mxfp4")]
kinds = pytest.mark.parametrize("heads,kv_heads,dim,fresh,lengths,fmt", KINDS)
long = pytest.mark.parametrize("long", [False, True])


@gpu
@long
@kinds
def test_tokens_of_no_page_are_left_out(tq, heads, kv_heads, dim, fresh, lengths, fmt, long):
    cache, q, starts, tables, lens, pages = case(tq, fresh, lengths, heads, kv_heads, dim, 16, fmt, "heads", 31)
    tables[0, 1], tables[1, 0] = -1, pages + 3
    if long:
        tables = lengthened(tables, 16, max(fresh))
    for rule in (Rule(), Rule(window=20), Rule(prefix=i32(17, 40)), Rule(slopes=slopes_of(heads))):
        want = reference(q, starts, values_of(cache, "k"), values_of(cache, "v"), tables, lens, 0.1, pages, rule)
        got = tq.torq_chunk_attention(q.to(DEV), starts.to(DEV), cache, tables.to(DEV), lens.to(DEV), 0.1, most=max(fresh), scores=rule.on(tq))
        check(got, *want, few(heads, kv_heads, max(fresh)))


@gpu
@long
@kinds
def test_any_lengths_starts_and_most(tq, heads, kv_heads, dim, fresh, lengths, fmt, long):
    cache, q, starts, tables, lens, pages = case(tq, fresh, lengths, heads, kv_heads, dim, 16, fmt, "heads", 32, gap=4)
    if long:
        tables = lengthened(tables, 16, max(fresh))
    k, v = values_of(cache, "k"), values_of(cache, "v")
    T, room = len(q), tables.shape[1] * 16

    def run(starts, lens, most):
        out = torch.full(q.shape, 7.0, dtype=BF, device=DEV)
        tq.torq_chunk_attention(q.to(DEV), starts.to(DEV), cache, tables.to(DEV), lens.to(DEV), 0.1, most=most, out=out)
        return out.cpu()
    # requests without tokens, whose rows are zeros, whatever their number says
    for n in (0, -5, -2 ** 31):
        out = run(starts, i32(n, lengths[1]), max(fresh))
        assert bool((out[:fresh[0]] == 0).all()) and bool((out[T - 4:] == 7.0).all())
        check(out[fresh[0]:T - 4], *[x[fresh[0]:T - 4] for x in reference(q, starts, k, v, tables, lens, 0.1, pages, Rule())], few(heads, kv_heads, max(fresh)))
    # more tokens than rows of the tables: the last pages are none, those before count
    far = i32(room + 1000, lengths[1])
    check(run(starts, far, max(fresh)), *reference(q, starts, k, v, tables, far, 0.1, pages, Rule()), few(heads, kv_heads, max(fresh)))
    # ends past the rows, beginnings ahead of them
    wide = i32(-9, fresh[0], T + 100)
    inside = i32(0, fresh[0], T)
    want = reference(q, inside, k, v, tables, lens, 0.1, pages, Rule())
    check(run(wide, lens, T), *want, few(heads, kv_heads, T))
    # fewer computed than there are
    most = max(fresh) - 1
    out, (want, weight) = run(starts, lens, most), reference(q, starts, k, v, tables, lens, 0.1, pages, Rule())
    for b in range(2):
        begin, end = int(starts[b]), int(starts[b + 1])
        done = min(begin + most, end)
        check(out[begin:done], want[begin:done], weight[begin:done], few(heads, kv_heads, most))
        assert bool((out[done:end] == 7.0).all())


@gpu
@kinds
def test_views_of_q_and_empty_calls(tq, either_way, heads, kv_heads, dim, fresh, lengths, fmt):
    cache, q, starts, tables, lens, pages = case(tq, fresh, lengths, heads, kv_heads, dim, 16, fmt, "pairs", 33)
    want = tq.torq_chunk_attention(q.to(DEV), starts.to(DEV), cache, tables.to(DEV), lens.to(DEV), -0.1)
    check(want, *reference(q, starts, values_of(cache, "k"), values_of(cache, "v"), tables, lens, -0.1, pages, Rule()), few(heads, kv_heads, len(q)))
    wide = torch.full((len(q), heads + 3, dim + 8), 9.0, dtype=BF, device=DEV)
    wide[:, 1:heads + 1, :dim] = q.to(DEV)
    turned = torch.empty((heads, len(q), dim), dtype=BF, device=DEV).transpose(0, 1)
    turned.copy_(q.to(DEV))
    two = torch.full((2, tables.shape[1] + 3), 99, dtype=torch.int32, device=DEV)
    two[:, :tables.shape[1]] = tables.to(DEV)
    for view in (wide[:, 1:heads + 1, :dim], turned):
        got = tq.torq_chunk_attention(view, starts.to(DEV), cache, two[:, :tables.shape[1]], lens.to(DEV), -0.1)
        assert torch.equal(got, want)
    none = tq.torq_chunk_attention(q[:0].to(DEV), starts.to(DEV) * 0, cache, tables.to(DEV), lens.to(DEV), 0.1)
    assert none.shape == (0, heads, dim)
    none = tq.torq_chunk_attention(q[:2].to(DEV), starts[:1].to(DEV), cache, tables[:0].to(DEV), lens[:0].to(DEV), 0.1, out=want[:2].clone())
    assert torch.equal(none, want[:2])


# ---- streams, graphs, bits ----------------------------------------------------------------------

@gpu
@long
@kinds
def test_the_same_bits_on_any_stream_and_in_a_graph(tq, heads, kv_heads, dim, fresh, lengths, fmt, long):
    cache, q, starts, tables, lens, pages = case(tq, fresh, lengths, heads, kv_heads, dim, 16, fmt, "heads", 34)
    if long:
        tables = lengthened(tables, 16, max(fresh))
    q, starts, tables, lens = q.to(DEV), starts.to(DEV), tables.to(DEV), lens.to(DEV)
    rule = tq.Scores(slopes=slopes_of(heads).to(DEV), window=50, prefix=i32(5, 9).to(DEV))
    most, need = max(fresh), tq.torq_chunk_attention_workspace_bytes(cache, heads, len(q), max(fresh), 2, tables.shape[1])
    ws, outs = torch.empty(need + 16, dtype=torch.uint8, device=DEV), [torch.empty_like(q) for _ in range(2)]
    calls = [lambda **kw: tq.torq_chunk_attention(q, starts, cache, tables, lens, 0.1, most=most, scores=rule, **kw),
             lambda **kw: tq.torq_chunk_attention(q, starts, cache, tables, lens, 0.2, most=most, **kw)]
    want = [c() for c in calls]
    for _ in range(3):
        assert all(torch.equal(c(), w) for c, w in zip(calls, want))
    # two streams at once, each with a workspace of its call's own
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [c(stream=s) for _ in range(4) for c, s in zip(calls, streams)]
    for g, s in zip(got, streams * 4):
        g.record_stream(s)
        s.synchronize()
    assert all(torch.equal(g, want[i % 2]) for i, g in enumerate(got))
    # two graphs that share a workspace, replayed by turns, with other work between; what the tensors hold changes
    graphs = []
    for c, out in zip(calls, outs):
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c(out=out, workspace=ws)
        graphs.append(graph)
    for turn in range(4):
        rule.prefix[0] = 3 * turn
        lens[1] = lengths[1] - turn
        ws.fill_(0xA5)
        fresh_want = [c() for c in calls]
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, fresh_want))
        (q.float() @ q.float().transpose(1, 2)).sum().item()


@gpu
@long
@pytest.mark.parametrize("slopes", [False, True])
@pytest.mark.parametrize("dim,kv_heads,fmt", [(64, 8, "bf16"), (96, 4, "bf16"), (128, 8, "bf16"), (256, 2, "bf16"), (128, 8, "mxfp8"), (128, 8, "mxfp4")])
def test_many_ragged_prompts_give_the_same_bits_every_time(tq, dim, kv_heads, fmt, slopes, long):
    """Workgroups that follow one another on a CU while the loads of the ones before may still be on their way."""
    g = rng(dim, kv_heads, fmt, 37)
    fresh = torch.randint(1, 500, (33,), generator=g).tolist()
    cache, q, starts, tables, lens, pages = case(tq, fresh, fresh, 16 * kv_heads, kv_heads, dim, 16, fmt, "tokens", 38)
    if long:
        tables = lengthened(tables, 16, max(fresh))
    rule = tq.Scores(slopes=slopes_of(16 * kv_heads).to(DEV)) if slopes else None
    q, starts, tables, lens = q.to(DEV), starts.to(DEV), tables.to(DEV), lens.to(DEV)
    run = lambda: tq.torq_chunk_attention(q, starts, cache, tables, lens, 0.1, most=max(fresh), scores=rule)
    want = run()
    for _ in range(40):
        assert torch.equal(run(), want)
    # a request alone, whose workgroups follow no other's
    for b in (0, 17):
        at = slice(int(starts[b]), int(starts[b + 1]))
        alone = tq.torq_chunk_attention(q[at], starts[b:b + 2] - starts[b], cache, tables[b:b + 1], lens[b:b + 1], 0.1, most=max(fresh), scores=rule)
        assert float((alone.float() - want[at].float()).abs().max()) <= 2.0 ** -6 * float(want[at].float().abs().max())


@gpu
def test_single_tokens_with_scores_in_a_graph(tq):
    cache, q, starts, tables, lens, pages = case(tq, [1] * 5, [300, 1, 0, 77, 40], 8, 2, 128, 16, "mxfp4", "heads", 35)
    q, tables, lens = q.to(DEV), tables.to(DEV), lens.to(DEV)
    rule = tq.Scores(cap=2.0, window=64, prefix=torch.full((5,), 4, dtype=torch.int32, device=DEV))
    ws, out = torch.empty(tq.torq_paged_attention_workspace_bytes(cache, 8, 5, tables.shape[1]) + 16, dtype=torch.uint8, device=DEV), torch.empty_like(q)
    step = lambda **kw: tq.torq_paged_attention(q, cache, tables, lens, 0.1, scores=rule, **kw)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out=out, workspace=ws)
    for turn in range(4):
        lens[0] = 300 - 50 * turn
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    check(out, *reference(q.cpu(), torch.arange(6), values_of(cache, "k"), values_of(cache, "v"), tables.cpu(), lens.cpu(), 0.1, pages,
                          Rule(cap=2.0, window=64, prefix=torch.full((5,), 4, dtype=torch.int32))), True)


@gpu
@pytest.mark.parametrize("fmt,fresh,wide", [("mxfp4", 1, False), ("mxfp4", 3, False), ("mxfp4", 90, False), ("mxfp4", 90, True), ("bf16", 90, True), ("mxfp8", 90, False)])
def test_a_cache_beyond_4_gib(tq, fmt, fresh, wide):
    """Pages on both sides of every 4 GiB of elements and at the end."""
    heads, dim, page = 8, 128, 64
    each = heads * page * dim * {"bf16": 16, "mxfp8": 8, "mxfp4": 4}[fmt] // 8
    pages = (9 << 30) // each + 5
    cache = tq.KVCache.empty(pages, heads, page, dim, getattr(tq, "TORQ_FMT_" + fmt.upper()), device=DEV)
    used = [pages - 1, (4 << 30) // each - 1, (4 << 30) // each, 0, (8 << 30) // each, (8 << 30) // each + 1]
    n = len(used) * page - 5
    g = rng(fmt, fresh, 36)
    x = torch.randn((n, 2, heads, dim), generator=g).to(BF)
    slots = torch.tensor([used[p // page] * page + p % page for p in range(n)])
    tq.torq_cache_append(cache, x[:, 0].to(DEV), x[:, 1].to(DEV), slots.to(DEV))
    # the same tokens in a small cache
    small = make_cache(tq, len(used), heads, page, dim, fmt, "heads")
    tq.torq_cache_append(small, x[:, 0].to(DEV), x[:, 1].to(DEV), torch.arange(n, device=DEV))
    q = torch.randn((fresh, 2 * heads, dim), generator=g).to(BF)
    tables, near, lens, starts = i32(*used)[None], torch.arange(len(used), dtype=torch.int32)[None], i32(n), i32(0, fresh)
    if wide:
        tables, near = lengthened(tables, page, fresh), lengthened(near, page, fresh)
    rule = tq.Scores(slopes=slopes_of(2 * heads).to(DEV))
    for scores in (None, rule):
        got, want = [tq.torq_chunk_attention(q.to(DEV), starts.to(DEV), c, t.to(DEV), lens.to(DEV), 0.1, scores=scores) for c, t in ((cache, tables), (small, near))]
        assert torch.equal(got, want)
    check(tq.torq_chunk_attention(q.to(DEV), starts.to(DEV), cache, tables.to(DEV), lens.to(DEV), 0.1),
          *reference(q, starts, values_of(small, "k"), values_of(small, "v"), near, lens, 0.1, len(used), Rule()), few(2 * heads, heads, fresh))
