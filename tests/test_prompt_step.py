"""Prompts in pieces, then single tokens, through two blocks (paper_2605_19561_amd/decode_step.py), over a cache in each format and scores by a rule: every
attention call is looked at with the inputs that it got, in 64 bits over keys and values kept in plain lists."""
import types

import pytest
import torch

from test_chunk_attention import Rule, check, few, mxfp4, seen_by, slopes_of, values4
from test_decode_ops import mxfp8

pytestmark = pytest.mark.gpu


def as_held(t, fmt):
    """What the cache holds of t, float64."""
    t = t.double().cpu()
    if fmt == "mxfp8":
        codes, scales = (torch.from_numpy(a) for a in mxfp8(t.numpy()))
        return codes.view(torch.float8_e4m3fn).double() * scales.view(torch.float8_e8m0fnu).double().repeat_interleave(32, -1)
    if fmt == "mxfp4":
        return values4(*(torch.from_numpy(a) for a in mxfp4(t.numpy())))
    return t


@pytest.mark.parametrize("rule", ["plain", "window", "slopes"])
@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
def test_prompts_and_single_tokens_of_two_blocks(fmt, rule, monkeypatch):
    from paper_2605_19561_amd import binding as tq, decode_step as ds, synth
    B, heads, kv, dim = 4, 8, 2, 128
    pieces = [[20, 0, 70, 1], [3, 40, 2, 5], [7, 1, 0, 8]]           # (of many rows, then of few)
    rule = {"plain": Rule(), "window": Rule(cap=4.0, window=24, prefix=torch.tensor([4, 0, 9, 2], dtype=torch.int32)), "slopes": Rule(slopes=slopes_of(heads))}[rule]
    pages = ds.Pages(B, 40, 16, 128)
    cache_of = lambda: tq.KVCache.empty(40, kv, 16, dim, getattr(tq, "TORQ_FMT_" + fmt.upper()))
    blocks = [ds.DecoderBlock(1024, heads, kv, dim, 2048, cache_of(), seed=100 * i) for i in range(2)]
    kept = {id(b.cache): [([], []) for _ in range(B)] for b in blocks}
    seen, now = {"chunk": 0, "single": 0}, None

    def append(cache, key, value, slots):
        tq.torq_cache_append(cache, key, value, slots)
        for t, which in ((key, 0), (value, 1)):
            t, at = as_held(t, fmt), 0
            for b, n in enumerate(now):
                kept[id(cache)][b][which].append(t[at:at + n])
                at += n

    def look(out, q, cache, scale, two_parts):
        at = 0
        for b, n in enumerate(now):
            k, v = (torch.cat(t).repeat_interleave(heads // kv, 1) for t in kept[id(cache)][b])                 # [tokens, heads, dim]
            p = len(k) - n + torch.arange(n)
            s = torch.einsum("qhd,thd->hqt", q[at:at + n].double().cpu(), k) * scale
            t = torch.arange(len(k))
            if rule.cap:
                s = rule.cap * torch.tanh(s / rule.cap)
            if rule.slopes is not None:
                s = s - rule.slopes.double()[:, None, None] * (p[:, None] - t).abs()
            s = torch.softmax(torch.where(seen_by(rule, b, p, t), s, -torch.inf), -1)
            check(out[at:at + n], torch.einsum("hqt,thd->qhd", s, v), torch.einsum("hqt,thd->qhd", s, v.abs()), two_parts)
            at += n

    def chunk(q, starts, cache, tables, lengths, scale, most, scores=None):
        out = tq.torq_chunk_attention(q, starts, cache, tables, lengths, scale, most=most, scores=scores)
        look(out, q, cache, scale, few(heads, kv, most))
        seen["chunk"] += 1
        return out

    def single(q, cache, tables, lengths, scale, scores=None):
        out = tq.torq_paged_attention(q, cache, tables, lengths, scale, scores=scores)
        look(out, q, cache, scale, True)
        seen["single"] += 1
        return out

    calls = {n: getattr(tq, n) for n in dir(tq) if n.startswith(("torq_", "TORQ_", "KVCache"))}
    monkeypatch.setattr(ds, "tq", types.SimpleNamespace(**dict(calls, torq_cache_append=append, torq_chunk_attention=chunk, torq_paged_attention=single)))
    scores = None if rule.cap == 0 and rule.slopes is None else rule.on(tq)
    total = torch.zeros(B, dtype=torch.long)
    for i, now in enumerate(pieces + [[1] * B] * 3):
        x = synth.activations(sum(now), 1024, outliers=4, outlier_scale=5.0, seed=i, device="cuda")
        if i < len(pieces):
            fresh = pages.admit(torch.tensor(now, dtype=torch.int32, device="cuda"), sum(now), max(now))
            assert fresh.positions.tolist() == [int(total[b]) + j for b, n in enumerate(now) for j in range(n)]
        else:
            pages.advance()
            fresh = None
        total += torch.tensor(now)
        state = (x, None)
        for block in blocks:
            state = block.step(*state, pages, fresh, scores)
        assert all(torch.isfinite(t.float()).all() for t in state)
    assert seen == {"chunk": 2 * len(pieces), "single": 6} and pages.lengths.tolist() == total.tolist()
