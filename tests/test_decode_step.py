"""The decode step put together (paper_2605_19561_amd/decode_step.py): two blocks over several tokens.  Every call that the step makes is
looked at with the inputs that it got: norms and attention against 64 bits, the attention over keys and values kept in plain lists, so that
pages, slots and lengths have to be right for it to come out.  (Whole steps are not compared: the products round their inputs to 4 bits, and two
runs whose inputs differ in the last bit differ by codes.)"""
import types

import pytest
import torch

from test_decode_ops import check_attention, mxfp8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
def test_decode_steps_of_two_blocks(fmt, monkeypatch):
    from paper_2605_19561_amd import binding as tq, decode_step as ds, synth
    B, steps, heads, kv, dim = 5, 37, 8, 2, 128      # two page borders of 16
    pages = ds.Pages(B, B * 3 + 1, 16, 48)
    form = tq.TORQ_FMT_BF16 if fmt == "bf16" else tq.TORQ_FMT_MXFP8
    blocks = [ds.DecoderBlock(1024, heads, kv, dim, 2048, tq.KVCache.empty(B * 3 + 1, kv, 16, dim, form), seed=100 * i) for i in range(2)]
    kept = {id(b.cache): ([], []) for b in blocks}   # each step's keys and values [B, kv, dim], float64, as the cache should hold them
    seen = {"norm": 0, "append": 0, "attention": 0}

    def norm(x, residual, weight, eps, *args):
        out, scales, total = tq.torq_add_rms_norm(x, residual, weight, eps, *args)
        s = x.double() + (0 if residual is None else residual.double())
        y = s / (s.pow(2).mean(-1, keepdim=True) + eps).sqrt() * weight.double()
        assert ((out.double() - y).abs() <= (2.0 ** -8 + 2.0 ** -16) * y.abs()).all()
        assert total is None or ((total.double() - s).abs() <= (2.0 ** -8 + 2.0 ** -23) * s.abs()).all()
        seen["norm"] += 1
        return out, scales, total

    def append(cache, key, value, slots):
        tq.torq_cache_append(cache, key, value, slots)
        for t, held in zip((key, value), kept[id(cache)]):
            t = t.double().cpu()
            if fmt == "mxfp8":
                codes, scales = (torch.from_numpy(a) for a in mxfp8(t.numpy()))
                t = codes.view(torch.float8_e4m3fn).double() * scales.view(torch.float8_e8m0fnu).double().repeat_interleave(32, -1)
            held.append(t)
        seen["append"] += 1

    def attention(q, cache, tables, lengths, scale):
        out = tq.torq_paged_attention(q, cache, tables, lengths, scale)
        k, v = (torch.stack(t, 2).repeat_interleave(heads // kv, 1) for t in kept[id(cache)])                # [B, heads, tokens, dim]
        p = torch.softmax((k * q.double().cpu()[:, :, None]).sum(-1) * scale, -1)[..., None]
        check_attention(out, (p * v).sum(2), (p * v.abs()).sum(2))
        seen["attention"] += 1
        return out

    calls = {n: getattr(tq, n) for n in dir(tq) if n.startswith(("torq_", "TORQ_", "KVCache"))}
    monkeypatch.setattr(ds, "tq", types.SimpleNamespace(**dict(calls, torq_add_rms_norm=norm, torq_cache_append=append, torq_paged_attention=attention)))
    for n in range(steps):
        state = (synth.activations(B, 1024, outliers=4, outlier_scale=5.0, seed=n, device="cuda"), None)
        pages.advance()
        for block in blocks:
            state = block.step(*state, pages)
        assert all(torch.isfinite(t.float()).all() for t in state)
    assert seen == {"norm": 4 * steps, "append": 2 * steps, "attention": 2 * steps}
    assert pages.lengths.tolist() == [steps] * B and int(pages.cursor) == 3 * B
    assert sorted(pages.tables.flatten().tolist()) == list(range(3 * B))
