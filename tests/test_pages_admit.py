"""decode_step.Pages.admit with a bound on the new tokens that is larger than what there are, as torq_block_tables takes it."""
import pytest
import torch

from paper_2605_19561_amd import binding, decode_step


def plain_tables(held, lengths, free, cursor, tables, page, tokens, slots=None, cursor_out=None):
    """torq_block_tables on the host, token by token."""
    slots = torch.full((tokens,), -1, dtype=torch.int64) if slots is None else slots
    at, taken = 0, int(cursor)
    for b, (h, n) in enumerate(zip(held.tolist(), lengths.tolist())):
        for p in range(h, n):
            if p % page == 0:
                tables[b, p // page] = free[taken]
                taken += 1
            if at < tokens:
                slots[at] = int(tables[b, p // page]) * page + p % page
            at += 1
    cursor_out.fill_(taken)
    return slots, cursor_out


def admitted(pages, tokens, total):
    fresh = pages.admit(tokens, total, most=total)
    positions, starts = fresh.positions.tolist(), fresh.starts.tolist()
    held = pages.held.tolist()
    assert starts == [0] + tokens.cumsum(0).tolist() and len(positions) == total == len(fresh.slots)
    for b, n in enumerate(tokens.tolist()):
        assert positions[starts[b]:starts[b + 1]] == list(range(held[b], held[b] + n))
    assert (fresh.slots[:starts[-1]] >= 0).all() and (fresh.slots[starts[-1]:] == -1).all()
    return fresh


@pytest.mark.parametrize("more", [0, 1, 9])
def test_rows_behind_the_last_token_on_the_host(monkeypatch, more):
    monkeypatch.setattr(decode_step.tq, "torq_block_tables", plain_tables)
    pages = decode_step.Pages(3, 20, 16, 64, device="cpu")
    for tokens in ([5, 0, 20], [1, 17, 0], [0, 0, 0]):
        tokens = torch.tensor(tokens, dtype=torch.int32)
        admitted(pages, tokens, int(tokens.sum()) + more)


@pytest.mark.gpu
def test_rows_behind_the_last_token_take_no_part():
    tq = binding
    pages = decode_step.Pages(3, 20, 16, 64)
    block = decode_step.DecoderBlock(512, 8, 2, 64, 1024, tq.KVCache.empty(20, 2, 16, 64), seed=7)
    x = torch.randn((34, 512), generator=torch.Generator().manual_seed(8)).to(torch.bfloat16).cuda()
    fresh = admitted(pages, torch.tensor([5, 0, 20], dtype=torch.int32, device="cuda"), 34)
    got, _ = block.step(x, None, pages, fresh)
    # the same rows with none behind them
    alone = decode_step.Fresh(fresh.starts, fresh.positions[:25], fresh.slots[:25], fresh.most)
    want, _ = block.step(x[:25], None, pages, alone)
    assert torch.equal(got[:25], want)
