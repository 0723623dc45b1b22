"""A decoder block's decode step, and its step over prompts, from this library's calls, as a serving program would put them together: residual
norm -> rotated W4A4 linear layers -> pages and slots -> keys and values into the paged cache -> attention -> linear layers, without a word to the host.

    python -m paper_2605_19561_amd.decode_step [--batch 16] [--context 2000] [--cache mxfp8] [--prompt 512] [--window 1024] [--cap 30]

Random weights of a LLaMA3-8B block (hidden 4096, 32 query and 8 key heads of 128, ffn 14336); the rotary embedding and the gated
activation between the calls are torch's.
"""
import argparse
import collections
import time

import torch

from . import binding as tq
from . import synth


def rotary(x: torch.Tensor, positions: torch.Tensor, base: float = 500000.0) -> torch.Tensor:
    """x [B, heads, head_dim] turned by its position: halves (i, i + head_dim / 2) by position * base^(-2 i / head_dim)."""
    half = x.shape[-1] // 2
    angle = positions[:, None].float() * base ** (-torch.arange(half, device=x.device, dtype=torch.float32) / half)
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    a, b = x[..., :half].float(), x[..., half:].float()
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(x.dtype)


# The new tokens of a step that has several of a request: rows starts[b] ... starts[b + 1] - 1 are request b's, at these positions and slots; no request
# has more than `most`.
Fresh = collections.namedtuple("Fresh", "starts positions slots most")


class Pages:
    """The requests' side of a paged cache: which pages hold whose tokens, shared by all blocks of a model."""

    def __init__(self, batch: int, pages: int, page_size: int, most_tokens: int, device="cuda"):
        i32 = dict(dtype=torch.int32, device=device)
        self.page_size = page_size
        self.free, self.cursor = torch.arange(pages, **i32), torch.zeros(1, **i32)
        self.tables = torch.full((batch, -(-most_tokens // page_size)), -1, **i32)
        self.held, self.lengths = torch.zeros(batch, **i32), torch.zeros(batch, **i32)
        self.slots = torch.empty(batch, dtype=torch.int64, device=device)

    def advance(self):
        """One more token for every request: its page, and its slot."""
        self.held.copy_(self.lengths)
        self.lengths.add_(1)
        tq.torq_block_tables(self.held, self.lengths, self.free, self.cursor, self.tables, self.page_size, self.slots.numel(),
                             slots=self.slots, cursor_out=self.cursor)

    def admit(self, tokens: torch.Tensor, total: int, most: int) -> Fresh:
        """tokens[b] (int32, `total` in all or fewer, at most `most`) more for every request, a prompt or a piece of one: their pages and slots."""
        self.held.copy_(self.lengths)
        self.lengths.add_(tokens)
        slots, _ = tq.torq_block_tables(self.held, self.lengths, self.free, self.cursor, self.tables, self.page_size, total, cursor_out=self.cursor)
        ends = tokens.cumsum(0, dtype=torch.int32)
        starts = torch.cat([ends.new_zeros(1), ends])
        rows = torch.arange(total, dtype=torch.int32, device=tokens.device)
        b = torch.searchsorted(ends, rows, right=True).clamp_(max=len(ends) - 1)          # (rows behind the last token: of no request, without a slot)
        return Fresh(starts, self.held[b] + rows - starts[b], slots, most)


class DecoderBlock:
    """One block: two norms, four packed products (q, k and v as one, gate and up as one) and its part of the cache."""

    def __init__(self, hidden, heads, kv_heads, head_dim, ffn, cache: tq.KVCache, seed: int, device="cuda"):
        self.heads, self.kv_heads, self.head_dim, self.ffn, self.cache = heads, kv_heads, head_dim, ffn, cache
        widths = {"qkv": (hidden, (heads + 2 * kv_heads) * head_dim), "o": (heads * head_dim, hidden), "gate_up": (hidden, 2 * ffn), "down": (ffn, hidden)}
        rotations = {d: tq.Rotation(d, synth.default_G(d), *synth.rotations(synth.default_G(d), seed + d)) for d, _ in widths.values()}
        self.layers = {}
        for i, (name, (d, n)) in enumerate(widths.items()):
            w = synth.weights(n, d, std=d ** -0.5, seed=seed + 10 + i, device=device)
            self.layers[name] = (rotations[d], *tq.torq_rotate_quantize(rotations[d], w))
        g = torch.Generator(device=device).manual_seed(seed + 20)
        self.norms = [(1 + 0.1 * torch.randn(hidden, generator=g, device=device)).to(torch.bfloat16) for _ in range(2)]

    def linear(self, name, x):
        return tq.torq_linear(self.layers[name][0], x, *self.layers[name][1:])

    def step(self, x, residual, pages: Pages, fresh: Fresh = None, scores=None):
        """x and residual [B, hidden], or [tokens, hidden] with what `Pages.admit` gave: the block before's output and the sum ahead of it (None
        in the first block).  scores: the model's rule (Scores).  Returns both for the next block."""
        B, kv = x.shape[0], self.kv_heads
        if residual is None:
            y, _, _ = tq.torq_add_rms_norm(x, None, self.norms[0], 1e-5)
            residual = x
        else:
            y, _, residual = tq.torq_add_rms_norm(x, residual, self.norms[0], 1e-5)
        qkv = self.linear("qkv", y).view(B, self.heads + 2 * kv, self.head_dim)
        positions, slots = (pages.held, pages.slots) if fresh is None else (fresh.positions, fresh.slots)
        q = rotary(qkv[:, : self.heads], positions)
        k = rotary(qkv[:, self.heads : self.heads + kv], positions)
        tq.torq_cache_append(self.cache, k, qkv[:, self.heads + kv :], slots)
        rule, scale = {} if scores is None else {"scores": scores}, self.head_dim ** -0.5
        if fresh is None:
            a = tq.torq_paged_attention(q, self.cache, pages.tables, pages.lengths, scale, **rule)
        else:
            a = tq.torq_chunk_attention(q, fresh.starts, self.cache, pages.tables, pages.lengths, scale, most=fresh.most, **rule)
        x = self.linear("o", a.view(B, -1))
        y, _, residual = tq.torq_add_rms_norm(x, residual, self.norms[1], 1e-5)
        gate, up = self.linear("gate_up", y).chunk(2, -1)
        return self.linear("down", torch.nn.functional.silu(gate) * up), residual


def main():
    p = argparse.ArgumentParser()
    p.add_argument("--batch", type=int, default=16)
    p.add_argument("--context", type=int, default=2000)
    p.add_argument("--cache", choices=["bf16", "mxfp8", "mxfp4"], default="bf16")
    p.add_argument("--prompt", type=int, default=0, help="the last so many tokens of each request's context go through the block")
    p.add_argument("--window", type=int, default=0, help="tokens that a query sees (0: all)")
    p.add_argument("--cap", type=float, default=0.0, help="cap tanh(score / cap) (0: as they are)")
    a = p.parse_args()
    page, steps = 16, 50
    most = a.context + 2 * steps
    pages = Pages(a.batch, a.batch * -(-most // page), page, most)
    fmt = {"bf16": tq.TORQ_FMT_BF16, "mxfp8": tq.TORQ_FMT_MXFP8, "mxfp4": tq.TORQ_FMT_MXFP4}[a.cache]
    scores = tq.Scores(cap=a.cap, window=a.window) if a.cap or a.window else None
    cache = tq.KVCache.empty(pages.free.numel(), 8, page, 128, fmt)
    block = DecoderBlock(4096, 32, 8, 128, 14336, cache, seed=1)
    # a context of random keys and values, as a prefill would leave it
    behind = max(a.context - a.prompt, 0)
    pages.lengths.fill_(behind)
    tokens = a.batch * behind
    slots, _ = tq.torq_block_tables(pages.held, pages.lengths, pages.free, pages.cursor, pages.tables, page, tokens, cursor_out=pages.cursor)
    kv = torch.randn((tokens, 2, 8, 128), device="cuda").to(torch.bfloat16)
    tq.torq_cache_append(cache, kv[:, 0], kv[:, 1], slots)
    new = a.context - behind
    if new:
        fresh = pages.admit(torch.full((a.batch,), new, dtype=torch.int32, device="cuda"), a.batch * new, new)
        x = synth.activations(a.batch * new, 4096, outliers=8, outlier_scale=10.0, seed=2, device="cuda")
        for n in range(2):                           # (the second time the same tokens into the same slots)
            torch.cuda.synchronize()
            t = time.perf_counter()
            y, _ = block.step(x, None, pages, fresh, scores)
            torch.cuda.synchronize()
        print(f"{a.batch} prompts of {new} tokens behind {behind}: {(time.perf_counter() - t) * 1e6:.1f} us for one block")
    x = synth.activations(a.batch, 4096, outliers=8, outlier_scale=10.0, seed=3, device="cuda")
    for n in range(2 * steps):
        if n == steps:
            torch.cuda.synchronize()
            t = time.perf_counter()
        pages.advance()
        y, _ = block.step(x, None, pages, scores=scores)
    torch.cuda.synchronize()
    print(f"batch {a.batch}, {a.context} tokens in the {a.cache} cache: {(time.perf_counter() - t) / steps * 1e6:.1f} us a step of one block, "
          f"{int(pages.lengths[0])} tokens held, output finite: {bool(torch.isfinite(y.float()).all())}")


if __name__ == "__main__":
    main()
