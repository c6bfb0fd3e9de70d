"""One decoder block around a paged MoE layer, as a serving loop runs it.

A step takes any mix of tokens: one new token of each decoding sequence, or a
prompt's tokens in a row (each attends to the cache up to itself, so a chunk is
written first and read afterwards). Per step:

    z  = x + residual;  8-bit rows of norm(z)      rms_norm
    q, k, v                                        Linear8
    k, v -> the sequences' blocks                  KVCache.append
    o  = attention over them                       KVCache.attend
    z  = z + o Wo;  16-bit rows h of norm(z)       (a plain product), rms_norm
    experts of h, and their order                  (a plain product), route_grouped
    y  = experts(h)                                PagedLayer.forward

A sequence's tokens lie in the blocks that its row of the block table names;
BlockTables hands blocks out and fills a step's arguments.

    python -m paper_2607_16184_amd.decoder --layer tiny --batch 16 --prompt 100 --steps 32
"""
from __future__ import annotations

import argparse
from typing import Sequence, Tuple

import numpy as np
import torch

from . import ops, synth
from .layer import PagedLayer


class BlockTables:
    """Which blocks hold which sequence, on the host."""

    def __init__(self, n_blocks: int, block_tokens: int, sequences: int, max_len: int):
        self.P, self.max_len = block_tokens, max_len
        self.free = list(range(n_blocks - 1, -1, -1))
        self.table = np.full((sequences, -(-max_len // block_tokens)), -1, dtype=np.int32)
        self.length = np.zeros(sequences, dtype=np.int64)

    def _new_blocks(self, sequence: int, tokens: int) -> range:
        """The table columns that so many more tokens need, refused where they
        cannot be had; nothing is changed."""
        if not 0 <= sequence < len(self.length):
            raise ValueError("there is no sequence %d" % sequence)
        if tokens < 0:
            raise ValueError("sequence %d: %d tokens" % (sequence, tokens))
        first, last = int(self.length[sequence]), int(self.length[sequence]) + tokens
        if last > self.max_len:
            raise ValueError("sequence %d would pass %d tokens" % (sequence, self.max_len))
        return range(-(-first // self.P), -(-last // self.P))

    def extend(self, sequence: int, tokens: int) -> np.ndarray:
        """The slots of the sequence's next tokens."""
        new = self._new_blocks(sequence, tokens)
        if len(new) > len(self.free):
            raise MemoryError("no block is free")
        first, last = int(self.length[sequence]), int(self.length[sequence]) + tokens
        for i in new:
            self.table[sequence, i] = self.free.pop()
        self.length[sequence] = last
        pos = np.arange(first, last)
        return self.table[sequence, pos // self.P].astype(np.int64) * self.P + pos % self.P

    def release(self, sequence: int):
        row = self.table[sequence]
        self.free.extend(int(b) for b in row[row >= 0][::-1])
        row[:] = -1
        self.length[sequence] = 0

    def step(self, sequences: Sequence[int], tokens: Sequence[int], device="cuda"):
        """(block_table, lens, slots) of a step that gives each listed sequence
        so many new tokens, a row per token. A step that is refused changes
        nothing."""
        if len(set(sequences)) < len(sequences):
            raise ValueError("a sequence is listed once, with all its new tokens")
        if len(tokens) != len(sequences):
            raise ValueError("%d counts of tokens for %d sequences" % (len(tokens), len(sequences)))
        need = sum(len(self._new_blocks(s, n)) for s, n in zip(sequences, tokens))
        if need > len(self.free):
            raise MemoryError("%d blocks are needed, %d are free" % (need, len(self.free)))
        slots = [self.extend(s, n) for s, n in zip(sequences, tokens)]
        rows = np.repeat(np.asarray(sequences, dtype=np.int64), tokens)
        lens = np.concatenate([np.arange(self.length[s] - n, self.length[s]) + 1 for s, n in zip(sequences, tokens)])
        return (torch.from_numpy(self.table[rows]).to(device), torch.from_numpy(lens.astype(np.int32)).to(device),
                torch.from_numpy(np.concatenate(slots)).to(device))


class DecoderBlock:
    """Attention and paged experts between two norms. ``w_qkv`` is [(heads + 2
    kv_heads) head_dim, H] e4m3 with its block scales; w_o [H, heads head_dim],
    w_router [E, H] and the norms' weights [H] (or None) are 16-bit. ``rotate``,
    if given, gets (qkv [T, heads + 2 kv_heads, head_dim], lens) and turns the
    queries and keys in it by their positions, in place."""

    def __init__(self, layer: PagedLayer, cache: ops.KVCache, heads: int, w_qkv: torch.Tensor, qkv_scale: torch.Tensor,
                 w_o: torch.Tensor, w_router: torch.Tensor, norm_attn: torch.Tensor = None, norm_moe: torch.Tensor = None,
                 eps: float = 1e-5, rotate=None, K: int = None, **routing):
        self.layer, self.cache, self.heads, self.eps, self.rotate = layer, cache, heads, eps, rotate
        self.qkv = ops.Linear8(w_qkv, qkv_scale)
        if w_qkv.shape != ((heads + 2 * cache.kv_heads) * cache.head_dim, layer.cfg.H):
            raise ValueError("w_qkv is not [(heads + 2 kv_heads) head_dim, H]")
        self.w_o, self.w_router = w_o.t().contiguous(), w_router.t().contiguous()
        self.norm_attn, self.norm_moe = norm_attn, norm_moe
        self.K, self.routing = K or layer.cfg.K, dict(n_shared=layer.cfg.n_shared, **routing)

    def step(self, x: torch.Tensor, residual: torch.Tensor, block_table: torch.Tensor, lens: torch.Tensor, slots: torch.Tensor,
             max_len: int) -> Tuple[torch.Tensor, torch.Tensor]:
        """(y, residual) of the block for x [T, H] and the residual so far (None
        at first): the next block's x and residual."""
        T, act, cache = x.shape[0], x.dtype, self.cache
        z, _, q8, qs = ops.rms_norm(x, self.norm_attn, residual, eps=self.eps, y16=False, y8=True)
        qkv = self.qkv.forward(q8, qs, dtype=act).view(T, -1, cache.head_dim)
        if self.rotate is not None:
            self.rotate(qkv, lens)
        q, k, v = qkv.split([self.heads, cache.kv_heads, cache.kv_heads], dim=1)
        cache.append(k, v, slots)
        o = cache.attend(q, block_table, lens, max_len)
        z, h, _, _ = ops.rms_norm(o.view(T, -1) @ self.w_o, self.norm_moe, x if z is None else z, eps=self.eps)
        routing = ops.route_grouped(h @ self.w_router, self.K, **self.routing)
        return self.layer.forward(h, routing).view(act), z


def random_block(name: str, n_blocks: int, block_tokens: int = 32, fp8_cache: bool = False, seed: int = 0, device="cuda",
                 **routing) -> DecoderBlock:
    """A block around the named synthetic layer, its other weights drawn so that
    activations keep their size: heads of 128 (64 below 1024 hidden), eight
    of them per key head."""
    cfg = synth.CONFIGS[name]
    act = torch.float16 if cfg.act == synth.F16 else torch.bfloat16
    bits = synth.bitmap(cfg)
    layer = PagedLayer(cfg, PagedLayer.pool_bytes_for(cfg, bits), device=device)
    layer.load_pages([synth.expert_weights(cfg, p) for p in range(3)], bits, synth.pool_order(cfg))
    if cfg.n_shared:
        layer.set_shared_experts(cfg.n_shared)
    H, D = cfg.H, 64 if cfg.H < 1024 else 128
    heads, kv = H // D, max(H // D // 8, 1)
    cache = ops.KVCache(n_blocks, block_tokens, kv, D, act, fp8=fp8_cache, device=device)
    cache.pool.zero_()
    g = torch.Generator().manual_seed(seed)
    N = (heads + 2 * kv) * D
    w = torch.randn(N, H, generator=g) * H ** -0.5
    # e4m3 with one scale per 128 x 128 block, the last rows' blocks cut short
    pad = torch.zeros(-(-N // 128) * 128, H)
    pad[:N] = w
    tiles = pad.view(-1, 128, H // 128, 128)
    scale = (tiles.abs().amax((1, 3)) / 448.0).clamp_min(2.0 ** -126)
    w8 = (tiles / scale[:, None, :, None]).to(torch.float8_e4m3fn).view(-1, H)[:N].contiguous()
    draw = lambda *shape: (torch.randn(*shape, generator=g) * shape[-1] ** -0.5).to(act).to(device)  # noqa: E731
    norms = [(1 + 0.1 * torch.randn(H, generator=g)).to(act).to(device) for _ in range(2)]
    return DecoderBlock(layer, cache, heads, w8.to(device), scale.to(device), draw(H, heads * D), draw(cfg.E_routed, H),
                        *norms, **routing)


def main(argv=None):
    ap = argparse.ArgumentParser(description="Decode through one block: a prompt per sequence, then single tokens.")
    ap.add_argument("--layer", default="tiny", choices=sorted(synth.CONFIGS))
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--prompt", type=int, default=100)
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--block-tokens", type=int, default=32)
    ap.add_argument("--fp8-cache", action="store_true")
    a = ap.parse_args(argv)
    if min(a.batch, a.prompt, a.steps) < 1:
        ap.error("--batch, --prompt and --steps must be at least 1")
    longest = a.prompt + a.steps
    n_blocks = a.batch * -(-longest // a.block_tokens)
    block = random_block(a.layer, n_blocks, a.block_tokens, a.fp8_cache)
    tables = BlockTables(n_blocks, a.block_tokens, a.batch, longest)
    H, act = block.layer.cfg.H, block.cache.act
    g = torch.Generator(device="cuda").manual_seed(1)
    draw = lambda n: torch.randn(n, H, generator=g, device="cuda").to(act)  # noqa: E731
    for s in range(a.batch):
        y, _ = block.step(draw(a.prompt), None, *tables.step([s], [a.prompt]), max_len=longest)

    # A decode step is captured once and replayed: its inputs are copied into
    # the captured ones, max_len bounds all lengths to come.
    everyone, one = list(range(a.batch)), [1] * a.batch
    x, args = draw(a.batch), tables.step(everyone, one)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block.step(x, None, *args, max_len=longest)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, _ = block.step(x, None, *args, max_len=longest)
    times = []
    for i in range(a.steps):
        if i:
            for t, new in zip((x, *args), (draw(a.batch), *tables.step(everyone, one))):
                t.copy_(new)
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        graph.replay()
        end.record()
        end.synchronize()
        times.append(begin.elapsed_time(end))
    print("%s: %d sequences, %d + %d tokens, %s cache: %.1f us per decode step, output rms %.3g" % (
        a.layer, a.batch, a.prompt, a.steps, "8-bit" if a.fp8_cache else "16-bit", 1e3 * float(np.median(times)),
        float(y.float().pow(2).mean().sqrt())))


if __name__ == "__main__":
    main()
