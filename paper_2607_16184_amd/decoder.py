"""One decoder block around a paged MoE layer, as a serving loop runs it.

A step takes any mix of tokens: one new token of each decoding sequence, or a
prompt's tokens in a row (each attends to the cache up to itself, so a chunk is
written first and read afterwards). Per step:

    z  = x + residual;  8-bit rows of norm(z)      rms_norm
    q, k, v                                        Linear8
    k, v -> the sequences' blocks                  KVCache.append, append_rotated
    o  = attention over them                       KVCache.attend, attend_rows
    z  = z + o Wo;  16-bit rows h of norm(z)       (a plain product), rms_norm
    experts of h, and their order                  (a plain product), route_grouped
    y  = experts(h)                                PagedLayer.forward

With a rotation, or norms of query and key heads, those are done where keys and
values are written. A step by sequences (``starts``) gives each sequence a run of
rows: a prompt's chunk reads the cache once for many rows, and with masks the rows are
a tree of drafted tokens, of which KVCache.keep keeps the accepted ones.

A sequence's tokens lie in the blocks that its row of the block table names;
BlockTables hands blocks out and fills a step's arguments.

    python -m paper_2607_16184_amd.decoder --layer tiny --batch 16 --prompt 100 --steps 32
    python -m paper_2607_16184_amd.decoder --layer tiny --batch 16 --rotate --draft 8
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

    def _extend_all(self, sequences: Sequence[int], tokens: Sequence[int]):
        """The slots of each listed sequence's new tokens, or nothing changed."""
        if len(set(sequences)) < len(sequences):
            raise ValueError("a sequence is listed once, with all its new tokens")
        if len(tokens) != len(sequences):
            raise ValueError("%d counts of tokens for %d sequences" % (len(tokens), len(sequences)))
        need = sum(len(self._new_blocks(s, n)) for s, n in zip(sequences, tokens))
        if need > len(self.free):
            raise MemoryError("%d blocks are needed, %d are free" % (need, len(self.free)))
        return [self.extend(s, n) for s, n in zip(sequences, tokens)]

    def step(self, sequences: Sequence[int], tokens: Sequence[int], device="cuda"):
        """(block_table, lens, slots) of a step that gives each listed sequence
        so many new tokens, a row per token. A step that is refused changes
        nothing."""
        slots = self._extend_all(sequences, tokens)
        rows = np.repeat(np.asarray(sequences, dtype=np.int64), tokens)
        lens = np.concatenate([np.arange(self.length[s] - n, self.length[s]) + 1 for s, n in zip(sequences, tokens)])
        return (torch.from_numpy(self.table[rows]).to(device), torch.from_numpy(lens.astype(np.int32)).to(device),
                torch.from_numpy(np.concatenate(slots)).to(device))

    def rows(self, sequences: Sequence[int], tokens: Sequence[int], depth: Sequence[Sequence[int]] = None, device="cuda"):
        """The arguments block_table, lens, slots, starts and positions of such a
        step by sequences: table and lens have a row per sequence, whose tokens are rows
        starts[i] .. starts[i + 1] - 1. Positions follow each other; of a tree of
        drafted tokens they are those after the context by ``depth``, a list per
        sequence (0: a first token)."""
        if depth is not None and ([len(d) for d in depth] != list(tokens) or any(j < 0 for d in depth for j in d)):
            raise ValueError("a depth of at least 0 for each new token")
        first = [int(self.length[s]) if 0 <= s < len(self.length) else 0 for s in sequences]
        slots = self._extend_all(sequences, tokens)
        after = [np.arange(n) for n in tokens] if depth is None else [np.asarray(d, dtype=np.int64) for d in depth]
        pos = np.concatenate([f + a for f, a in zip(first, after)] or [np.zeros(0)])
        starts = np.concatenate([[0], np.cumsum(tokens)])
        put = lambda a, t: torch.from_numpy(np.asarray(a).astype(t)).to(device)  # noqa: E731
        return dict(block_table=put(self.table[list(sequences)], np.int32), lens=put(self.length[list(sequences)], np.int32),
                    slots=put(np.concatenate(slots or [np.zeros(0)]), np.int64), starts=put(starts, np.int32),
                    positions=put(pos, np.int32))

    def truncate(self, sequence: int, length: int):
        """Forget a sequence's tokens from ``length`` on; blocks without any are
        free again."""
        if not 0 <= sequence < len(self.length) or not 0 <= length <= self.length[sequence]:
            raise ValueError("sequence %d has no %d tokens" % (sequence, length))
        keep = -(-length // self.P)
        row = self.table[sequence, keep:]
        self.free.extend(int(b) for b in row[row >= 0][::-1])
        row[:] = -1
        self.length[sequence] = length


class DecoderBlock:
    """Attention and paged experts between two norms. ``w_qkv`` is [(heads + 2
    kv_heads) head_dim, H] e4m3 with its block scales; w_o [H, heads head_dim],
    w_router [E, H] and the norms' weights [H] (or None) are 16-bit. ``rotate``,
    if given, is an ops.Rotation, or gets (qkv [T, heads + 2 kv_heads, head_dim],
    lens) and turns the queries and keys in it by their positions, in place.
    ``q_norm`` and ``k_norm`` [head_dim], if either is given: heads are normed."""

    def __init__(self, layer: PagedLayer, cache: ops.KVCache, heads: int, w_qkv: torch.Tensor, qkv_scale: torch.Tensor,
                 w_o: torch.Tensor, w_router: torch.Tensor, norm_attn: torch.Tensor = None, norm_moe: torch.Tensor = None,
                 eps: float = 1e-5, rotate=None, K: int = None, q_norm: torch.Tensor = None, k_norm: torch.Tensor = None,
                 **routing):
        self.layer, self.cache, self.heads, self.eps, self.rotate = layer, cache, heads, eps, rotate
        self.q_norm, self.k_norm, self.head_norm = q_norm, k_norm, q_norm is not None or k_norm is not None
        if self.head_norm and not (rotate is None or isinstance(rotate, ops.Rotation)):
            raise ValueError("norms of heads go before the rotation: it must be an ops.Rotation, or none")
        self.qkv = ops.Linear8(w_qkv, qkv_scale)
        if w_qkv.shape != ((heads + 2 * cache.kv_heads) * cache.head_dim, layer.cfg.H):
            raise ValueError("w_qkv is not [(heads + 2 kv_heads) head_dim, H]")
        self.w_o, self.w_router = w_o.t().contiguous(), w_router.t().contiguous()
        self.norm_attn, self.norm_moe = norm_attn, norm_moe
        self.K, self.routing = K or layer.cfg.K, dict(n_shared=layer.cfg.n_shared, **routing)

    def step(self, x: torch.Tensor, residual: torch.Tensor, block_table: torch.Tensor, lens: torch.Tensor, slots: torch.Tensor,
             max_len: int, starts: torch.Tensor = None, positions: torch.Tensor = None,
             masks: torch.Tensor = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """(y, residual) of the block for x [T, H] and the residual so far (None
        at first): the next block's x and residual. The table and lens have a row
        per token (BlockTables.step), or with ``starts`` and ``positions`` one per
        sequence (BlockTables.rows), whose rows see what is before them or, with
        ``masks``, the tokens whose bits are set (KVCache.attend_rows)."""
        if (starts is None) != (positions is None) or (masks is not None and starts is None):
            raise ValueError("a step by sequences has starts and positions; masks are for such steps")
        T, act, cache = x.shape[0], x.dtype, self.cache
        z, _, q8, qs = ops.rms_norm(x, self.norm_attn, residual, eps=self.eps, y16=False, y8=True)
        qkv = self.qkv.forward(q8, qs, dtype=act).view(T, -1, cache.head_dim)
        fused = self.head_norm or isinstance(self.rotate, ops.Rotation)
        if self.rotate is not None and not fused:
            self.rotate(qkv, lens if positions is None else positions + 1)
        q, k, v = qkv.split([self.heads, cache.kv_heads, cache.kv_heads], dim=1)
        if fused:
            pos, offset = (lens, -1) if positions is None else (positions, 0)
            cache.append_rotated(k, v, slots, pos, self.rotate, q, self.q_norm, self.k_norm, norm=self.head_norm, eps=self.eps,
                                 offset=offset, q_out=q)
        else:
            cache.append(k, v, slots)
        if starts is None:
            o = cache.attend(q, block_table, lens, max_len)
        else:
            o = cache.attend_rows(q, starts, block_table, lens, max_len, masks=masks)
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
    ap.add_argument("--rotate", action="store_true", help="turn queries and keys by their positions")
    ap.add_argument("--draft", type=int, default=0, help="drafted tokens per sequence and step, in a tree of two branches")
    a = ap.parse_args(argv)
    if min(a.batch, a.prompt, a.steps) < 1 or not 0 <= a.draft <= 64:
        ap.error("--batch, --prompt and --steps must be at least 1, --draft 0 to 64")
    new = max(a.draft, 1)                                        # rows of a sequence and step
    longest = a.prompt + a.steps * -(-new // 2) + new
    n_blocks = a.batch * -(-longest // a.block_tokens)
    block = random_block(a.layer, n_blocks, a.block_tokens, a.fp8_cache)
    if a.rotate:
        block.rotate = ops.Rotation(block.cache.head_dim)
    tables = BlockTables(n_blocks, a.block_tokens, a.batch, longest)
    H, act = block.layer.cfg.H, block.cache.act
    g = torch.Generator(device="cuda").manual_seed(1)
    draw = lambda n: torch.randn(n, H, generator=g, device="cuda").to(act)  # noqa: E731
    for s in range(a.batch):
        y, _ = block.step(draw(a.prompt), None, **tables.rows([s], [a.prompt]), max_len=longest)

    # A step is captured once and replayed: its inputs are copied into the captured
    # ones, max_len bounds all lengths to come. Drafted token j sees j - 2, j - 4, ..:
    # two branches after the context. Of one of them, drawn anew each step, a part is
    # accepted.
    everyone = list(range(a.batch))
    if a.draft:
        sees = torch.tensor([sum(1 << i for i in range(j % 2, j + 1, 2)) for j in range(min(new, 63))] +
                            [sum(1 << i for i in range(1, 63, 2)) - (1 << 63)] * (new == 64), dtype=torch.int64)
        masks = sees.repeat(a.batch)[:, None].cuda()
        chosen, kept = masks.new_zeros(a.batch, 1), torch.zeros(a.batch, dtype=torch.int32, device="cuda")
        depth = [[j // 2 for j in range(new)]] * a.batch
    else:
        masks = None

    def arguments():
        if a.draft:
            return tables.rows(everyone, [new] * a.batch, depth)
        return dict(zip(("block_table", "lens", "slots"), tables.step(everyone, [1] * a.batch)))

    args = arguments()
    x = draw(a.batch * new)

    def step():
        y, _ = block.step(x, None, **args, max_len=longest, masks=masks)
        if a.draft:
            block.cache.keep(args["starts"], args["block_table"], args["lens"], longest, chosen, out=kept)
        return y

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = step()
    times, total = [], 0
    for i in range(a.steps):
        if i:
            x.copy_(draw(a.batch * new))
            for name, fresh in arguments().items():
                args[name].copy_(fresh)
        if a.draft:
            paths = [list(range(s % 2, new, 2))[:(i + s) % (-(-new // 2)) + 1] for s in everyone]
            chosen.copy_(torch.tensor([[sum(1 << j for j in p) - (1 << 64) * (63 in p)] for p in paths]))
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        graph.replay()
        end.record()
        end.synchronize()
        times.append(begin.elapsed_time(end))
        if a.draft:
            for s, n in enumerate(kept.tolist()):
                total += n - (int(tables.length[s]) - new)
                tables.truncate(s, n)
    print("%s: %d sequences, %d + %d tokens, %s cache: %.1f us per decode step, output rms %.3g" % (
        a.layer, a.batch, a.prompt, a.steps, "8-bit" if a.fp8_cache else "16-bit", 1e3 * float(np.median(times)),
        float(y.float().pow(2).mean().sqrt())))
    if a.draft:
        print("%d drafted tokens per sequence and step, %.2f kept" % (new, total / (a.steps * a.batch)))


if __name__ == "__main__":
    main()
