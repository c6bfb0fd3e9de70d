"""Accepted drafted tokens moved together in the paged cache, and a drafting loop's
step through all operators of several new tokens per sequence."""
import numpy as np
import pytest
import torch

import ops_ref as R
import rows_ref as RR
from test_gpu_ops import BF, FP, _cache, _gen, _ops, _same, _within
from test_gpu_rows import _bound, _once, _tree

pytestmark = pytest.mark.gpu


def _bits(lists, words):
    signed = lambda w: w - (1 << 64) if w >> 63 else w  # noqa: E731
    rows = [sum(1 << j for j in js) for js in lists]
    return torch.tensor([[signed(r >> 64 * w & (1 << 64) - 1) for w in range(words)] for r in rows], dtype=torch.int64).view(-1, words)


def _keep(seqs, chosen, P, H, D, act, bits, words=1, missing=(), max_len=None, lens=None, seed=0):
    """seqs: (context, new) per sequence; chosen: lists of new tokens. The pool's bytes
    are compared with those of a copy on the host, slot by slot."""
    g = _gen(seed)
    B = len(seqs)
    L = max(a + n for a, n in seqs) if max_len is None else max_len
    nb = -(-max(L, 1) // P)
    table = (torch.randperm(B * nb, generator=g)).int().view(B, nb)
    c = _cache(B * nb, P, H, D, act, bits)
    c.pool.copy_(torch.randint(0, 256, (c.pool.numel(),), generator=g, dtype=torch.uint8))
    want = c.pool.cpu().numpy().copy()
    for b, j, bad in missing:
        table[b, j] = bad
    starts = np.cumsum([0] + [n for _, n in seqs])
    lens = [a + n for a, n in seqs] if lens is None else lens
    d, totals = np.arange(D), []
    for b, (_, n) in enumerate(seqs):
        ctx = lens[b] - n
        base = max(ctx, 0)
        js = [j for j in sorted(chosen[b]) if j < n and ctx + j >= 0]
        totals.append(base + len(js))
        for i, j in enumerate(js):
            slots = []
            for p in (ctx + j, base + i):
                blk = int(table[b, p // P]) if p < L else -1
                slots.append(blk * P + p % P if 0 <= blk < B * nb else -1)
            if min(slots) < 0:
                continue
            for h in range(H):
                for side, place in ((0, R.key_byte), (1, R.value_byte)):
                    at = [s // P * c.block_bytes + (2 * h + side) * P * D * bits // 8 + place(s % P, d, D, bits) for s in slots]
                    for e in range(bits // 8):
                        want[at[1] + e] = want[at[0] + e]
                    if bits == 8:
                        so = [s // P * c.block_bytes + 2 * H * P * D + 4 * ((side * H + h) * P + s % P) for s in slots]
                        want[so[1]:so[1] + 4] = want[so[0]:so[0] + 4]
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    got = c.keep(dev(starts), table.cuda(), dev(lens), L, _bits(chosen, words).cuda())
    assert got.tolist() == totals
    assert np.array_equal(c.pool.cpu().numpy(), want)


@pytest.mark.parametrize("D", [64, 128, 192, 256])
@pytest.mark.parametrize("act,bits", [(BF, 16), (FP, 8)])
def test_moves(D, act, bits):
    seqs = [(0, 5), (30, 8), (31, 40), (100, 1), (64, 64), (7, 0), (10, 3)]
    chosen = [[0, 2, 4], [1, 5, 7], list(range(1, 40, 3)), [0], list(range(1, 64)), [], []]
    _keep(seqs, chosen, 32, 3, D, act, bits, seed=D)


@pytest.mark.parametrize("bits", [16, 8])
def test_more_words_and_bits_past_the_end(bits):
    _keep([(50, 130), (3, 70), (0, 20)], [list(range(0, 130, 2)), [1, 63, 64, 69, 70, 120], [19, 20, 100]], 64, 2, 64, BF, bits, words=3)
    _keep([(50, 130)], [[5, 60]], 64, 1, 64, BF, bits, words=1)
    _keep([(2, 190)], [list(range(1, 190))], 32, 1, 64, BF, bits, words=3)   # each into its neighbour's place


@pytest.mark.parametrize("bits", [16, 8])
def test_missing_blocks_bounds_and_short_lengths(bits):
    _keep([(40, 60), (20, 30)], [list(range(1, 60, 2)), [3, 13, 14, 20]], 32, 2, 64, BF, bits,
          missing=[(0, 2, -1), (1, 0, 1 << 20)])
    _keep([(40, 60)], [list(range(1, 60, 2))], 32, 2, 64, BF, bits, max_len=70)
    _keep([(0, 30), (5, 9)], [[2, 11, 12, 20], [4]], 32, 1, 64, BF, bits, lens=[20, 0])


def _draft_step(c, x, pos, slots, starts, table, lens, masks, chosen, n_q, H, rot, max_len, out, kept):
    q, k, v = x.split([n_q, H, H], dim=1)
    q_out = c.append_rotated(k, v, slots, pos, rot, q)
    c.attend_rows(q_out, starts, table, lens, max_len, masks=masks, out=out)
    c.keep(starts, table, lens, max_len, chosen, out=kept)
    return q_out


@pytest.mark.parametrize("act,bits", [(BF, 16), (FP, 16), (BF, 8)])
def test_a_drafting_loop(act, bits):
    """Prompts in chunks, then trees of drafted tokens: rotated append, attention
    under the trees' masks, and the accepted path kept; after each step the cache
    holds the accepted tokens in a row, as a sequence decoded one by one would. The
    whole step is also captured and replayed with other inputs."""
    g = _gen(3)
    n_q, H, D, P, N = 4, 2, 64, 32, 9
    B, max_len = 3, 256
    c = _cache(B * 8, P, H, D, act, bits)
    c.pool.zero_()
    table = torch.randperm(B * 8, generator=g).int().view(B, 8)
    rot = _ops().Rotation(D)
    slot = lambda b, p: table[b, p // P].long() * P + p % P  # noqa: E731
    dev = lambda t: t.cuda()  # noqa: E731
    history = [[[], []] for _ in range(B)]                      # normed, turned keys and values as cached
    length = [0] * B

    def check(out, q_out, on_of, rows):
        at = 0
        for b, n in rows:
            k64 = torch.stack([R.cached(t, bits) for t in history[b][0]] + extra[b][0])
            v64 = torch.stack([R.cached(t, bits) for t in history[b][1]] + extra[b][1])
            o, _, mass, size = RR.attend(q_out[at:at + n].cpu(), k64, v64, on_of(b, n), D ** -0.5)
            # keys of 16-bit caches as the definition rounds them: a code that lies
            # beside it is one step off
            step = R.U[act] if bits == 16 else 2 * R.U[R.F8]
            ds, bound = _bound(act, D, len(k64), size, o, mass, _once(len(out), B, n_q // H, act, bits))
            _within(out[at:at + n], o, bound + (2 * step * size[..., None] + step) * mass, "sequence %d" % b)
            at += n

    def turned(k, pos):
        return RR.heads(k, pos, rot.inv_freq.cpu(), D, False, 1.0, True, None, 1e-6)[0].float()

    graph = None
    for turn, counts in enumerate([[40, 33, 70], [20, 1, 5]] + [[N] * B] * 5):
        tree = turn >= 2
        T = sum(counts)
        x = torch.randn(T, n_q + 2 * H, D, generator=g).to(act)
        starts = torch.tensor([sum(counts[:b]) for b in range(B + 1)], dtype=torch.int32)
        masks = torch.cat([_tree(n, 1, g) for n in counts]) if tree else None
        pos, slots, extra = [], [], []
        for b, n in enumerate(counts):
            depth = [bin(int(masks[starts[b] + j]) & (1 << n) - 1).count("1") - 1 if tree else j for j in range(n)]
            p = torch.tensor([length[b] + d for d in depth])
            pos.append(p)
            slots.append(slot(b, length[b] + torch.arange(n)))
            rows = x[starts[b]:starts[b] + n]
            extra.append([[R.cached(t, bits) for t in turned(rows[:, n_q:n_q + H], p).to(act if bits == 16 else torch.float32)],
                          [R.cached(t, bits) for t in rows[:, n_q + H:]]])
        lens = torch.tensor([length[b] + n for b, n in enumerate(counts)], dtype=torch.int32)
        leaf = [int(torch.randint(0, n, (1,), generator=g)) for n in counts]
        chosen = (torch.stack([masks[starts[b] + leaf[b]] for b in range(B)]) if tree
                  else _bits([list(range(min(n, 64))) for n in counts], 1))
        inputs = [dev(x), dev(torch.cat(pos).int()), dev(torch.cat(slots)), dev(starts), dev(table), dev(lens),
                  dev(masks) if tree else None, dev(chosen)]
        if tree and graph is None:
            held = [t if t is None else t.clone() for t in inputs]
            held_out = torch.empty(T, n_q, D, dtype=act, device="cuda")
            held_kept = torch.empty(B, dtype=torch.int32, device="cuda")
            side = torch.cuda.Stream()
            pool = c.pool.clone()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                _draft_step(c, *held, n_q, H, rot, max_len, held_out, held_kept)
            torch.cuda.current_stream().wait_stream(side)
            c.pool.copy_(pool)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                held_q = _draft_step(c, *held, n_q, H, rot, max_len, held_out, held_kept)
        if tree:
            pool = c.pool.clone()
            out, kept = torch.empty_like(held_out), torch.empty_like(held_kept)
            q_out = _draft_step(c, *inputs, n_q, H, rot, max_len, out, kept)
            eager = c.pool.clone()
            c.pool.copy_(pool)
            for t, new in zip(held, inputs):
                if t is not None:
                    t.copy_(new)
            graph.replay()
            assert _same(held_out, out) and _same(held_q, q_out) and torch.equal(held_kept, kept) and torch.equal(c.pool, eager)
        else:
            out = torch.empty(T, n_q, D, dtype=act, device="cuda")
            kept = torch.empty(B, dtype=torch.int32, device="cuda")
            if max(counts) > 64:                                # a chunk's tokens all stay
                q, k, v = inputs[0].split([n_q, H, H], dim=1)
                q_out = c.append_rotated(k, v, inputs[2], inputs[1], rot, q)
                c.attend_rows(q_out, *inputs[3:6], max_len, out=out)
                kept = inputs[5]
            else:
                q_out = _draft_step(c, *inputs, n_q, H, rot, max_len, out, kept)
        check(out, q_out, lambda b, n: RR.seen(n, length[b], masks[starts[b]:starts[b] + n] if tree else None),
              list(enumerate(counts)))
        for b, n in enumerate(counts):
            path = [j for j in range(n) if not tree or int(masks[starts[b] + leaf[b]]) >> j & 1]
            rows = x[starts[b]:starts[b] + n]
            kk = turned(rows[:, n_q:n_q + H], pos[b]).to(act if bits == 16 else torch.float32)
            for j in path:
                history[b][0].append(kk[j])
                history[b][1].append(rows[j, n_q + H:])
            length[b] += len(path)
        assert kept.tolist() == length
