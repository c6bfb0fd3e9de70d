"""Attention of several new tokens per sequence over the paged cache (prompt chunks,
trees of drafted tokens) against its definition in 64 bits (tests/rows_ref.py)."""
import math

import pytest
import torch

import ops_ref as R
import rows_ref as RR
from test_gpu_ops import BF, FP, _cache, _gen, _same, _within

pytestmark = pytest.mark.gpu


def _tree(n, words, g, empty=False):
    """Masks of a random tree: each token's parent is an earlier one, or the context;
    bits past n are set, they are not to be looked at."""
    rows = []
    for j in range(n):
        p = int(torch.randint(-1, max(j, 1), (1,), generator=g)) if j else -1
        rows.append((rows[p] if p >= 0 else 0) | 1 << j)
    if empty and n > 1:
        rows[n // 2] = 0
    junk = ((1 << 64 * words) - 1) >> n << n
    rows = [r & ((1 << 64 * words) - 1) | junk for r in rows]
    signed = lambda w: w - (1 << 64) if w >> 63 else w  # noqa: E731
    return torch.tensor([[signed(r >> 64 * w & (1 << 64) - 1) for w in range(words)] for r in rows], dtype=torch.int64).view(n, words)


def _bound(act, D, n_keys, size, o, mass, once=None):
    # scores: D products summed in fp32 and two scalings; weights: twice the score's
    # error, an exponential, a sum of n_keys terms; values: the second 16-bit term
    # leaves 2^-16 of a weight. Calls of many columns round a weight once, to the type
    # `once`: it is then off by up to half a step, U of itself, and so is its product;
    # the sum of the products' errors is at most U times the mass.
    ds = (D + 8) * 2.0 ** -23 * size
    rel = 2 * ds + (n_keys + 64) * 2.0 ** -23 + 2.0 ** -15 + (R.U[once] if once else 0.0)
    return ds, R.U[act] * (1 + 2 ** -8) * o.abs() + rel[..., None] * mass + 2 * R.TINY[act]


def _once(T, B, g, act, bits):
    """The type that a call's weights are rounded to, None: two terms."""
    return None if T * g <= 64 * B or (act is FP and bits == 8) else act


def _case(seqs, P, H, g, D, act, bits, tree=None, window=0, seed=0, scale=None, missing=(), odd=(), pad_rows=0, max_len=None,
          stride=None, empty=False, cut=None, stream=None):
    """seqs: (context, new tokens) per sequence. The cache is filled through append
    (NaN elsewhere); odd: (sequence, position, value) that keys and values get. tree:
    words of the masks. Every row is checked, and that no other row is written."""
    gen = _gen(seed)
    B, lens = len(seqs), [a + n for a, n in seqs]
    L = max_len or max(max(lens), 1)
    nb = -(-max(L, max(lens)) // P)
    table = (torch.randperm(B * nb, generator=gen) + 1).int().view(B, nb)    # block 0 holds NaN
    unit = 1
    if stride == 256:
        unit = R.block_bytes(H, P, D, bits) // 256
        table *= unit
    c = _cache(B * nb * unit + 1, P, H, D, act, bits, stride)
    kv = torch.randn(sum(lens), 2, H, D, generator=gen).to(act)
    first = [sum(lens[:b]) for b in range(B)]
    for b, t, x in odd:
        kv[first[b] + t] = x if not isinstance(x, tuple) else kv[first[b] + t]
        if isinstance(x, tuple):                                # (side, channel, value)
            kv[first[b] + t, x[0], :, x[1]] = x[2]
    slots = torch.cat([table[b, torch.arange(m) // P].long() * P + torch.arange(m) % P for b, m in enumerate(lens)])
    dev = kv.cuda()
    c.append(dev[:, 0], dev[:, 1], slots.cuda())
    new = [n for _, n in seqs]
    T = sum(new) + 2 * pad_rows
    starts = torch.tensor([pad_rows + sum(new[:b]) for b in range(B + 1)], dtype=torch.int32)
    q = torch.randn(T, H * g + 2, D, generator=gen).to(act)
    masks = None
    if tree:
        masks = torch.full((T, tree), -1, dtype=torch.int64)
        for b, n in enumerate(new):
            if n:
                masks[starts[b]:starts[b + 1]] = _tree(n, tree, gen, empty)
    bad = {}
    for b, j, block in missing:
        table[b, j] = block
        bad.setdefault(b, []).append(j)
    out = torch.full((T, H * g, D), 7.0, dtype=act, device="cuda")
    lse = torch.full((T, H * g), 7.0, device="cuda")
    args = [starts.cuda(), table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")]
    q_d, m_d = q.cuda(), None if masks is None else masks.cuda()
    torch.cuda.synchronize()
    got = c.attend_rows(q_d[:, 1:1 + H * g], *args, L, masks=m_d, scale=scale, window=window, out=out, lse=lse, stream=stream)
    torch.cuda.synchronize()
    assert got is out
    sc = D ** -0.5 if scale is None else scale
    where = "cuda" if sum(lens) * sum(new) > 200000 else "cpu"
    for b, (ctx, n) in enumerate(seqs):
        if not n:
            continue
        r0 = int(starts[b])
        on = RR.seen(n, ctx, None if masks is None else masks[r0:r0 + n], window)
        on[:, L:] = False
        for j in bad.get(b, ()):
            on[:, j * P:(j + 1) * P] = False
        k64, v64 = (RR.cached(kv[first[b]:first[b] + lens[b], i], bits).to(where) for i in (0, 1))
        o, e, mass, size = (x.cpu() for x in RR.attend(q[r0:r0 + n, 1:1 + H * g].to(where), k64, v64, on.to(where), sc))
        ds, bound = _bound(act, D, lens[b], size, o, mass, _once(T, B, g, act, bits))
        _within(out[r0:r0 + n], o, bound, "sequence %d" % b)
        _within(lse[r0:r0 + n], e, ds + (lens[b] + 64) * 2.0 ** -23 + 2.0 ** -21 * e.abs().nan_to_num(0, 0, 0), "lse %d" % b)
    out[pad_rows:pad_rows + sum(new)] = 7.0
    lse[pad_rows:pad_rows + sum(new)] = 7.0
    assert (out == 7.0).all() and (lse == 7.0).all()
    return c


SEQS = [(0, 1), (0, 3), (5, 2), (31, 1), (30, 5), (32, 16), (1, 33), (200, 7), (0, 0), (64, 64), (95, 1)]


@pytest.mark.parametrize("D", [64, 128, 192, 256])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("act", [BF, FP])
@pytest.mark.parametrize("tree", [None, 1])
def test_lengths(D, bits, act, tree):
    _case(SEQS, 64, 2, 3, D, act, bits, tree, seed=D)
    _case([(3, 2), (40, 1)], 32, 1, 1, D, act, bits, tree, seed=D)           # one wave's columns
    _case([(3, 9), (300, 6), (33, 8)], 32, 2, 4, D, act, bits, tree, seed=D)  # two


@pytest.mark.parametrize("P", [32, 64, 128, 256])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("g", [1, 2, 7, 16, 24])
@pytest.mark.parametrize("tree", [None, 1])
def test_heads_and_blocks(P, bits, g, tree):
    _case([(P - 1, 2), (3 * P, 17), (0, 1), (10, 40)], P, 2, g, 64, BF, bits, tree, seed=P + g)


@pytest.mark.parametrize("window", [1, 2, 20, 64, 333])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("tree", [None, 1])
def test_windows(window, bits, tree):
    _case([(0, 1), (0, 40), (31, 2), (64, 9), (300, 50), (777, 3)], 32, 1, 2, 128, FP, bits, tree, window=window, seed=window)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("words,n", [(1, 64), (1, 63), (2, 65), (2, 100), (2, 128), (3, 130), (1, 100), (4, 20)])
def test_words_of_a_mask(words, n, bits):
    """Trees of up to 130 tokens; 100 tokens with one word: those past it are not
    seen. The trees begin at every place of a tile."""
    for ctx in (0, 7, 31, 33):
        _case([(ctx, n), (ctx + 50, 3)], 32, 1, 2, 64, BF, bits, words, seed=n + ctx)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("act,bits", [(BF, 16), (FP, 16), (BF, 8), (FP, 8)])
@pytest.mark.parametrize("tree", [None, 1])
def test_long_contexts(D, act, bits, tree):
    """Contexts that are split over workgroups, ragged, with and without a window."""
    seqs = [(6000, 5), (0, 3), (2500, 30), (9000, 1), (33, 2)]
    _case(seqs, 64, 2, 4, D, act, bits, tree, seed=D)
    _case(seqs, 64, 2, 4, D, act, bits, tree, window=1500, seed=D)
    _case([(3000, 4)], 64, 1, 4, D, act, bits, tree, seed=D)


@pytest.mark.parametrize("act,bits,D,g", [(BF, 16, 128, 4), (FP, 16, 64, 8), (BF, 8, 128, 4), (FP, 8, 64, 3), (BF, 16, 256, 2),
                                          (BF, 8, 192, 5), (FP, 16, 192, 2), (FP, 16, 128, 4), (BF, 16, 64, 1)])
def test_chunks(act, bits, D, g):
    """Prompt chunks of many rows, with odd ends."""
    _case([(0, 700), (900, 333)], 64, 2, g, D, act, bits, seed=D + g)
    _case([(130, 257)], 32, 1, g, D, act, bits, window=100, seed=g)
    _case([(2000, 300)] + [(37 * i, 1) for i in range(20)], 32, 2, g, D, act, bits, seed=g)   # a mixed batch


@pytest.mark.parametrize("bits", [16, 8])
def test_large_trees_of_many_heads(bits):
    _case([(500, 60), (1200, 33)], 64, 2, 8, 128, BF, bits, 1, seed=2)
    _case([(500, 90), (0, 96)], 64, 1, 16, 64, FP, bits, 2, seed=3)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("tree", [None, 1])
def test_missing_blocks(bits, tree):
    """Table entries outside the pool: their positions are left out, those of the new
    tokens among them."""
    _case([(200, 20), (150, 9), (0, 40), (3000, 3)], 32, 1, 4, 128, BF, bits, tree, seed=3,
          missing=[(0, 0, -1), (0, 3, 1 << 30), (1, 4, -5), (2, 0, -1), (2, 1, -1), (3, 50, -1), (3, 93, -1)])


@pytest.mark.parametrize("tree", [None, 1])
def test_rows_that_see_nothing(tree):
    """Masks without a bit before an empty context, and rows of sequences whose
    blocks are all missing: zeros."""
    _case([(0, 5), (0, 9), (40, 3)], 32, 2, 2, 64, BF, 16, tree, seed=1, empty=True, missing=[(1, 0, -1)])


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("act", [BF, FP])
@pytest.mark.parametrize("D", [64, 128, 192])
@pytest.mark.parametrize("tree", [None, 1])
def test_values_that_are_no_numbers_stay_with_the_rows_that_see_them(D, bits, act, tree):
    odd = [(0, 40, math.nan), (1, 21, (1, 5, math.inf)), (1, 25, (1, D - 1, -math.inf)), (2, 70, (0, 3, math.nan)),
           (3, 9, (1, 17, math.nan)), (3, 30, (1, 18, math.inf))]
    _case([(33, 20), (20, 12), (64, 40), (0, 64)], 32, 2, 2, D, act, bits, tree, seed=D, odd=odd)
    _case([(2000, 50), (1990, 12)], 32, 2, 2, D, act, bits, tree, seed=D,
          odd=[(0, 2010, math.nan), (0, 2040, (1, 7, math.inf)), (1, 1995, (1, 0, math.nan))])
    # a chunk: rows before the value, in the same and other groups of columns
    _case([(100, 500)], 32, 1, 4, D, act, bits, None if tree is None else 8, seed=D, odd=[(0, 350, math.nan), (0, 420, (1, 7, math.inf))])


@pytest.mark.parametrize("bits", [16, 8])
def test_padding_rows_bounds_and_units(bits):
    for tree in (None, 1):
        _case([(100, 5), (3, 7)], 32, 2, 2, 64, BF, bits, tree, pad_rows=13, max_len=400)
        _case([(100, 5), (3, 7)], 32, 2, 2, 64, BF, bits, tree, stride=256)
        _case([(100, 40), (3, 7)], 32, 1, 2, 64, BF, bits, tree, stride=(1 << 30) + 256)
        _case([(100, 60), (300, 7)], 32, 1, 2, 64, BF, bits, tree, max_len=130)   # lengths past the bound


def test_more_new_tokens_than_cached_ones():
    """A length below the count of new tokens: tokens before position 0 do not
    exist."""
    g = _gen(0)
    c = _cache(3, 32, 1, 64, BF, 16)
    kv, q = torch.randn(20, 2, 1, 64, generator=g).to(BF), torch.randn(30, 2, 64, generator=g).to(BF)
    dev = kv.cuda()
    c.append(dev[:, 0], dev[:, 1], torch.arange(20).cuda() + 32)
    args = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 30], [[1]], [20])]
    masks = _tree(30, 1, g)
    for m in (None, masks):
        out = c.attend_rows(q.cuda(), *args, 32, masks=None if m is None else m.cuda())
        o, _, mass, size = RR.attend(q, kv[:, 0].double(), kv[:, 1].double(), RR.seen(30, -10, m), 0.125)
        _within(out, o, _bound(BF, 64, 20, size, o, mass)[1], "rows")


@pytest.mark.parametrize("bits", [16, 8])
def test_many_sequences(bits):
    for tree in (None, 1):
        _case([((37 * i) % 90, i % 4) for i in range(200)], 32, 1, 2, 64, BF, bits, tree, seed=11)


def test_large_and_small_scores():
    for tree in (None, 1):
        for scale in (4.0, -3.0, 1e-6, 0.0):
            _case([(50, 9), (700, 40)], 32, 2, 2, 64, BF, 16, tree, scale=scale, seed=5)
            _case([(50, 9), (700, 40)], 32, 2, 2, 64, FP, 16, tree, scale=scale, seed=5)


def _sink(act, bits, D, n, ctx, ahead, g):
    """Keys that tie behind one that is `ahead` nats in front and has no value."""
    k, v = torch.zeros(ctx + n, 1, D), torch.randn(ctx + n, 1, D, generator=g).abs() + 1.0
    k[0, 0, 1] = 8.0
    v[0] = 0.0
    q = torch.zeros(n, 4, D)
    q[:, :, 1] = torch.tensor(ahead) / 8.0
    return k.to(act), v.to(act), q.to(act)


@pytest.mark.parametrize("act,bits", [(FP, 16), (BF, 16), (FP, 8)])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n,ctx", [(3, 2000), (17, 600), (300, 1500)])
def test_sink_without_a_value(act, bits, D, n, ctx):
    """Weights far below the largest keep their bits: the outputs are made of them
    alone."""
    k, v, q = _sink(act, bits, D, n, ctx, [8.0, 15.0, 20.0, 27.0], _gen(D))
    nb = -(-(ctx + n) // 64)
    c = _cache(nb, 64, 1, D, act, bits)
    c.append(k.cuda(), v.cuda(), torch.arange(ctx + n).cuda())
    args = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, n], [list(range(nb))], [ctx + n])]
    out = c.attend_rows(q.cuda(), *args, ctx + n, scale=1.0)
    o, _, mass, size = RR.attend(q, R.cached(k, bits), R.cached(v, bits), RR.seen(n, ctx), 1.0)
    _within(out, o, _bound(act, D, ctx + n, size, o, mass, _once(n, 1, 4, act, bits))[1], "rows")


def test_a_row_per_sequence_is_one_token_attention():
    """The same inputs through attend, with its bounds on both."""
    g = _gen(6)
    lens = [1, 40, 333, 1200]
    c = _cache(200, 32, 2, 128, BF, 16)
    table = torch.randperm(200, generator=g)[:160].int().view(4, 40)
    kv = torch.randn(sum(lens), 2, 2, 128, generator=g).to(BF).cuda()
    slots = torch.cat([table[b, torch.arange(m) // 32].long() * 32 + torch.arange(m) % 32 for b, m in enumerate(lens)])
    c.append(kv[:, 0], kv[:, 1], slots.cuda())
    q = torch.randn(4, 8, 128, generator=g).to(BF).cuda()
    dev = [table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), 1280]
    a = c.attend(q, *dev).float()
    b = c.attend_rows(q, torch.arange(5, dtype=torch.int32, device="cuda"), *dev).float()
    m = c.attend_rows(q, torch.arange(5, dtype=torch.int32, device="cuda"), *dev,
                      masks=torch.ones(4, 1, dtype=torch.int64, device="cuda")).float()
    # two roundings to bf16 of values that are 2^-14 of the row's largest apart at most
    for x in (b, m):
        assert ((a - x).abs() <= 2 * R.U[BF] * a.abs() + 2.0 ** -13 * a.abs().amax()).all()


def test_runs_twice_the_same_and_on_other_streams():
    side = torch.cuda.Stream()
    g = _gen(7)
    c = _cache(300, 32, 2, 128, BF, 16)
    c.pool.view(torch.bfloat16).copy_(torch.randn(c.pool.numel() // 2, generator=g))
    q = torch.randn(40, 8, 128, generator=g).to(BF).cuda()
    args = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 30, 40], [list(range(150)), list(range(150, 300))],
                                                                        [4000, 4790])]
    want = c.attend_rows(q, *args, 4800)
    side.wait_stream(torch.cuda.current_stream())
    again = c.attend_rows(q, *args, 4800, stream=side)
    third = c.attend_rows(q, *args, 4800)
    side.synchronize()
    assert _same(want, again) and _same(want, third)


@pytest.mark.parametrize("act,bits", [(BF, 16), (FP, 16), (BF, 8), (FP, 8)])
@pytest.mark.parametrize("D", [64, 128, 192, 256])
@pytest.mark.parametrize("tree", [None, 2])
def test_many_columns_under_windows_bounds_and_missing_blocks(act, bits, D, tree):
    """What the tests above do with few columns per sequence, with more than a
    workgroup's 128."""
    seqs = [(0, 70), (40, 33), (700, 100), (0, 0), (300, 1)]
    for window in (1, 50, 640):
        _case(seqs, 32, 1, 4, D, act, bits, tree, window=window, seed=window)
    _case(seqs, 32, 1, 4, D, act, bits, tree, seed=D, missing=[(0, 0, -1), (0, 1, 1 << 29), (1, 1, -3), (2, 5, -1), (2, 24, -1)])
    _case(seqs, 64, 2, 5, D, act, bits, tree, pad_rows=9, max_len=760, seed=D)
    _case(seqs, 32, 1, 4, D, act, bits, tree, max_len=90, empty=True, seed=D, scale=-0.2)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("tree", [None, 1])
def test_shares_over_missing_blocks_and_odd_values(bits, tree):
    """Few rows after long contexts: equal shares of all tiles, some of them in no
    block, one whole sequence without any, one that sees values that are no numbers."""
    seqs = [(5000, 4), (0, 2), (3300, 6), (96, 1), (4000, 9)]
    _case(seqs, 64, 2, 2, 128, BF, bits, tree, seed=8, missing=[(0, j, -1) for j in range(10, 60)] + [(1, 0, -1), (3, 0, -1), (3, 1, -1)])
    _case(seqs, 64, 1, 4, 64, FP, bits, tree, seed=9, odd=[(0, 100, (1, 3, math.inf)), (2, 3303, math.nan), (4, 4004, (1, 9, math.nan))])
    _case(seqs, 64, 1, 4, 64, BF, bits, tree, seed=9, window=3200, max_len=4003)
