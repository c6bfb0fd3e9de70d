"""How attention of several rows cuts its work: 32 columns a wave, first rounds of
workgroups whole beside split ones. Every row against the definition in 64 bits; the
workspace that a call asks for shows which cut it takes."""
import pytest
import torch

from paper_2607_16184_amd import pw
from test_gpu_ops import BF, FP, _cache
from test_gpu_rows import _case

pytestmark = pytest.mark.gpu


def _workspace(c, seqs, g, max_len, window=0):
    return pw.pw_attn_rows_workspace(c.desc, len(seqs), sum(n for _, n in seqs), c.kv_heads * g, max_len, window)


def _items(seqs, g, group):
    """At most: groups of columns of all sequences."""
    B, T = len(seqs), sum(n for _, n in seqs)
    return g * T // group + min(B, T)


# 16 columns a wave would fit less than 256 workgroups' worth; the items are the same
# for trees and chunks
SMALL = [(17 * i % 190, 9 + i % 8) for i in range(64)]           # 5 to 16 rows


@pytest.mark.parametrize("D", [64, 128, 192, 256])
@pytest.mark.parametrize("act", [BF, FP])
@pytest.mark.parametrize("tree", [None, 1])
def test_two_column_tiles_whole(D, act, tree):
    """64 sequences of 9 to 16 rows x 4 heads of 3 key heads: 16-bit caches, a workgroup
    per item (its last group of columns is full, short, or of one tile)."""
    c = _case(SMALL, 32, 3, 4, D, act, 16, tree, seed=D, empty=True, missing=[(1, 0, -1), (9, 2, 1 << 20)])
    assert _items(SMALL, 4, 32) * 3 >= 256 and _workspace(c, SMALL, 4, 206) == 0
    _case(SMALL, 64, 3, 4, D, act, 16, tree, seed=D, window=40, pad_rows=3, max_len=150)


@pytest.mark.parametrize("D,H", [(64, 10), (128, 10), (192, 6), (256, 6)])
@pytest.mark.parametrize("act", [BF, FP])
@pytest.mark.parametrize("tree", [None, 1])
def test_two_column_tiles_in_shares(D, H, act, tree):
    """16 sequences of 15 to 17 rows after up to 2100 tokens: equal shares of the tiles
    that an item's end may lie in."""
    seqs = [((0, 2100, 37, 700)[i % 4] + i, (15, 16, 17, 16)[i % 4]) for i in range(16)]
    L = max(a + n for a, n in seqs)
    c = _case(seqs, 64, H, 4, D, act, 16, tree, seed=D)
    # the parts' slots: shares and items of 32 columns
    items = _items(seqs, 4, 32)
    shares = (512 if D <= 128 else 256) // H
    assert _workspace(c, seqs, 4, L) == (shares + items) * H * 32 * (D + 2) * 4 + items * H * 8
    odd = [(2, 40, float("nan")), (5, 2100, float("inf")), (9, 1000, float("-inf"))]
    _case(seqs, 64, H, 4, D, act, 16, tree, seed=D, window=900, odd=odd, missing=[(1, j, -1) for j in range(3, 20)])


@pytest.mark.parametrize("act,bits,D,n,g", [(BF, 16, 256, 560, 8), (FP, 16, 256, 560, 8), (BF, 8, 256, 560, 8), (FP, 8, 256, 570, 8),
                                            (FP, 16, 192, 600, 8), (BF, 16, 192, 1100, 8), (FP, 16, 128, 1100, 8)])
@pytest.mark.parametrize("tree", [False, True])
def test_first_rounds_whole_and_the_last_split(act, bits, D, n, g, tree):
    """One chunk whose items are a round of workgroups or more and a few: those few are
    split, and 8 key heads' parts joined, from the chunk's first rows."""
    seqs = [(2400, n)]
    c = _case(seqs, 64, 8, g, D, act, bits, -(-n // 64) if tree else None, seed=D)
    need, items = _workspace(c, seqs, g, 2400 + n), _items(seqs, g, 128)
    slots = (need - items * 64) // ((D + 2) * 4)
    assert 0 < slots < 2 * items * 8 * 128, "all items in at least two parts"
    # (what the cut leaves whole is a whole number of rounds; the others share the rest)
    assert slots % (8 * 128) == 0
