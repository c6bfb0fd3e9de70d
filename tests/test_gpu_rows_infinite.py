"""Infinite values in the cache at positions that all rows see, under weights of any
size: attention of several rows against its definition in 64 bits (tests/rows_ref.py)."""
import math

import pytest
import torch

import ops_ref as R
import rows_ref as RR
from test_gpu_ops import BF, FP, _cache, _gen, _within
from test_gpu_rows import _once

pytestmark = pytest.mark.gpu

INF = math.inf


@pytest.mark.parametrize("act", [BF, FP])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("gap", [3.0, 30.0, 60.0, 120.0, 500.0])
@pytest.mark.parametrize("n,ctx", [(5, 200), (9, 4000), (150, 600), (300, 3000)])
@pytest.mark.parametrize("tree", [False, True])
def test_infinite_values_under_weights_of_any_size(act, D, gap, n, ctx, tree):
    """One channel of the keys makes the scores: rows have one key `gap` nats above the
    others, at the beginning, in the middle or at the end. Infinities stand at the first
    positions, in the middle and at the context's end, in channels of their own: each
    makes its channel infinite, the two of one channel that differ in sign make it no
    number, and so does one whose key is -infinity (no weight at all). In 64 bits no
    weight is nothing below 745 nats. In workgroups, splits and shares, few columns and
    many."""
    g = _gen(n)
    L = ctx + n
    for peak in (3, ctx // 2 + 1, ctx - 2):
        k, v = torch.zeros(L, 1, D), torch.randn(L, 1, D, generator=g)
        k[peak, 0, 1] = gap
        for at, c, x in ((0, 0, INF), (ctx // 2, 5, -INF), (ctx - 1, 17, INF), (33, 40, INF), (ctx - 40, 40, -INF), (ctx // 3, D - 1, INF)):
            v[at, 0, c] = x
        k[ctx // 3, 0, 1] = -INF                                 # of channel D - 1
        k[ctx // 4, 0, 1] = -INF                                 # finite values without weight
        q = torch.zeros(n, 4, D)
        q[:, :, 1] = 1.0
        q[:, 2, 1] = 0.5
        q, k, v = q.to(act), k.to(act), v.to(act)
        nb = -(-L // 64)
        c = _cache(nb, 64, 1, D, act, 16)
        c.append(k.cuda(), v.cuda(), torch.arange(L).cuda())
        args = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, n], [list(range(nb))], [L])]
        masks = None
        if tree:                                                 # each row its own token alone
            masks = torch.zeros(n, 5, dtype=torch.int64)
            for i in range(n):
                masks[i, i // 64] = (1 << i % 64) - (1 << 64) * (i % 64 == 63)
        out = c.attend_rows(q.cuda(), *args, L, masks=None if masks is None else masks.cuda(), scale=1.0).cpu()
        # (the reference goes row by row where values are no numbers: rows of the ends and the middle)
        rows = sorted({0, 1, n // 2, n - 2, n - 1} | ({31, 32, 127, 128} if n > 129 else set()))
        on = RR.seen(n, ctx, masks)[rows]
        o, _, mass, size = RR.attend(q[rows], k.double(), v.double(), on, 1.0)
        for x in (INF, -INF):
            assert torch.equal(out[rows] == x, o == x), "infinities in other places"
        assert o[0, 0, 0] == INF and o[0, 0, 5] == -INF and o[0, 0, 40].isnan() and o[0, 0, D - 1].isnan()
        # scores are one product of numbers that their type holds, and at most two
        # factors; weights and sums as in the tests of finite values
        once = _once(n, 1, 4, act, 16)
        rel = 2 * 4 * 2.0 ** -23 * size.nan_to_num(0, gap, gap) + (L + 64) * 2.0 ** -23 + 2.0 ** -15 + (R.U[once] if once else 0.0)
        finite = o.isfinite()
        bound = R.U[act] * (1 + 2 ** -8) * o.abs() + rel[..., None] * mass + 2 * R.TINY[act]
        _within(torch.where(finite, out[rows], 0.0), torch.where(finite, o, 0.0), torch.where(finite, bound, 0.0), "finite channels")
        assert torch.equal(out[rows].isnan(), o.isnan())
