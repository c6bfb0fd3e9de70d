"""Scores of attention of several rows in the kernel of many columns: large, small and
tied ones, against the definition in 64 bits (tests/rows_ref.py)."""
import pytest
import torch

import ops_ref as R
import rows_ref as RR
from test_gpu_ops import BF, FP, _cache, _gen, _within
from test_gpu_rows import _case, _once

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act,bits", [(BF, 16), (FP, 16), (BF, 8), (FP, 8)])
@pytest.mark.parametrize("scale", [4.0, -3.0, 1e-6, 0.0, 0.3])
@pytest.mark.parametrize("tree", [None, 3])
def test_scales(act, bits, scale, tree):
    """More than 64 columns per sequence on average (two of 170 rows, 2 heads)."""
    _case([(50, 33), (700, 137)], 32, 2, 2, 64, act, bits, tree, scale=scale, seed=5)


# the size of a query's and of a key's only channel
TIES = {(FP, 16): [(3.0, 5.0), (1500.0, 9000.0), (3001.0, 31008.0), (65504.0, 65504.0)],
        (BF, 16): [(3.0, 5.0), (2.0 ** 13, 2.0 ** 13), (2.0 ** 20, 2.0 ** 21), (2.0 ** 50, 2.0 ** 55)],
        (FP, 8): [(1500.0, 9000.0), (3001.0, 31008.0), (65504.0, 65504.0)],
        (BF, 8): [(2.0 ** 13, 2.0 ** 13), (2.0 ** 20, 2.0 ** 21), (2.0 ** 50, 2.0 ** 55)]}


@pytest.mark.parametrize("act,bits,size", [(a, b, s) for (a, b), sizes in TIES.items() for s in sizes])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("n,ctx", [(9, 600), (150, 600)])
def test_tied_scores_of_any_size(act, bits, size, D, sign, n, ctx):
    """Keys that tie in front of all others by half of their score, from the first
    position on: the output is the mean of their values, however large the score is.
    Tied keys are equal, so whatever the roundings of their scores, these are equal, too,
    and the weights are; the others' are below 2^-10 of the keys' (16 bits' unit at
    scores of 15) or nothing, and in the definition as well. Few columns and many."""
    g = _gen(n)
    L, amp_q, amp_k = ctx + n, *size
    tied = torch.zeros(L, dtype=torch.bool)
    tied[torch.tensor([0, 5, 31, 32, 100, 101, 333, ctx + 1, ctx + n - 1])] = True
    k, v = torch.zeros(L, 1, D), torch.randn(L, 1, D, generator=g)
    k[:, 0, 3] = torch.where(tied, 1.0, 0.5) * amp_k * sign
    q = torch.zeros(n, 4, D)
    # row by row another size, so another residue of the rounded score
    q[:, :, 3] = amp_q * (0.5 + 0.5 * torch.rand(n, 4, generator=g))
    q, k, v = q.to(act), k.to(act), v.to(act)
    nb = -(-L // 64)
    c = _cache(nb, 64, 1, D, act, bits)
    c.append(k.cuda(), v.cuda(), torch.arange(L).cuda())
    args = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, n], [list(range(nb))], [L])]
    lse = torch.empty(n, 4, device="cuda")
    out = c.attend_rows(q.cuda(), *args, L, scale=sign, lse=lse)
    o, e, mass, big = RR.attend(q, RR.cached(k, bits), RR.cached(v, bits), RR.seen(n, ctx), sign)
    # a score is one product and at most three factors, each rounded; it matters where
    # scores are small enough for the others to have weight, and then twice
    err = 4 * 2.0 ** -23 * torch.where(big < 200.0, big, 0.0)
    once = _once(n, 1, 4, act, bits)
    rel = 2 * err + (L + 64) * 2.0 ** -23 + 2.0 ** -15 + (R.U[once] if once else 0.0)
    _within(out, o, R.U[act] * (1 + 2 ** -8) * o.abs() + rel[..., None] * mass + 2 * R.TINY[act], "rows")
    # score and sum: eight roundings and the sum's
    _within(lse, e, 8 * 2.0 ** -24 * e.abs() + (L + 64) * 2.0 ** -23, "lse")
