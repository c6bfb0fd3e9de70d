"""Attention over the range of its scores: a key that takes nearly all of the
weight and has no value (an attention sink), so that the others' values alone
make the output. Bounds as in the other attention tests: relative to the weights
that make the output, however small they are."""
import pytest
import torch

import ops_ref as R
from test_gpu_ops import BF, FP, _cache, _gen, _within

pytestmark = pytest.mark.gpu


def _attend(k, v, q, P, act, bits, max_len=None):
    """k, v [B][n, H, D], q [B, heads, D] of type act, scale 1, through a cache:
    (out, lse)."""
    B, lens = len(k), [len(x) for x in k]
    H, D = k[0].shape[1:]
    nb = -(-max(lens) // P)
    c = _cache(B * nb, P, H, D, act, bits)
    table = torch.randperm(B * nb, generator=_gen(B)).int().view(B, nb)
    slots = torch.cat([table[b, torch.arange(n) // P].long() * P + torch.arange(n) % P for b, n in enumerate(lens)])
    c.append(torch.cat(k).cuda(), torch.cat(v).cuda(), slots.cuda())
    if max_len:                                                 # a longer bound and table
        table = torch.cat([table, torch.full((B, -(-max_len // P) - nb), -1, dtype=torch.int32)], 1)
    lse = torch.empty(B, q.shape[1], device="cuda")
    out = c.attend(q.cuda(), table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), max_len or max(lens), scale=1.0, lse=lse)
    return out, lse


def _check(out, lse, k, v, q, act, bits):
    D = q.shape[2]
    for b in range(len(k)):
        m = len(k[b])
        o, e, mass, size = R.attend(q[b], R.cached(k[b], bits), R.cached(v[b], bits), m, 1.0, 0)
        # scores: D products summed in fp32 and two scalings; weights: twice the
        # score's error, an exponential, a sum of m terms; values: the second
        # 16-bit term leaves 2^-16 of a weight
        ds = (D + 8) * 2.0 ** -23 * size
        rel = 2 * ds + (m + 64) * 2.0 ** -23 + 2.0 ** -15
        _within(out[b], o, R.U[act] * (1 + 2 ** -8) * o.abs() + rel[:, None] * mass + 2 * R.TINY[act], "row %d" % b)
        _within(lse[b], e, ds + (m + 64) * 2.0 ** -23 + 2.0 ** -21 * e.abs(), "lse %d" % b)


@pytest.mark.parametrize("act,bits", [(FP, 16), (BF, 16), (FP, 8)])
@pytest.mark.parametrize("D", [64, 128, 192, 256])
@pytest.mark.parametrize("lens,max_len", [([2, 20, 33, 300], None), ([4000], None), ([1500, 40, 7000], 40000)])
def test_sink_without_a_value(act, bits, D, lens, max_len):
    """The sink first, in the middle and last, 8 to 40 nats above the others, which
    tie or spread; values of size one and near the end of fp16."""
    g = _gen(D + len(lens))
    heads, ahead = 8, torch.tensor([8.0, 12.0, 14.0, 15.0, 17.0, 20.0, 27.0, 40.0])
    k, v = [], []
    for i, n in enumerate(lens):
        kb = torch.zeros(n, 2, D)
        kb[:, :, 2] = torch.randn(n, 2, generator=g) * (0.0, 2.0)[i % 2]
        vb = torch.randn(n, 2, D, generator=g)
        vb[:, 1] = (vb[:, 1].abs() + 1.0) * 8000.0              # the second key head: large, of one sign
        at = (0, n // 2, n - 1)[i % 3]
        kb[at] = 0.0
        kb[at, :, 1] = 8.0
        vb[at] = 0.0
        k.append(kb.to(act))
        v.append(vb.clamp(-6e4, 6e4).to(act))
    q = torch.zeros(len(lens), heads, D)
    q[:, :, 1] = torch.cat([ahead[0::2], ahead[1::2]]) / 8.0
    q[:, :, 2] = 1.0
    q = q.to(act)
    out, lse = _attend(k, v, q, 64, act, bits, max_len)
    _check(out, lse, k, v, q, act, bits)


def test_sink_before_equal_keys_in_one_workgroup():
    """2000 equal keys behind a sink, values of one: the output is their share of
    the weight. As many items as CUs, so that no other workgroup takes a part."""
    n, H, D = 2000, 128, 64
    k, v = torch.zeros(n, H, D), torch.ones(n, H, D)
    k[0, :, 0], v[0] = 1.0, 0.0
    q = torch.zeros(2, H, D)
    q[:, :, 0] = 8.0 + torch.arange(H) / 8.0
    k, v, q = k.to(FP), v.to(FP), q.to(FP)
    out, lse = _attend([k, k], [v, v], q, 64, FP, 16)
    _check(out, lse, [k, k], [v, v], q, FP, 16)


@pytest.mark.parametrize("act,bits", [(BF, 16), (BF, 8)])
@pytest.mark.parametrize("lens,max_len", [([1, 20, 33, 300], None), ([5000], None), ([1500, 40, 7000], 40000)])
def test_scores_near_the_lowest_number(act, bits, lens, max_len):
    """Scores of -2^105 and multiples of it, none above: the softmax is that of
    their differences, the lowest magnitude's tokens in equal parts."""
    g = _gen(len(lens))
    k, v = [], []
    for n in lens:
        kb = torch.randn(n, 2, 64, generator=g)
        kb[:, :, 1] = -2.0 ** 55 * (1 + torch.arange(n) % 4)[:, None]
        k.append(kb.to(act))
        v.append(torch.randn(n, 2, 64, generator=g).to(act))
    q = torch.zeros(len(lens), 4, 64)
    q[:, :, 1] = 2.0 ** 50
    q = q.to(act)
    out, lse = _attend(k, v, q, 64, act, bits, max_len)
    for b, n in enumerate(lens):
        vv = R.cached(v[b], bits)[::4].repeat_interleave(2, 1)
        o, mass = vv.mean(0), vv.abs().mean(0)
        _within(out[b], o, R.U[act] * (1 + 2 ** -8) * o.abs() + ((n + 64) * 2.0 ** -23 + 2.0 ** -15) * mass, "row %d" % b)
        _within(lse[b], torch.full((4,), -2.0 ** 105), torch.tensor(2.0 ** 105 * 2.0 ** -21), "lse %d" % b)
