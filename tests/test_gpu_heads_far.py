"""Rotations by angles that 64 bits no longer tell to a part of a turn: whatever their
sine and cosine are, values are turned, not stretched."""
import pytest
import torch

import ops_ref as R
import rows_ref as RR
from test_gpu_ops import BF, FP, _cache, _gen, _ops, _within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("freq", [2.0 ** 16, 1e6, 3.7e8, 1e13, 1e100])
@pytest.mark.parametrize("act", [BF, FP])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("T", [5, 2100])
def test_angles_past_64_bits(freq, act, inter, T):
    """An angle in 64 bits is off by 2^-53 of itself, so from 2^53 radians on nothing is
    known of it; sines and cosines stay within 1 all the same, and a pair's values
    within the sum of its magnitudes. As rows, and into the cache by tokens and runs."""
    g = _gen(T)
    x = torch.randn(T, 10, 64, generator=g).to(act)
    pos = torch.randint(-(1 << 31), (1 << 31) - 1, (T,), generator=g)
    inv = torch.full((32,), freq, dtype=torch.float64)
    inv[1], inv[5] = 0.25, -freq
    rot = _ops().Rotation(64, inv_freq=inv.cuda(), interleaved=inter)
    dev = x.cuda()
    q, _ = _ops().norm_rotate(dev[:, :2], None, pos.int().cuda(), rot, norm=False)
    nb = -(-T // 32)
    c = _cache(nb, 32, 8, 64, act, 16)
    c.append_rotated(dev[:, 2:], dev[:, 2:], torch.arange(T).cuda(), pos.int().cuda(), rot, norm=False)
    pool = c.pool.cpu().numpy()
    at = list(range(0, T, max(T // 40, 1)))
    keys = torch.stack([torch.from_numpy(RR.read_slot(pool, c.desc.block_stride, t, 8, 32, 64, 16)[0].view("int16").copy()).view(act)
                        for t in at])
    for got, part, p in ((q.cpu(), x[:, :2], pos), (keys, x[at][:, 2:], pos[at])):
        want, mass = RR.heads(part, p, inv, 64, inter, 1.0, False, None, 0.0)
        assert (got.double().abs() <= mass * (1 + 2.0 ** -7) + 2 * R.TINY[act]).all()
        i = [2, 3] if inter else [1, 33]                         # the pair whose angle is known
        rel = RR.heads_rel(64, p, torch.tensor([0.25]))
        _within(got[..., i], want[..., i], R.U[act] * (1 + 2 ** -8) * want[..., i].abs() + rel * mass[..., i] + 2 * R.TINY[act], "pair")
