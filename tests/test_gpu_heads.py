"""Norms of query and key heads with the position rotation, into rows and into the
paged cache, against their definitions in 64 bits (tests/rows_ref.py)."""
import math

import numpy as np
import pytest
import torch

import ops_ref as R
import rows_ref as RR
from test_gpu_ops import BF, FP, F8, _cache, _gen, _ops, _same, _within

pytestmark = pytest.mark.gpu


def _freq(dims, base=10000.0):
    return base ** (-torch.arange(0, dims, 2, dtype=torch.float64) / max(dims, 1))


def _check(got, x, pos, dims, inter, amp, norm, w, eps, what):
    want, mass = RR.heads(x, pos, _freq(dims), dims, inter, amp, norm, w, eps)
    rel = RR.heads_rel(x.shape[2], pos, _freq(dims))
    act = got.dtype
    _within(got, want, R.U[act] * (1 + 2 ** -8) * want.abs() + rel * mass + 2 * R.TINY[act], what)


def _run(T, n_q, n_k, D, dims, act, inter, amp=1.0, norm=True, weights=True, far=5000, seed=0, eps=1e-6, offset=0):
    g = _gen(seed)
    x = (torch.randn(T, n_q + n_k, D, generator=g) * torch.exp(torch.randn(T, 1, 1, generator=g))).to(act)
    w = [torch.randn(D, generator=g).to(act) if weights else None for _ in range(2)]
    pos = torch.randint(-far, far + 1, (T,), generator=g).int()
    rot = _ops().Rotation(dims, amplitude=amp, interleaved=inter)
    dev, wd = x.cuda(), [None if t is None else t.cuda() for t in w]
    q, k = _ops().norm_rotate(dev[:, :n_q], dev[:, n_q:] if n_k else None, pos.cuda(), rot, *wd, norm=norm, eps=eps, offset=offset)
    at = pos.long() + offset
    _check(q, x[:, :n_q], at, dims, inter, amp, norm, w[0], eps, "queries")
    if n_k:
        _check(k, x[:, n_q:], at, dims, inter, amp, norm, w[1], eps, "keys")
    return dev, pos, rot, wd, q, k


@pytest.mark.parametrize("act", [BF, FP])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D,dims", [(16, 16), (48, 32), (64, 64), (64, 16), (80, 80), (128, 128), (128, 64), (128, 96), (128, 0),
                                    (192, 192), (192, 64), (240, 176), (256, 256), (256, 48)])
def test_sizes(D, dims, inter, act):
    _run(3, 5, 2, D, dims, act, inter, amp=1.25, seed=D + dims)
    _run(1, 1, 1, D, dims, act, inter, norm=False, seed=D)
    _run(67, 3, 0, D, dims, act, inter, weights=False, seed=dims)


@pytest.mark.parametrize("T,n_q,n_k", [(1, 32, 8), (64, 32, 8), (200, 7, 1), (1000, 32, 8), (4097, 9, 2), (9000, 4, 4), (2, 1, 0)])
def test_batches(T, n_q, n_k):
    _run(T, n_q, n_k, 128, 128, BF, False, seed=T)
    _run(T, n_q, n_k, 64, 32, FP, True, norm=False, seed=T)


@pytest.mark.parametrize("far,offset", [(0, 0), (1 << 20, 0), ((1 << 31) - 1, 0), ((1 << 31) - 1, 1 << 30), (100, -1)])
def test_far_positions(far, offset):
    _run(300, 2, 1, 128, 128, FP, False, far=far, offset=offset, seed=3)
    _run(300, 2, 1, 64, 64, BF, True, norm=False, far=far, offset=offset, seed=4)


def test_small_angles_keep_their_bits():
    """A pair (0, y) becomes (-y sin, y cos): a small sine is correct to the output's
    rounding."""
    dims = 128
    x = torch.zeros(6, 1, dims)
    x[:, :, 64:] = 1.0
    pos = torch.tensor([1, 2, 3, 7, 100, 6283])
    q, _ = _ops().norm_rotate(x.to(FP).cuda(), None, pos.int().cuda(), _ops().Rotation(dims), norm=False)
    want = -torch.sin(pos.double()[:, None] * _freq(dims))
    _within(q[:, 0, :64], want, (R.U[FP] + 2.0 ** -20) * want.abs() + 2 * R.TINY[FP], "sines")


def test_strides_and_own_buffers():
    g = _gen(8)
    T, D = 37, 128
    x = torch.randn(T, 9, D + 8, generator=g).to(BF)
    pos = torch.arange(T) * 3
    rot = _ops().Rotation(D)
    wide = x.cuda()
    q, k = wide[:, 1:5, :D], wide[:, 5:7, :D]
    out = torch.full((4, T, D), 5.0, dtype=BF, device="cuda")     # heads outermost
    kept = torch.full((T, 4, D), 5.0, dtype=BF, device="cuda")
    _ops().norm_rotate(q, k, pos.int().cuda(), rot, out=(out.transpose(0, 1), kept[:, 1:3]))
    for got, part in ((out.transpose(0, 1), x[:, 1:5, :D]), (kept[:, 1:3], x[:, 5:7, :D])):
        _check(got, part, pos, D, False, 1.0, True, None, 1e-6, "strided")
    assert (kept[:, 0] == 5.0).all() and (kept[:, 3] == 5.0).all() and _same(wide.cpu(), x)
    _ops().norm_rotate(q, k, pos.int().cuda(), rot, out=(q, k))   # in place: the same bits, nothing else
    assert _same(q, out.transpose(0, 1)) and _same(k, kept[:, 1:3])
    wide[:, 1:7, :D] = x[:, 1:7, :D].cuda()
    assert _same(wide.cpu(), x)


def test_rows_that_hold_no_numbers_stay_alone():
    x = torch.randn(4, 3, 64, generator=_gen(2)).to(BF)
    x[1, 1, 5], x[2, 0, 40], x[3, 2] = math.nan, math.inf, 0.0
    pos = torch.tensor([4, 5, 6, 7])
    q, _ = _ops().norm_rotate(x.cuda(), None, pos.int().cuda(), _ops().Rotation(32))
    good = torch.ones(4, 3, dtype=torch.bool)
    good[1, 1] = good[2, 0] = False
    want, mass = RR.heads(x, pos, _freq(32), 32, False, 1.0, True, None, 1e-6)
    rel = RR.heads_rel(64, pos, _freq(32))
    _within(q.cpu()[good], want[good], R.U[BF] * (1 + 2 ** -8) * want[good].abs() + rel * mass[good] + 2 * R.TINY[BF], "others")
    assert torch.isnan(q[1, 1].float()).all() and torch.isnan(q[2, 0, 40].float()) and (q[3, 2] == 0).all()


def test_empty_batches():
    rot = _ops().Rotation(64)
    q, k = _ops().norm_rotate(torch.empty(0, 4, 64, dtype=BF, device="cuda"), torch.empty(0, 2, 64, dtype=BF, device="cuda"),
                              torch.empty(0, dtype=torch.int32, device="cuda"), rot)
    assert q.shape == (0, 4, 64) and k.shape == (0, 2, 64)


# ---------------------------------------------------------------------------
# Into the cache
# ---------------------------------------------------------------------------

def _append(T, n_q, H, D, dims, act, bits, inter=False, norm=True, amp=1.0, P=32, slots=None, n_blocks=None, seed=0, big=None):
    g = _gen(seed)
    x = torch.randn(T, n_q + 2 * H, D, generator=g)
    x = (x * (torch.exp(torch.randn(T, 1, 1, generator=g)) if big is None else big)).to(act)
    w = [torch.randn(D, generator=g).to(act) for _ in range(2)]
    pos = torch.randint(0, 20000, (T,), generator=g).int()
    if slots is None:
        n_blocks = 2 * T
        slots = torch.randperm(n_blocks, generator=g)[:T] * P + torch.randint(0, P, (T,), generator=g)
        slots[3::7] = -1
        slots[5::11] = n_blocks * P + 3
    c = _cache(n_blocks, P, H, D, act, bits)
    dev = x.cuda()
    q, k, v = dev.split([n_q, H, H], dim=1)
    got = c.append_rotated(k, v, slots.cuda(), pos.cuda(), _ops().Rotation(dims, amplitude=amp, interleaved=inter),
                           q if n_q else None, w[0].cuda(), w[1].cuda(), norm=norm, eps=1e-6)
    if n_q:
        _check(got, x[:, :n_q], pos.long(), dims, inter, amp, norm, w[0], 1e-6, "queries")
    else:
        assert got is None
    want, mass = RR.heads(x[:, n_q:n_q + H], pos.long(), _freq(dims), dims, inter, amp, norm, w[1], 1e-6)
    rel = RR.heads_rel(D, pos.long(), _freq(dims))
    pool = c.pool.cpu().numpy()
    # values, and the bytes of all other slots, as one written by the definition;
    # the keys' bytes are then taken over
    by_def = np.full(pool.size, 0xFF, np.uint8)
    R.write_slots(by_def, c.block_bytes, x[:, n_q:n_q + H], x[:, n_q + H:], slots, P, bits, n_blocks)
    d = np.arange(D)
    for n in range(T):
        s = int(slots[n])
        if s < 0 or s // P >= n_blocks:
            continue
        kk, _, ks, _ = RR.read_slot(pool, c.block_bytes, s, H, P, D, bits)
        if bits == 16:
            y = torch.from_numpy(kk.view(np.int16)).view(act)
            _within(y, want[n], R.U[act] * (1 + 2 ** -8) * want[n].abs() + rel * mass[n] + 2 * R.TINY[act], "keys of %d" % n)
        else:
            s64 = (want[n].abs().amax(-1) / 448).clamp_min(2.0 ** -126)
            _within(torch.from_numpy(ks), s64, rel * mass[n].amax(-1) / 448 + 2.0 ** -22 * s64, "scales of %d" % n)
            y = torch.from_numpy(kk).view(F8).double() * torch.from_numpy(ks).double()[:, None]
            _within(y, want[n], R.U[F8] * (1 + 2 ** -8) * want[n].abs() + 2 * rel * mass[n] + 1.001 * R.TINY[F8] * s64[:, None],
                    "keys of %d" % n)
        for h in range(H):
            at = s // P * c.block_bytes + 2 * h * P * D * bits // 8 + R.key_byte(s % P, d, D, bits)
            for b in range(bits // 8):
                by_def[at + b] = pool[at + b]
            if bits == 8:
                so = s // P * c.block_bytes + 2 * H * P * D + 4 * (h * P + s % P)
                by_def[so:so + 4] = pool[so:so + 4]
                at = s // P * c.block_bytes + (2 * h + 1) * P * D + R.value_byte(s % P, d, D, bits)
                by_def[at[(by_def[at] == 0x80) & (pool[at] == 0)]] = 0   # -0 as 0: the same value
    assert np.array_equal(pool, by_def), "values or other slots"
    return c, x, w, pos


@pytest.mark.parametrize("act", [BF, FP])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("D,dims,inter", [(64, 64, False), (64, 32, True), (128, 128, False), (128, 48, False), (128, 128, True),
                                          (192, 192, False), (192, 64, True), (256, 256, False), (256, 0, False)])
def test_append_sizes(D, dims, inter, bits, act):
    _append(9, 4, 2, D, dims, act, bits, inter, seed=D)
    _append(1, 3, 1, D, dims, act, bits, inter, norm=False, amp=0.75, seed=dims, P=64)
    _append(40, 0, 3, D, dims, act, bits, inter, seed=dims + 1)


def _runs(lengths, P, n_blocks, seed):
    """Slots of runs of these lengths at odd places, lone tokens and padding between."""
    g, out, at = _gen(seed), [], 0
    for n in lengths:
        at += int(torch.randint(1, 40, (1,), generator=g))
        out += list(range(at, at + n)) + ([-1] if n % 2 else [])
        at += n
    assert at < n_blocks * P
    return torch.tensor(out)


@pytest.mark.parametrize("act,bits", [(BF, 16), (FP, 8), (BF, 8)])
@pytest.mark.parametrize("D,dims,inter,norm,H", [(128, 128, False, True, 8), (64, 32, True, False, 16), (64, 64, False, True, 16),
                                                 (192, 128, False, True, 6), (256, 96, False, False, 5), (128, 48, False, True, 8),
                                                 (256, 256, True, True, 8)])
def test_append_runs_of_many_tokens(D, dims, inter, norm, H, act, bits):
    """Prefill chunks: runs that start and end inside tiles and blocks."""
    lengths = [700, 1, 31, 33, 7, 8, 9, 64, 500, 100, 3, 5, 150, 600]
    slots = _runs(lengths, 64, 60, D)
    _append(len(slots), 3, H, D, dims, act, bits, inter, norm, P=64, slots=slots, n_blocks=60, seed=D + dims)


@pytest.mark.parametrize("bits", [16, 8])
def test_append_in_place_equals_two_steps(bits):
    """The fused call and norm_rotate followed by append write the same queries, and
    in 16 bits the same cache."""
    g = _gen(5)
    T, n_q, H, D = 70, 6, 2, 128
    x = torch.randn(T, n_q + 2 * H, D, generator=g).to(BF).cuda()
    pos, slots = torch.arange(T, dtype=torch.int32).cuda() + 11, torch.arange(T).cuda() + 5
    rot, a, b = _ops().Rotation(D), _cache(4, 32, H, D, BF, bits), _cache(4, 32, H, D, BF, bits)
    q, k, v = x.split([n_q, H, H], dim=1)
    want_q, want_k = _ops().norm_rotate(q, k, pos, rot)
    a.append(want_k, v.contiguous(), slots)
    got = b.append_rotated(k, v, slots, pos - 3, rot, q, offset=3, q_out=q)
    assert got is q and _same(got, want_q)
    if bits == 16:
        assert torch.equal(a.pool, b.pool)
    else:                              # codes of the fp32 keys, not of rounded ones: values alike
        assert torch.equal(a.pool.view(4, -1)[:, 32 * D:2 * 32 * D], b.pool.view(4, -1)[:, 32 * D:2 * 32 * D])


def test_append_of_nothing_and_without_rotation():
    c = _cache(2, 32, 2, 64, BF, 16)
    before = c.pool.clone()
    e = torch.empty(0, 2, 64, dtype=BF, device="cuda")
    c.append_rotated(e, e, torch.empty(0, dtype=torch.int64, device="cuda"), None, None)
    assert torch.equal(c.pool, before)
    kv = torch.randn(3, 2, 2, 64, generator=_gen(1)).to(BF).cuda()
    slots = torch.tensor([0, 40, 33]).cuda()
    c.append_rotated(kv[:, 0], kv[:, 1], slots, None, None, norm=False)
    d = _cache(2, 32, 2, 64, BF, 16)
    d.append(kv[:, 0], kv[:, 1], slots)
    assert torch.equal(c.pool, d.pool)
