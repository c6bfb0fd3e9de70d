"""Appends of so many tokens and heads that runs are written as pieces of tiles,
and of as many as just are not: every byte of the pool against the header's layout."""
import numpy as np
import pytest
import torch

import ops_ref as R
from test_gpu_ops import BF, FP, _cache, _gen

pytestmark = pytest.mark.gpu


def _write(pool, k, v, slots, P, bits, n_blocks):
    """ops_ref.write_slots for all tokens at once (no slot twice)."""
    H, D = k.shape[1:]
    keep = (slots >= 0) & (slots < n_blocks * P)
    slots = slots[keep].numpy()
    stride = R.block_bytes(H, P, D, bits)
    t, h, d = (slots % P)[:, None, None], np.arange(H)[None, :, None], np.arange(D)[None, None, :]
    base = (slots // P * stride)[:, None, None]
    for i, x in enumerate((k[keep], v[keep])):
        at = base + (2 * h + i) * P * D * bits // 8 + (R.key_byte, R.value_byte)[i](t, d, D, bits)
        if bits == 16:
            b = x.contiguous().view(torch.uint8).numpy().reshape(*x.shape, 2)
            pool[at], pool[at + 1] = b[..., 0], b[..., 1]
        else:
            q, sc = R.quant(x, D)
            pool[at] = q.view(torch.uint8).numpy()
            so = (base + 2 * H * P * D + 4 * ((i * H + h) * P + t))[:, :, 0]
            b = sc[..., 0].contiguous().view(torch.uint8).numpy().reshape(*so.shape, 4)
            for j in range(4):
                pool[so + j] = b[..., j]


def _check(slots, n, P, H, D, act, bits, seed):
    kv = (torch.randn(len(slots), 2, H, D, generator=_gen(seed)) * 3).to(act)
    c = _cache(n, P, H, D, act, bits)
    dev = kv.cuda()
    c.append(dev[:, 0], dev[:, 1], slots.cuda())
    want = np.full(c.pool.numel(), 0xFF, np.uint8)
    _write(want, kv[:, 0], kv[:, 1], slots, P, bits, n)
    assert np.array_equal(c.pool.cpu().numpy(), want)


def test_write_as_the_definition():
    """The writer above against the tests' own, on the host."""
    g = _gen(1)
    kv, slots = torch.randn(9, 2, 3, 64, generator=g).to(BF), torch.tensor([5, -1, 63, 64, 200, 31, 32, 99, 1])
    for bits in (16, 8):
        a, b = (np.full(3 * R.block_bytes(3, 32, 64, bits), 0xFF, np.uint8) for _ in range(2))
        _write(a, kv[:, 0], kv[:, 1], slots, 32, bits, 3)
        R.write_slots(b, R.block_bytes(3, 32, 64, bits), kv[:, 0], kv[:, 1], slots, 32, bits, 3)
        assert np.array_equal(a, b)


@pytest.mark.parametrize("act", [BF, FP])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("D", [64, 128, 192, 256])
@pytest.mark.parametrize("H", [2, 24])
def test_runs_of_every_length(D, bits, act, H):
    """Whole tiles, runs that start and end anywhere in a tile, padding and lone
    tokens between them, runs past the last block, lone tokens backwards; tokens
    one by one (2 heads) and in pieces of tiles (24)."""
    P, n = 64, 60
    g = _gen(D)
    slots, at = [], 0
    for length in [40, 1, 7, 8, 9, 31, 32, 33, 64, 3, 2, 100, 5, 16, 17, 65, 150]:
        at += int(torch.randint(1, 50, (1,), generator=g))
        slots += list(range(at, at + length)) + ([-1] if length % 2 else [])
        at += length
    slots += list(range(n * P - 70, n * P + 30))
    slots += (torch.arange(40) * 3 + at).flip(0).tolist()
    slots = torch.tensor(slots)
    assert 16384 / 24 < len(slots) < 6144 / 2 and at + 120 < n * P - 70
    _check(slots, n, P, H, D, act, bits, D + H)


@pytest.mark.parametrize("bits,T,H", [(16, 511, 16), (16, 512, 12), (16, 512, 11), (16, 767, 8), (16, 768, 8), (16, 6144, 1), (16, 6143, 1),
                                      (8, 511, 40), (8, 512, 32), (8, 2047, 8), (8, 2048, 8)])
@pytest.mark.parametrize("P,first", [(32, 17), (128, 96)])
def test_around_the_first_runs(bits, T, H, P, first):
    n = (first + T) // P + 2
    blocks = torch.randperm(n, generator=_gen(T))
    pos = torch.arange(first, first + T)
    _check(blocks[pos // P] * P + pos % P, n, P, H, 64, BF, bits, T)
