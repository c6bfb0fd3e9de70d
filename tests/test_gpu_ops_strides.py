"""Strides of dimensions of one: they say nothing, and any are taken."""
import pytest
import torch

from paper_2607_16184_amd import ops
from test_gpu_ops import BF, _gen, _same

pytestmark = pytest.mark.gpu


def _odd(t, dim, stride):
    """t with another stride in a dimension of one."""
    assert t.shape[dim] == 1
    return t.as_strided(t.shape, [stride if i == dim else x for i, x in enumerate(t.stride())])


@pytest.mark.parametrize("T,H", [(1, 2), (5, 1), (1, 1)])
def test_append_of_one_token_or_head(T, H):
    g = _gen(T + H)
    k, v = (torch.randn(T, H, 64, generator=g).to(BF).cuda() for _ in range(2))
    slots = torch.arange(T, device="cuda") * 3
    want, got = (ops.KVCache(1, 32, H, 64, BF) for _ in range(2))
    for c in (want, got):
        c.pool.zero_()
    want.append(k, v, slots)
    if T == 1:
        k, v = _odd(k, 0, 3), _odd(v, 0, 1000)
    if H == 1:
        k, v = _odd(k, 1, 7), _odd(v, 1, 64)
    got.append(k, v, slots)
    assert _same(want.pool, got.pool) and want.pool.any()


@pytest.mark.parametrize("B,heads", [(1, 2), (3, 1), (1, 1)])
def test_attention_of_one_sequence_or_head(B, heads):
    g = _gen(B + heads)
    c = ops.KVCache(B, 32, 1, 64, BF)
    c.pool.zero_()
    n = 20 * B
    kv = torch.randn(2, n, 1, 64, generator=g).to(BF).cuda()
    c.append(kv[0], kv[1], torch.arange(n, device="cuda") % 20 + torch.arange(n, device="cuda") // 20 * 32)
    q = torch.randn(B, heads, 64, generator=g).to(BF).cuda()
    table = torch.arange(B, dtype=torch.int32, device="cuda")[:, None]
    lens = torch.full((B,), 20, dtype=torch.int32, device="cuda")
    want = c.attend(q, table, lens, 20)
    if B == 1:
        q = _odd(q, 0, 5)
    if heads == 1:
        q = _odd(q, 1, 3)
    assert _same(want, c.attend(q, table, lens, 20)) and want.any()
