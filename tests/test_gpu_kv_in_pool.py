"""KV blocks in the pages that a downshift freed: block numbers in units of 256
bytes over a layer's own pool."""
import numpy as np
import pytest
import torch

import ops_ref as R
from helpers import case, gpu_layer, to_dev, to_dev16
from paper_2607_16184_amd import ops, pw, synth
from test_gpu_ops import _gen, _within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [16, 8])
def test_blocks_lie_in_freed_pages(bits):
    cfg, w16, widths, order = case("tiny")
    layer = gpu_layer(cfg, w16, widths, order, slack=0.5)
    pages = [(e, p, rb) for p in range(3) for e in range(cfg.E) for rb in range(cfg.nrb(p)) if widths[p][e, rb] == 16][:6]
    freed = [(layer.entry(*x).data_off, pw.pw_page_bytes(cfg, x[1], 16)) for x in pages]
    layer.requant(pages, 4)
    layer.commit()
    torch.cuda.synchronize()
    layer.reclaim()
    x, logits = to_dev16(synth.activations(cfg)), to_dev(synth.logits(cfg))
    before = layer.forward(x, layer.route(logits, cfg.K)).clone()

    H, P, D, act = 2, 32, 64, torch.float16
    nb = R.block_bytes(H, P, D, bits)
    base = layer.pool_ptr - layer._pool_t.data_ptr()
    pool = layer._pool_t[base:base + layer.pool_bytes]
    n_blocks = (pool.numel() - nb) // 256 + 1
    cache = ops.KVCache(n_blocks, P, H, D, act, fp8=bits == 8, pool=pool, block_stride=256)
    held = [(off + i * nb) // 256 for off, n in freed for i in range(n // nb)]
    assert all(off % 256 == 0 for off, _ in freed) and len(set(held)) == len(held) > 6
    lens = [3 * P, 2 * P + 5, 7]
    g = _gen(bits)
    table = torch.tensor([held[0:3], held[3:6], held[-1:] + held[-1:] * 2], dtype=torch.int32)
    kv = torch.randn(sum(lens), 2, H, D, generator=g).to(act)
    q = torch.randn(3, 4, D, generator=g).to(act)
    slots = torch.cat([table[b, torch.arange(m) // P].long() * P + torch.arange(m) % P for b, m in enumerate(lens)])
    want = pool.cpu().numpy().copy()
    R.write_slots(want, 256, kv[:, 0], kv[:, 1], slots, P, bits, n_blocks)
    dev = kv.cuda()
    cache.append(dev[:, 0], dev[:, 1], slots.cuda())
    assert np.array_equal(pool.cpu().numpy(), want)            # nothing else of the pool is touched
    out = cache.attend(q.cuda(), table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), 3 * P)
    at = 0
    for b, m in enumerate(lens):
        o, _, mass, size = R.attend(q[b], R.cached(kv[at:at + m, 0], bits), R.cached(kv[at:at + m, 1], bits), m, D ** -0.5, 0)
        at += m
        # scores: D products summed in fp32 and two scalings; weights: twice the
        # score's error, an exponential, a sum of m terms and 2^-16 of themselves
        rel = 2 * (D + 8) * 2.0 ** -23 * size + (m + 64) * 2.0 ** -23 + 2.0 ** -15
        _within(out[b], o, R.U[act] * (1 + 2 ** -8) * o.abs() + rel[:, None] * mass + 2 * R.TINY[act], "row %d" % b)
    assert torch.equal(layer.forward(x, layer.route(logits, cfg.K)), before)
    layer.close()
