"""The decoder block on the GPU against its formula in 64 bits: prompts of
several sequences in one step, single tokens after them.

Bound on a row's relative error in norm. About eight 16-bit roundings lie between
the input and the output (projection, cache, attention, output projection, sum,
norm, expert rows, result), each of at most 2^-11 in fp16, and the norms and the
softmax scale relative errors by factors of order one: 4 x 8 x 2^-11 = 2^-6. An
8-bit cache stores the code next to the one of the exact keys where the roundings
before it pass a code boundary: of values off by 2^-12 of themselves, codes 2^-3
apart, one in 2^9, each by up to 2^-3, in norm 2^-3 / 2^4.5 < 2^-7 more."""
import numpy as np
import pytest
import torch

import oracle
import ops_ref as R
from paper_2607_16184_amd import synth

pytestmark = pytest.mark.gpu


def _reference(block, O, x, r, groups_of):
    """x, r [T, H] in 64 bits; groups_of: per row its sequence's keys and values
    so far, appended to here. Returns (y, z, ids)."""
    c, H = block.cache, x.shape[1]
    w = block.test_w
    z = x if r is None else x + r
    n = z / torch.sqrt((z * z).mean(-1, keepdim=True) + block.eps) * block.norm_attn.cpu().double()
    q8, qs = R.quant(n.float(), 128)
    qkv = ((q8.double() * qs.double().repeat_interleave(128, 1)) @ w.T).view(len(x), -1, c.head_dim)
    bits = c.desc.bits
    o = torch.zeros(len(x), block.heads, c.head_dim, dtype=torch.float64)
    for t, kv in enumerate(groups_of):
        kv[0].append(R.cached(qkv[t, block.heads:block.heads + c.kv_heads], bits))
        kv[1].append(R.cached(qkv[t, block.heads + c.kv_heads:], bits))
        o[t] = R.attend(qkv[t, :block.heads], torch.stack(kv[0]), torch.stack(kv[1]), len(kv[0]), c.head_dim ** -0.5, 0)[0]
    z = z + o.view(len(x), -1) @ block.w_o.cpu().double()
    h = z / torch.sqrt((z * z).mean(-1, keepdim=True) + block.eps) * block.norm_moe.cpu().double()
    opt = {k: v for k, v in block.routing.items() if k != "n_shared"}
    ids, wt = R.route((h @ block.w_router.cpu().double()).numpy(), block.K, **opt)
    n_sh = block.routing["n_shared"]
    all_ids = np.concatenate([ids, np.tile(np.arange(n_sh) + block.layer.cfg.E_routed, (len(x), 1))], 1).astype(np.int32)
    all_w = np.concatenate([wt, np.ones((len(x), n_sh))], 1).astype(np.float32)
    h16 = h.to(block.cache.act).view(torch.int16).numpy().view(np.uint16)
    return torch.from_numpy(O.forward(h16, all_ids, all_w, h_round=True)), z, ids


def _rel(a, b):
    return ((a.cpu().double() - b).norm(dim=-1) / b.norm(dim=-1))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("name,routing", [("tiny", dict()), ("tiny_shared", dict(score="sigmoid", groups=4, top_groups=2, scale=2.5))])
def test_prompt_and_single_tokens(name, routing, fp8):
    from paper_2607_16184_amd import decoder
    block = decoder.random_block(name, 24, fp8_cache=fp8, **routing)
    cfg = block.layer.cfg
    O = oracle.OracleLayer(cfg.E, cfg.H, cfg.F, cfg.R, cfg.G, cfg.act, cfg.sdt, [synth.expert_weights(cfg, p) for p in range(3)],
                           synth.bitmap(cfg))
    # the weights as the packed tiles hold them
    lin = block.qkv
    t = lin.packed.cpu().view(-1, cfg.H // 128, 2, 4, 16, 16)            # [row tile, block, half, piece, row, byte]
    codes = t.permute(0, 4, 1, 2, 3, 5).reshape(-1, cfg.H)[:lin.N].contiguous().view(R.F8)
    block.test_w = codes.double() * lin.w_scale.cpu().double().repeat_interleave(128, 0)[:lin.N].repeat_interleave(128, 1)
    tables = decoder.BlockTables(24, 32, 3, 200)
    kv = [([], []) for _ in range(3)]
    g = torch.Generator().manual_seed(9)
    bound = 2.0 ** -6 + (2.0 ** -7 if fp8 else 0.0)
    rows = same = 0
    for seqs, counts in [([0, 2], [45, 33]), ([0, 1, 2], [1, 20, 1]), ([2, 0], [1, 1]), ([1], [1])]:
        T = sum(counts)
        x, r = (torch.randn(T, cfg.H, generator=g).to(block.cache.act) for _ in range(2))
        r = r if len(seqs) > 1 else None
        y, z = block.step(x.cuda(), None if r is None else r.cuda(), *tables.step(seqs, counts), max_len=200)
        yr, zr, ids = _reference(block, O, x.double(), None if r is None else r.double(),
                                 [kv[s] for s, n in zip(seqs, counts) for _ in range(n)])
        assert (_rel(z, zr) <= bound).all()
        # the experts of a token may differ from the exact ones where their
        # scores do by less than the roundings; its output is then another one
        ok = _rel(y, yr) <= bound
        rows, same = rows + T, same + int(ok.sum())
    assert same >= 0.95 * rows, "%d of %d rows are within the bound" % (same, rows)
    block.layer.close()


def test_command_runs(capsys):
    from paper_2607_16184_amd import decoder
    decoder.main(["--layer", "tiny", "--batch", "5", "--prompt", "37", "--steps", "30", "--fp8-cache"])
    line = capsys.readouterr().out
    assert "5 sequences, 37 + 30 tokens" in line and "nan" not in line
