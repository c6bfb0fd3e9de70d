"""The decoder block's steps by sequences: head norms and rotation on the way into the
cache, prompt chunks, trees of drafted tokens and the accepted ones kept. Bound on a
row's relative error in norm as in the decoder block's other tests."""
import pytest
import torch

import ops_ref as R
import rows_ref as RR
from test_gpu_decoder import _rel

pytestmark = pytest.mark.gpu
BOUND = 2.0 ** -6


def _weights(block):
    """The projection as its packed tiles hold it, in 64 bits."""
    lin, H = block.qkv, block.layer.cfg.H
    t = lin.packed.cpu().view(-1, H // 128, 2, 4, 16, 16)
    codes = t.permute(0, 4, 1, 2, 3, 5).reshape(-1, H)[:lin.N].contiguous().view(R.F8)
    return codes.double() * lin.w_scale.cpu().double().repeat_interleave(128, 0)[:lin.N].repeat_interleave(128, 1)


def _before_experts(block, w, x, pos, seen_of, history):
    """The residual after attention, in 64 bits: x [T, H]; seen_of [rows, history]
    per row; history: keys and values so far, these rows' appended."""
    c = block.cache
    z = x.double()
    n = z / torch.sqrt((z * z).mean(-1, keepdim=True) + block.eps) * block.norm_attn.cpu().double()
    q8, qs = R.quant(n.float(), 128)
    qkv = ((q8.double() * qs.double().repeat_interleave(128, 1)) @ w.T).view(len(x), -1, c.head_dim)
    q, k, v = qkv.split([block.heads, c.kv_heads, c.kv_heads], 1)
    freq, dims = block.rotate.inv_freq.cpu(), block.rotate.dims
    turn = lambda t, weight: RR.heads(t, pos, freq, dims, block.rotate.interleaved, 1.0, block.head_norm,  # noqa: E731
                                      None if weight is None else weight.cpu(), block.eps)[0]
    q, k = turn(q, block.q_norm), turn(k, block.k_norm)
    keys = torch.cat([history[0], k]) if len(history[0]) else k
    values = torch.cat([history[1], v]) if len(history[1]) else v
    o = RR.attend(q, keys, values, seen_of, c.head_dim ** -0.5)[0]
    return z + o.reshape(len(x), -1) @ block.w_o.cpu().double(), k, v


@pytest.mark.parametrize("inter,norms", [(False, True), (True, False)])
def test_chunks_trees_and_kept_tokens(inter, norms):
    from paper_2607_16184_amd import decoder, ops
    g = torch.Generator().manual_seed(4)
    D, act = 64, torch.float16
    head = [(1 + 0.1 * torch.randn(D, generator=g)).to(act).cuda() if norms else None for _ in range(2)]
    block = decoder.random_block("tiny", 20, rotate=ops.Rotation(D, interleaved=inter), q_norm=head[0], k_norm=head[1])
    w, H = _weights(block), block.layer.cfg.H
    tables = decoder.BlockTables(20, 32, 3, 200)
    hist = [[torch.zeros(0, block.cache.kv_heads, D, dtype=torch.float64) for _ in range(2)] for _ in range(3)]
    draw = lambda n: torch.randn(n, H, generator=g).to(act)  # noqa: E731

    def check(x, z, seqs, counts, pos, seen):
        at = 0
        out = []
        for i, (s, n) in enumerate(zip(seqs, counts)):
            zr, k, v = _before_experts(block, w, x[at:at + n], pos[at:at + n].cpu(), seen[i], hist[s])
            assert (_rel(z[at:at + n], zr) <= BOUND).all()
            out.append((k, v))
            at += n
        return out

    for seqs, counts in [([0, 2], [70, 33]), ([2, 0, 1], [40, 1, 50])]:        # prompts, in chunks
        x = draw(sum(counts))
        args = tables.rows(seqs, counts)
        _, z = block.step(x.cuda(), None, **args, max_len=200)
        seen = [RR.seen(n, len(hist[s][0])) for s, n in zip(seqs, counts)]
        for s, kv in zip(seqs, check(x, z, seqs, counts, args["positions"], seen)):
            hist[s] = [torch.cat([a, b]) for a, b in zip(hist[s], kv)]
    x = draw(3)                                                               # a token each, by rows
    args = tables.step([0, 1, 2], [1, 1, 1])
    _, z = block.step(x.cuda(), None, *args, max_len=200)
    for s, kv in enumerate(check(x, z, [0, 1, 2], [1] * 3, args[1] - 1, [RR.seen(1, len(hist[s][0])) for s in range(3)])):
        hist[s] = [torch.cat([a, b]) for a, b in zip(hist[s], kv)]
    sees = [1, 2, 1 | 4, 1 | 8, 2 | 16, 1 | 4 | 32]                           # 0 and 1; 2, 3 after 0; 4 after 1; 5 after 2
    depth = [bin(m).count("1") - 1 for m in sees]
    for path in (sees[5], sees[4], 0):
        x = draw(18)
        args = tables.rows([0, 1, 2], [6] * 3, [depth] * 3)
        masks = torch.tensor(sees * 3)[:, None]
        _, z = block.step(x.cuda(), None, **args, max_len=200, masks=masks.cuda())
        seen = [RR.seen(6, len(hist[s][0]), masks[:6]) for s in range(3)]
        kept = block.cache.keep(args["starts"], args["block_table"], args["lens"], 200, torch.tensor([[path]] * 3).cuda())
        for s, kv in enumerate(check(x, z, [0, 1, 2], [6] * 3, args["positions"], seen)):
            js = [j for j in range(6) if path >> j & 1]
            hist[s] = [torch.cat([a, b[js]]) for a, b in zip(hist[s], kv)]
            tables.truncate(s, int(kept[s]))
            assert int(kept[s]) == len(hist[s][0])
    block.layer.close()


def test_a_rotation_as_a_function_and_as_an_operator_agree():
    """A callback that turns rows with norm_rotate, and the rotation given as itself:
    the same queries and keys, so the same outputs."""
    from paper_2607_16184_amd import decoder, ops
    rot = ops.Rotation(64)
    out = []
    for which in (0, 1):
        block = decoder.random_block("tiny", 10, seed=3)

        def turn(qkv, lens, block=block):
            q, k = qkv[:, :block.heads], qkv[:, block.heads:block.heads + block.cache.kv_heads]
            ops.norm_rotate(q, k, lens, rot, norm=False, offset=-1, out=(q, k))

        block.rotate = (turn, rot)[which]
        tables = decoder.BlockTables(10, 32, 2, 100)
        g = torch.Generator().manual_seed(1)
        for counts in ([50, 20], [1, 1]):
            x = torch.randn(sum(counts), 256, generator=g).half().cuda()
            y, z = block.step(x, None, *tables.step([0, 1], counts), max_len=100)
        out.append((y, z))
        block.layer.close()
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])


def test_refusals():
    from paper_2607_16184_amd import decoder, ops
    block = decoder.random_block("tiny", 4)
    tables = decoder.BlockTables(4, 32, 1, 64)
    x = torch.zeros(2, 256, dtype=torch.float16, device="cuda")
    args = tables.rows([0], [2])
    plain = [args[n] for n in ("block_table", "lens", "slots")]
    with pytest.raises(ValueError):
        block.step(x, None, *plain, 64, args["starts"])
    with pytest.raises(ValueError):
        block.step(x, None, *plain, 64, masks=torch.ones(2, 1, dtype=torch.int64, device="cuda"))
    block.layer.close()
    with pytest.raises(ValueError):
        decoder.random_block("tiny", 4, rotate=lambda qkv, lens: None, q_norm=torch.ones(64, dtype=torch.float16, device="cuda"))


@pytest.mark.parametrize("extra", [["--rotate", "--draft", "7"], ["--draft", "1"], ["--rotate", "--fp8-cache"], ["--draft", "64", "--steps", "3"]])
def test_command_runs(capsys, extra):
    from paper_2607_16184_amd import decoder
    decoder.main(["--layer", "tiny", "--batch", "5", "--prompt", "37", "--steps", "9"] + extra)
    out = capsys.readouterr().out
    assert "5 sequences, 37 + " in out and "nan" not in out and ("kept" in out) == ("--draft" in extra)
