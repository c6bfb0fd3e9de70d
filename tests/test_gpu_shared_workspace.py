"""Several layers' caches with one workspace: what each computes, eager and in captured
graphs, and what they hold together."""
import pytest
import torch

from paper_2607_16184_amd import ops
from test_gpu_ops import BF, _gen, _same

pytestmark = pytest.mark.gpu

SHAPES = [(2, 64, [4000, 3100], [7, 9]), (1, 128, [6000, 100], [300, 2]), (4, 256, [2500, 2600], [3, 3])]   # kv heads, head_dim, ..


def _layers(workspace):
    g, out = _gen(3), []
    for H, D, lens, new in SHAPES:
        nb = -(-max(lens) // 64)
        c = ops.KVCache(2 * nb, 64, H, D, BF, workspace=workspace)
        c.pool.view(BF).copy_(torch.randn(c.pool.numel() // 2, generator=g))
        starts = torch.tensor([0, new[0], sum(new)], dtype=torch.int32, device="cuda")
        table = torch.arange(2 * nb, dtype=torch.int32, device="cuda").view(2, nb)
        q = torch.randn(sum(new), 4 * H, D, generator=g).to(BF).cuda()
        out.append((c, q, starts, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), max(lens)))
    return out


def _step(layers, stream=None):
    rows = [c.attend_rows(q, s, t, n, L, stream=stream) for c, q, s, t, n, L in layers]
    return rows + [c.attend(q[:2], t, n, L, stream=stream) for c, q, _, t, n, L in layers]


def test_layers_with_one_workspace():
    alone, shared = _layers(None), ops.Workspace()
    want = _step(alone)
    need = [max(n for _, n in c._ws.of.values()) for c, *_ in alone]
    assert min(need) > 0 and len(set(need)) > 1
    layers = _layers(shared)
    for _ in range(3):
        assert all(_same(a, b) for a, b in zip(_step(layers), want))
    assert [n for _, n in shared.of.values()] == [max(need)] and sum(t.numel() for t in shared.kept) < 2 * max(need)
    # another stream, other buffers
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = _step(layers, side)
    again = _step(layers)
    side.synchronize()
    assert all(_same(a, b) and _same(a, c) for a, b, c in zip(want, got, again)) and len(shared.of) == 2
    # a step of all layers, captured; replays between eager steps on the same buffers' stream
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = _step(layers)
    for i in range(4):
        for c, q, *_ in layers:
            q.mul_(-1.0)
        flipped = _step(layers)
        for x in out:
            x.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(_same(a, b) for a, b in zip(out, flipped))
        assert i % 2 == 0 or all(_same(a, b) for a, b in zip(out, want))
