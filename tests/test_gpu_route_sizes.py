"""Grouped routing at the ends of its sizes, checked on the device."""
import pytest
import torch

from paper_2607_16184_amd import ops

pytestmark = pytest.mark.gpu


def test_route_almost_2_to_31_slots():
    """One routed and 255 shared experts: the last slots lie within a round of
    2^31, and every index follows from the formula."""
    T, E = (1 << 23) - 1, 256
    ids, w, off, ss, sp = ops.route_grouped(torch.zeros(T, 1, device="cuda"), 1, n_shared=255)
    e = torch.arange(E, device="cuda")
    assert torch.equal(off, (torch.arange(E + 1, device="cuda") * T).int())
    for a in range(0, T, 1 << 20):
        t = torch.arange(a, min(a + (1 << 20), T), device="cuda")
        assert (ids[t] == e).all() and (w[t] == 1.0).all()
        assert torch.equal(sp.view(T, E)[t], (e * T + t[:, None]).int())
        assert torch.equal(ss.view(E, T)[:, t], (t * E + e[:, None]).int())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_route_more_tokens_than_a_launch_takes(dtype):
    """2^26 tokens and some: more than 2^32 threads, a wave a token."""
    T = (1 << 26) + 5
    g = torch.Generator(device="cuda").manual_seed(1)
    logits = torch.randn(T, 2, generator=g, device="cuda").to(dtype)
    gate = torch.rand(T, 1, generator=g, device="cuda")
    ids, w, off, ss, sp = ops.route_grouped(logits, 1, score="sigmoid", renorm=False, n_shared=1, gate=gate)
    second = logits[:, 1] > logits[:, 0]
    assert torch.equal(ids[:, 0], second.int()) and (ids[:, 1] == 2).all() and torch.equal(w[:, 1:], gate)
    want = torch.sigmoid(logits.double().amax(1))
    assert ((w[:, 0] - want).abs() <= 2.0 ** -23 * want).all()            # 64 bits, rounded once
    n = int(second.sum())
    assert off.tolist() == [0, T - n, T, 2 * T]
    order = torch.cat([(~second).nonzero()[:, 0], second.nonzero()[:, 0]])
    assert torch.equal(ss[:T], (2 * order).int()) and torch.equal(ss[T:], (2 * torch.arange(T, device="cuda") + 1).int())
    assert torch.equal(sp[ss.long()], torch.arange(2 * T, device="cuda").int())
