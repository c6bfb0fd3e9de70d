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
