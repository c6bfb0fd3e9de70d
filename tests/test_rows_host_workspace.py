"""Caches that share a workspace: their device (no GPU is needed)."""
import pytest
import torch

from paper_2607_16184_amd import ops
from test_ops_devices import _make, gpu  # noqa: F401
from test_rows_host import BF, POOL


def test_a_workspace_of_another_device_is_refused(gpu):  # noqa: F811
    pool = _make([POOL], 0)["pool"]
    for device in ("cpu", torch.device("cpu")):
        shared = ops.Workspace(device)
        a, b = (ops.KVCache(4, 32, 2, 64, BF, pool=pool, workspace=shared) for _ in range(2))
        assert a._ws is shared and b._ws is shared
    with pytest.raises(ValueError):
        ops.KVCache(4, 32, 2, 64, BF, pool=pool, workspace=ops.Workspace("meta"))
    assert ops.KVCache(4, 32, 2, 64, BF, pool=pool)._ws is not ops.KVCache(4, 32, 2, 64, BF, pool=pool)._ws
