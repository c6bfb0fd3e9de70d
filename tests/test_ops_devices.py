"""Which device a call of the operators around the experts runs on, with
tensors that say they lie on device 0 or 1: no GPU is needed."""
import contextlib

import pytest
import torch

from paper_2607_16184_amd import ops, pw


class On(torch.Tensor):
    """A host tensor that names a device."""

    def get_device(self):
        return self.dev

    is_cuda = True


def _t(dev, *shape, dtype=torch.bfloat16):
    t = torch.zeros(shape, dtype=dtype).as_subclass(On)
    t.dev = dev
    return t


class Stream:
    def __init__(self, dev):
        self.device_index, self.cuda_stream = dev, 70 + dev


@pytest.fixture
def gpu(monkeypatch):
    """Device 0 is current; calls into the library are noted as (name, device that
    is current, stream)."""
    now, calls = [0], []

    @contextlib.contextmanager
    def device(d):
        now.append(d)
        yield
        now.pop()

    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: now[-1], raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 0, raising=False)
    for name in ("pw_rms_norm", "pw_gemm_fp8_pack", "pw_gemm_fp8", "pw_kv_append", "pw_attn_decode", "pw_route_grouped"):
        monkeypatch.setattr(pw, name, lambda *a, name=name: calls.append((name, now[-1], a[-1])))
    return calls


F8, F32, I32, I64 = torch.float8_e4m3fn, torch.float32, torch.int32, torch.int64
# every operator's tensors: (argument, shape, type)
NORM = [("x", (4, 256), torch.bfloat16), ("weight", (256,), torch.bfloat16), ("residual", (4, 256), torch.bfloat16),
        ("o0", (4, 256), torch.bfloat16), ("o1", (4, 256), torch.bfloat16), ("o2", (4, 256), F8), ("o3", (4, 2), F32)]
GEMM = [("w", (200, 256), F8), ("ws", (2, 2), F32), ("x", (4, 256), F8), ("xs", (4, 2), F32), ("out", (4, 200), torch.bfloat16)]
APPEND = [("pool", (4 * 32 * 2 * 2 * 64 * 2,), torch.uint8), ("k", (3, 2, 64), torch.bfloat16), ("v", (3, 2, 64), torch.bfloat16),
          ("slots", (3,), I64)]
ATTN = [APPEND[0], ("q", (3, 4, 64), torch.bfloat16), ("table", (3, 4), I32), ("lens", (3,), I32), ("out", (3, 4, 64), torch.bfloat16),
        ("lse", (3, 4), F32)]
ROUTE = [("logits", (5, 16), F32), ("bias", (16,), F32), ("gate", (5, 1), F32), ("o0", (5, 5), I32), ("o1", (5, 5), F32),
         ("o2", (18,), I32), ("o3", (25,), I32), ("o4", (25,), I32)]


def _norm(t, stream=None):
    ops.rms_norm(t["x"], t["weight"], t["residual"], out=tuple(t["o%d" % i] for i in range(4)), stream=stream)


def _gemm(t, stream=None):
    ops.Linear8(t["w"], t["ws"]).forward(t["x"], t["xs"], out=t["out"], stream=stream)


def _kv(t):
    return ops.KVCache(4, 32, 2, 64, torch.bfloat16, pool=t["pool"])


def _append(t, stream=None):
    _kv(t).append(t["k"], t["v"], t["slots"], stream=stream)


def _attend(t, stream=None):
    _kv(t).attend(t["q"], t["table"], t["lens"], 100, out=t["out"], lse=t["lse"], stream=stream)


def _route(t, stream=None):
    ops.route_grouped(t["logits"], 4, bias=t["bias"], n_shared=1, gate=t["gate"], out=tuple(t["o%d" % i] for i in range(5)),
                      stream=stream)


CALLS = [(_norm, NORM), (_gemm, GEMM), (_append, APPEND), (_attend, ATTN), (_route, ROUTE)]


def _make(spec, dev, other=None):
    return {n: _t(1 - dev if n == other else dev, *shape, dtype=dt) for n, shape, dt in spec}


@pytest.mark.parametrize("dev", [0, 1])
@pytest.mark.parametrize("fn,spec", CALLS)
def test_calls_run_on_the_tensors_device(gpu, fn, spec, dev):
    """The default stream's handle, 0, is that of the current device."""
    fn(_make(spec, dev))
    assert gpu and all(d == dev and st == 0 for _, d, st in gpu), gpu
    del gpu[:]
    fn(_make(spec, dev), stream=Stream(dev))
    assert gpu[-1][1:] == (dev, 70 + dev)


@pytest.mark.parametrize("dev", [0, 1])
@pytest.mark.parametrize("fn,spec,other", [(f, s, n) for f, s in CALLS for n, _, _ in s])
def test_tensors_of_two_devices_are_refused(gpu, fn, spec, other, dev):
    with pytest.raises(ValueError):
        fn(_make(spec, dev, other))
    assert all(name == "pw_gemm_fp8_pack" for name, _, _ in gpu)


@pytest.mark.parametrize("fn,spec", CALLS)
def test_streams_of_another_device_are_refused(gpu, fn, spec):
    with pytest.raises(ValueError):
        fn(_make(spec, 0), stream=Stream(1))
    assert all(name == "pw_gemm_fp8_pack" for name, _, _ in gpu)
