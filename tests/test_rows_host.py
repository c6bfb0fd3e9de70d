"""Refusals of the operators of several new tokens per sequence, and the device that
they run on: answered on the host, so no GPU is needed."""
import ctypes

import pytest
import torch

from paper_2607_16184_amd import ops, pw
from test_ops_devices import F32, I32, I64, Stream, _make, _t, gpu  # noqa: F401
from test_ops_host import A, _call, _desc, _refused

BF = torch.bfloat16


def _rot(dims=64, freq=A, amplitude=1.0, interleaved=0):
    return pw.pw_rotation(freq, dims, interleaved, amplitude)


HEADS = "rot pos off q ldq ldqh nq k ldk ldkh nk qw kw norm eps T D act qo ldqo ldqoh ko ldko ldkoh st".split()
HEADS_OK = dict(rot=_rot(), pos=A, off=0, q=A, ldq=256, ldqh=64, nq=4, k=A + 64, ldk=128, ldkh=64, nk=2, qw=A, kw=A, norm=1, eps=1e-6,
                T=3, D=64, act=pw.PW_BF16, qo=A + 4096, ldqo=256, ldqoh=64, ko=A + 8192, ldko=128, ldkoh=64, st=0)


@pytest.mark.parametrize("bad", [
    dict(T=-1), dict(nq=-1), dict(nk=-1), dict(D=8), dict(D=72), dict(D=272), dict(act=2), dict(norm=1, eps=-1.0),
    dict(eps=float("nan")), dict(eps=float("inf")), dict(rot=_rot(8)), dict(rot=_rot(-16)), dict(rot=_rot(80)),
    dict(rot=_rot(amplitude=float("inf"))), dict(rot=_rot(amplitude=float("nan"))), dict(rot=_rot(freq=0)), dict(rot=_rot(freq=A + 4)),
    dict(pos=0), dict(pos=A + 2), dict(q=0), dict(k=0), dict(qo=0), dict(ko=0), dict(q=A + 8), dict(k=A + 2), dict(qw=A + 4),
    dict(kw=A + 8), dict(qo=A + 4104), dict(ko=A + 8196), dict(ldq=260), dict(ldqh=60), dict(ldk=12), dict(ldkh=4), dict(ldqo=252),
    dict(ldqoh=68), dict(ldko=4), dict(ldkoh=12), dict(ldqo=248), dict(ldqoh=56), dict(ldko=0), dict(ldkoh=0),
    dict(ldqo=64, ldqoh=64), dict(qo=A), dict(qo=A, ldq=512), dict(qo=A + 64), dict(ko=A), dict(ko=A + 4096),
    dict(ldqo=1 << 62, ldqoh=1 << 62)])
def test_heads_refusals(bad):
    if bad == dict(qo=A):
        bad = dict(qo=A, ldqo=320)
    _refused(pw.PW_EINVAL, _call(pw.pw_heads_norm_rotate, HEADS, HEADS_OK, **bad))


def test_heads_too_many_and_none():
    _refused(pw.PW_EUNSUPPORTED, _call(pw.pw_heads_norm_rotate, HEADS, HEADS_OK, T=1 << 25))
    _refused(pw.PW_EUNSUPPORTED, _call(pw.pw_heads_norm_rotate, HEADS, HEADS_OK, T=1 << 24, nq=64, ldqo=4096))
    _call(pw.pw_heads_norm_rotate, HEADS, HEADS_OK, T=0, q=0, k=0, qo=0, ko=0)()
    _call(pw.pw_heads_norm_rotate, HEADS, HEADS_OK, nq=0, nk=0)()


APPEND = "c rot pos off q ldq ldqh nq k v ld ldh qw kw norm eps slots T qo ldqo ldqoh st".split()
APPEND_OK = dict(c=_desc(), rot=_rot(), pos=A, off=0, q=A, ldq=256, ldqh=64, nq=4, k=A + 512, v=A + 1024, ld=128, ldh=64, qw=A, kw=A,
                 norm=1, eps=1e-6, slots=A, T=3, qo=A + 4096, ldqo=256, ldqoh=64, st=0)


@pytest.mark.parametrize("bad", [
    dict(T=-1), dict(nq=-1), dict(c=_desc(head_dim=96)), dict(c=_desc(bits=4)), dict(c=_desc(pool=A + 128)), dict(c=_desc(n_blocks=0)),
    dict(eps=-1.0), dict(eps=float("nan")), dict(rot=_rot(24)), dict(rot=_rot(128)), dict(rot=_rot(amplitude=float("nan"))),
    dict(rot=_rot(freq=0)), dict(pos=0), dict(pos=A + 1), dict(k=0), dict(v=0), dict(slots=0), dict(slots=A + 4), dict(q=0),
    dict(qo=0), dict(q=A + 8), dict(k=A + 4), dict(v=A + 2), dict(qw=A + 8), dict(kw=A + 8), dict(qo=A + 4100), dict(ldq=12),
    dict(ldqh=4), dict(ld=12), dict(ldh=4), dict(ldqo=260), dict(ldqoh=60), dict(ldqo=64), dict(qo=A, ldqo=320), dict(qo=A + 512),
    dict(qo=A + 1024)])
def test_rotated_append_refusals(bad):
    _refused(pw.PW_EINVAL, _call(pw.pw_kv_append_rotated, APPEND, APPEND_OK, **bad))


def test_rotated_append_too_many_and_none():
    _refused(pw.PW_EUNSUPPORTED, _call(pw.pw_kv_append_rotated, APPEND, APPEND_OK, T=1 << 25))
    _refused(pw.PW_EUNSUPPORTED, _call(pw.pw_kv_append_rotated, APPEND, dict(APPEND_OK, c=_desc(n_kv_heads=64)), T=1 << 24))
    _call(pw.pw_kv_append_rotated, APPEND, APPEND_OK, T=0, k=0, v=0, slots=0)()


ROWS = "c q ldq ldqh nq starts T masks words table ldt lens B max_len scale window out lse ws wsb st".split()
ROWS_OK = dict(c=_desc(), q=A, ldq=256, ldqh=64, nq=4, starts=A, T=6, masks=A, words=1, table=A, ldt=4, lens=A, B=3, max_len=100, scale=0.1,
               window=0, out=A, lse=A, ws=0, wsb=0, st=0)


@pytest.mark.parametrize("bad", [
    dict(T=-1), dict(B=-1), dict(nq=3), dict(nq=0), dict(c=_desc(block_tokens=48)), dict(c=_desc(block_stride=100)), dict(words=0),
    dict(words=1025), dict(max_len=-1), dict(max_len=(1 << 31) - 200), dict(window=-1), dict(scale=float("inf")),
    dict(scale=float("nan")), dict(ldt=3), dict(q=0), dict(starts=0), dict(lens=0), dict(out=0), dict(table=0), dict(q=A + 8),
    dict(out=A + 8), dict(masks=A + 4), dict(starts=A + 2), dict(table=A + 2), dict(lens=A + 2), dict(lse=A + 2), dict(ldq=12),
    dict(ldqh=4)])
def test_rows_refusals(bad):
    _refused(pw.PW_EINVAL, _call(pw.pw_attn_rows, ROWS, ROWS_OK, **bad))


def test_rows_too_many_and_none():
    for over in (dict(B=65536), dict(T=1 << 21), dict(T=1 << 20, nq=8), dict(c=_desc(n_kv_heads=64), nq=64, B=65535, T=65536)):
        _refused(pw.PW_EUNSUPPORTED, _call(pw.pw_attn_rows, ROWS, ROWS_OK, **over))
    _call(pw.pw_attn_rows, ROWS, ROWS_OK, T=0, q=0)()
    _call(pw.pw_attn_rows, ROWS, ROWS_OK, B=0, q=0)()


def test_rows_workspace():
    for bad in ((-1, 1, 4, 100, 0), (1, -1, 4, 100, 0), (1, 1, 3, 100, 0), (1, 1, 4, -1, 0), (1, 1, 4, 100, -1)):
        _refused(pw.PW_EINVAL, pw.pw_attn_rows_workspace, _desc(), *bad)
    _refused(pw.PW_EUNSUPPORTED, pw.pw_attn_rows_workspace, _desc(), 65536, 1, 4, 100, 0)
    assert pw.pw_attn_rows_workspace(_desc(), 0, 5, 4, 100, 0) == 0 and pw.pw_attn_rows_workspace(_desc(), 5, 0, 4, 100, 0) == 0
    need = pw.pw_attn_rows_workspace(_desc(), 1, 8, 4, 100000, 0)
    assert need > 0
    over = dict(B=1, T=8, max_len=100000, ldt=100000 // 32 + 1)
    _refused(pw.PW_ENOMEM, _call(pw.pw_attn_rows, ROWS, ROWS_OK, **over))
    _refused(pw.PW_ENOMEM, _call(pw.pw_attn_rows, ROWS, ROWS_OK, ws=A, wsb=need - 1, **over))
    _refused(pw.PW_EINVAL, _call(pw.pw_attn_rows, ROWS, ROWS_OK, ws=A + 8, wsb=need, **over))


def test_rows_workspace_stays_small_for_long_bounds():
    """A bound of a million tokens for a batch of trees: the parts of a few rounds of
    workgroups, not of every piece that such lengths would have."""
    big = _desc(n_kv_heads=8, head_dim=128, block_stride=1 << 22)
    for B, T in ((16, 960), (64, 1100), (190, 60 * 190), (1, 64), (1, 4096), (64, 64 * 16)):
        assert pw.pw_attn_rows_workspace(big, B, T, 32, 1 << 20, 0) < 3 << 30


KEEP = "c starts table ldt lens B max_len chosen words new st".split()
KEEP_OK = dict(c=_desc(), starts=A, table=A, ldt=4, lens=A, B=3, max_len=100, chosen=A, words=1, new=A + 64, st=0)


@pytest.mark.parametrize("bad", [dict(B=-1), dict(max_len=-1), dict(max_len=(1 << 31) - 200), dict(words=0), dict(words=1025), dict(ldt=3),
                                 dict(c=_desc(head_dim=100)), dict(c=_desc(n_blocks=0)), dict(starts=0), dict(table=0), dict(lens=0),
                                 dict(chosen=0), dict(new=0), dict(new=A), dict(starts=A + 2), dict(table=A + 1), dict(lens=A + 2),
                                 dict(chosen=A + 4), dict(new=A + 66)])
def test_keep_refusals(bad):
    _refused(pw.PW_EINVAL, _call(pw.pw_kv_keep, KEEP, KEEP_OK, **bad))


def test_keep_too_many_and_none():
    _refused(pw.PW_EUNSUPPORTED, _call(pw.pw_kv_keep, KEEP, KEEP_OK, B=65536))
    _call(pw.pw_kv_keep, KEEP, KEEP_OK, B=0, starts=0)()


# ---------------------------------------------------------------------------
# On tensors
# ---------------------------------------------------------------------------

@pytest.fixture
def calls(gpu, monkeypatch):  # noqa: F811
    for name in ("pw_heads_norm_rotate", "pw_kv_append_rotated", "pw_attn_rows", "pw_kv_keep"):
        monkeypatch.setattr(pw, name, lambda *a, name=name: gpu.append((name, torch._C._cuda_getDevice(), a[-1])))
    return gpu


POOL = ("pool", (4 * 32 * 2 * 2 * 64 * 2,), torch.uint8)
FREQ, POS = ("freq", (32,), torch.float64), ("pos", (3,), I32)
TABLE = [("starts", (3,), I32), ("table", (2, 4), I32), ("lens", (2,), I32)]
HEADS_T = [FREQ, POS, ("q", (3, 4, 64), BF), ("k", (3, 2, 64), BF), ("qw", (64,), BF), ("kw", (64,), BF), ("qo", (3, 4, 64), BF),
           ("ko", (3, 2, 64), BF)]
APPEND_T = [POOL, FREQ, POS, ("q", (3, 4, 64), BF), ("k", (3, 2, 64), BF), ("v", (3, 2, 64), BF), ("slots", (3,), I64), ("qw", (64,), BF),
            ("kw", (64,), BF), ("qo", (3, 4, 64), BF)]
ROWS_T = [POOL, *TABLE, ("q", (3, 4, 64), BF), ("masks", (3, 1), I64), ("out", (3, 4, 64), BF), ("lse", (3, 4), F32)]
KEEP_T = [POOL, *TABLE, ("chosen", (2, 1), I64), ("new", (2,), I32)]


def _kv(t):
    return ops.KVCache(4, 32, 2, 64, BF, pool=t["pool"])


def _rotation(t):
    return ops.Rotation(64, inv_freq=t["freq"])


def _heads(t, stream=None, **over):
    a = dict(t, **over)
    ops.norm_rotate(a["q"], a["k"], a["pos"], _rotation(t), a["qw"], a["kw"], out=(a["qo"], a["ko"]), stream=stream)


def _append(t, stream=None, **over):
    a = dict(t, **over)
    _kv(t).append_rotated(a["k"], a["v"], a["slots"], a["pos"], _rotation(t), a["q"], a["qw"], a["kw"], q_out=a["qo"], stream=stream)


def _rows(t, stream=None, **over):
    a = dict(t, **over)
    _kv(t).attend_rows(a["q"], a["starts"], a["table"], a["lens"], 100, masks=a["masks"], out=a["out"], lse=a["lse"], stream=stream)


def _keep(t, stream=None, **over):
    a = dict(t, **over)
    _kv(t).keep(a["starts"], a["table"], a["lens"], 100, a["chosen"], out=a["new"], stream=stream)


CALLS = [(_heads, HEADS_T), (_append, APPEND_T), (_rows, ROWS_T), (_keep, KEEP_T)]


@pytest.mark.parametrize("dev", [0, 1])
@pytest.mark.parametrize("fn,spec", CALLS)
def test_calls_run_on_the_tensors_device(calls, fn, spec, dev):
    fn(_make(spec, dev))
    assert calls and all(d == dev and st == 0 for _, d, st in calls), calls
    del calls[:]
    fn(_make(spec, dev), stream=Stream(dev))
    assert calls[-1][1:] == (dev, 70 + dev)


@pytest.mark.parametrize("dev", [0, 1])
@pytest.mark.parametrize("fn,spec,other", [(f, s, n) for f, s in CALLS for n, _, _ in s])
def test_tensors_of_two_devices_are_refused(calls, fn, spec, other, dev):
    with pytest.raises(ValueError):
        fn(_make(spec, dev, other))
    assert not calls


@pytest.mark.parametrize("fn,spec", CALLS)
def test_streams_of_another_device_are_refused(calls, fn, spec):
    with pytest.raises(ValueError):
        fn(_make(spec, 0), stream=Stream(1))
    assert not calls


@pytest.mark.parametrize("fn,spec,name,shape,dtype", [
    (_heads, HEADS_T, "q", (3, 4, 32), BF), (_heads, HEADS_T, "k", (4, 2, 64), BF), (_heads, HEADS_T, "k", (3, 2, 64), torch.float16),
    (_heads, HEADS_T, "pos", (3,), I64), (_heads, HEADS_T, "pos", (2,), I32), (_heads, HEADS_T, "qw", (32,), BF),
    (_heads, HEADS_T, "kw", (64,), F32), (_heads, HEADS_T, "qo", (3, 2, 64), BF), (_heads, HEADS_T, "ko", (3, 2, 64), F32),
    (_append, APPEND_T, "k", (3, 1, 64), BF), (_append, APPEND_T, "v", (2, 2, 64), BF), (_append, APPEND_T, "v", (3, 2, 64), F32),
    (_append, APPEND_T, "slots", (3,), I32), (_append, APPEND_T, "pos", (4,), I32), (_append, APPEND_T, "q", (2, 4, 64), BF),
    (_append, APPEND_T, "qo", (3, 3, 64), BF), (_append, APPEND_T, "qw", (128,), BF),
    (_rows, ROWS_T, "q", (3, 4, 128), BF), (_rows, ROWS_T, "q", (3, 4, 64), torch.float16), (_rows, ROWS_T, "starts", (2,), I32),
    (_rows, ROWS_T, "starts", (3,), I64), (_rows, ROWS_T, "lens", (3,), I32), (_rows, ROWS_T, "table", (3, 4), I32),
    (_rows, ROWS_T, "table", (2, 3), I32), (_rows, ROWS_T, "table", (2, 4), I64), (_rows, ROWS_T, "masks", (2, 1), I64),
    (_rows, ROWS_T, "masks", (3, 1), I32), (_rows, ROWS_T, "out", (3, 4, 64), F32), (_rows, ROWS_T, "lse", (3, 2), F32),
    (_keep, KEEP_T, "starts", (2,), I32), (_keep, KEEP_T, "lens", (2,), I64), (_keep, KEEP_T, "chosen", (3, 1), I64),
    (_keep, KEEP_T, "chosen", (2, 1), I32), (_keep, KEEP_T, "new", (3,), I32), (_keep, KEEP_T, "new", (2,), I64)])
def test_shapes_and_types_are_refused(calls, fn, spec, name, shape, dtype):
    with pytest.raises(ValueError):
        fn(_make(spec, 0), **{name: _t(0, *shape, dtype=dtype)})
    assert not calls


def test_positions_and_frequencies_are_refused(calls):
    with pytest.raises(ValueError):
        _heads(_make(HEADS_T, 0), pos=None)
    for dims, freq in ((24, None), (-16, None), (64, _t(0, 16, dtype=torch.float64)), (64, torch.zeros(32))):
        with pytest.raises(ValueError):
            ops.Rotation(dims, inv_freq=freq)
    strided = _t(0, 3, 2, 128)[..., ::2]
    strided.dev = 0
    with pytest.raises(ValueError):
        _heads(_make(HEADS_T, 0), k=strided)
    assert not calls


def test_masks_without_words_are_refused(calls):
    with pytest.raises(ValueError):
        _rows(_make(ROWS_T, 0), masks=_t(0, 3, 0, dtype=I64))
    assert not calls


def test_limits_are_the_ones_stated():
    _refused(pw.PW_EUNSUPPORTED, _call(pw.pw_heads_norm_rotate, HEADS, HEADS_OK, T=1 << 24))
    _refused(pw.PW_EUNSUPPORTED, _call(pw.pw_heads_norm_rotate, HEADS, HEADS_OK, T=1 << 23, nq=62, ldqo=62 * 64))
    _refused(pw.PW_EUNSUPPORTED, _call(pw.pw_kv_append_rotated, APPEND, APPEND_OK, T=1 << 24))


def test_structure_matches_the_header():
    assert ctypes.sizeof(pw.pw_rotation) == 24
