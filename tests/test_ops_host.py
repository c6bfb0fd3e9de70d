"""Refusals and sizes of the operators around the experts: answered on the host
before any GPU work, so no GPU is needed."""
import numpy as np
import pytest
import torch

import ops_ref as R
from paper_2607_16184_amd import pw

A = 1 << 20          # an address that passes the alignment checks and is never read


def _refused(status, fn, *args):
    with pytest.raises(pw.PWError) as e:
        fn(*args)
    assert e.value.status == status, str(e.value)
    assert pw._lib.pw_last_error()


def _call(fn, order, base, **over):
    args = dict(base, **over)
    return lambda: fn(*(args[k] for k in order))


NORM = "x ldx r ldr w T H eps act s y q qs st".split()
NORM_OK = dict(x=A, ldx=256, r=A, ldr=256, w=A, T=4, H=256, eps=1e-5, act=pw.PW_BF16, s=A, y=A, q=A, qs=A, st=0)


@pytest.mark.parametrize("bad", [dict(T=-1), dict(H=0), dict(H=12), dict(H=32776, ldx=32776, ldr=32776), dict(act=2), dict(eps=-1.0),
                                 dict(eps=float("nan")), dict(eps=float("inf")), dict(ldx=248), dict(ldx=260), dict(ldr=255),
                                 dict(q=0), dict(qs=0), dict(H=264, ldx=264, ldr=264), dict(x=0), dict(x=A + 8), dict(r=A + 2),
                                 dict(w=A + 4), dict(s=A + 8), dict(y=A + 2), dict(q=A + 8), dict(qs=A + 2),
                                 dict(s=0, y=0, q=0, qs=0)])
def test_norm_refusals(bad):
    _refused(pw.PW_EINVAL, _call(pw.pw_rms_norm, NORM, NORM_OK, **bad))


GEMM = "a lda as_ w ws_ M N K y ldy t ws wsb st".split()
GEMM_OK = dict(a=A, lda=256, as_=A, w=A, ws_=A, M=4, N=100, K=256, y=A, ldy=100, t=pw.PW_BF16, ws=0, wsb=0, st=0)


@pytest.mark.parametrize("bad", [dict(M=-1), dict(N=0), dict(K=0), dict(K=192), dict(lda=255), dict(lda=264),
                                 dict(lda=(1 << 22) + 16), dict(K=(1 << 22) + 128, lda=(1 << 22) + 128), dict(ldy=99), dict(t=3), dict(t=-1), dict(a=0),
                                 dict(as_=0), dict(w=0), dict(ws_=0), dict(y=0), dict(a=A + 8), dict(w=A + 1), dict(as_=A + 2),
                                 dict(ws_=A + 1), dict(y=A + 1), dict(y=A + 2, t=pw.PW_F32)])
def test_gemm_refusals(bad):
    _refused(pw.PW_EINVAL, _call(pw.pw_gemm_fp8, GEMM, GEMM_OK, **bad))


PACK = "w ldw N K p st".split()
PACK_OK = dict(w=A, ldw=256, N=100, K=256, p=A, st=0)


@pytest.mark.parametrize("bad", [dict(N=0), dict(K=0), dict(K=200), dict(K=1 << 23, ldw=1 << 23), dict(ldw=255), dict(ldw=264),
                                 dict(w=0), dict(p=0), dict(w=A + 8), dict(p=A + 4), dict(N=1 << 30, K=1 << 14, ldw=1 << 14)])
def test_pack_refusals(bad):
    _refused(pw.PW_EINVAL, _call(pw.pw_gemm_fp8_pack, PACK, PACK_OK, **bad))


def test_packed_bytes():
    assert [pw.pw_gemm_fp8_packed_bytes(n, 256) for n in (1, 16, 17, 4000)] == [4096, 4096, 8192, 4000 * 256]
    _refused(pw.PW_EINVAL, pw.pw_gemm_fp8_packed_bytes, 1, 100)


def test_gemm_workspace():
    for bad in ((-1, 1, 128), (1, 0, 128), (1, 1, 100), (1, 1, 0)):
        _refused(pw.PW_EINVAL, pw.pw_gemm_fp8_workspace, *bad)
    assert pw.pw_gemm_fp8_workspace(0, 100, 128) == 0
    for M, N, K in ((1, 256, 4096), (16, 6144, 4096), (100, 512, 4096), (128, 640, 8192), (300, 4096, 14336)):
        need = pw.pw_gemm_fp8_workspace(M, N, K)
        if need:
            over = dict(M=M, N=N, K=K, lda=K, ldy=N)
            _refused(pw.PW_ENOMEM, _call(pw.pw_gemm_fp8, GEMM, GEMM_OK, **over))
            _refused(pw.PW_ENOMEM, _call(pw.pw_gemm_fp8, GEMM, GEMM_OK, ws=A, wsb=need - 1, **over))
            _refused(pw.PW_EINVAL, _call(pw.pw_gemm_fp8, GEMM, GEMM_OK, ws=A + 8, wsb=need, **over))


def _desc(**over):
    c = dict(pool=A, block_stride=1 << 20, n_blocks=4, block_tokens=32, n_kv_heads=2, head_dim=64, act=pw.PW_BF16, bits=16)
    c.update(over)
    return pw.pw_kv_cache(*(c[k] for k in ("pool", "block_stride", "n_blocks", "block_tokens", "n_kv_heads", "head_dim", "act",
                                           "bits")))


BAD_SHAPES = [dict(head_dim=96), dict(head_dim=0), dict(block_tokens=16), dict(block_tokens=48), dict(block_tokens=512),
              dict(n_kv_heads=0), dict(n_kv_heads=1025), dict(act=2), dict(bits=4)]
BAD_MEMORY = [dict(n_blocks=0), dict(block_stride=0), dict(block_stride=100), dict(block_stride=-256), dict(block_stride=1 << 40),
              dict(pool=0), dict(pool=A + 16)]


@pytest.mark.parametrize("D", [64, 128, 192, 256])
@pytest.mark.parametrize("bits", [16, 8])
def test_block_bytes(D, bits):
    for H, P in ((1, 32), (3, 64), (8, 256)):
        c = _desc(head_dim=D, bits=bits, n_kv_heads=H, block_tokens=P, pool=0, n_blocks=0)
        assert pw.pw_kv_block_bytes(c) == R.block_bytes(H, P, D, bits)
        assert R.block_bytes(H, P, D, bits) % 256 == 0


@pytest.mark.parametrize("D", [64, 128, 192, 256])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("P", [32, 128])
def test_layout_is_a_permutation(D, bits, P):
    t, d = np.meshgrid(np.arange(P), np.arange(D), indexing="ij")
    for f in (R.key_byte, R.value_byte):
        at = np.sort(f(t, d, D, bits).ravel())
        assert np.array_equal(at, np.arange(P * D) * (bits // 8))


APPEND = "c k v ld ldh slots T st".split()
APPEND_OK = dict(k=A, v=A, ld=512, ldh=64, slots=A, T=3, st=0)


@pytest.mark.parametrize("bad", BAD_SHAPES + BAD_MEMORY)
def test_cache_refusals(bad):
    _refused(pw.PW_EINVAL, _call(pw.pw_kv_append, APPEND, dict(APPEND_OK, c=_desc(**bad))))
    _refused(pw.PW_EINVAL, _call(pw.pw_attn_decode, ATTN, dict(ATTN_OK, c=_desc(**bad))))
    if bad in BAD_SHAPES:
        _refused(pw.PW_EINVAL, pw.pw_kv_block_bytes, _desc(**bad))
        _refused(pw.PW_EINVAL, pw.pw_attn_workspace, _desc(**bad), 1, 2, 10, 0)


@pytest.mark.parametrize("bad", [dict(T=-1), dict(T=(1 << 30) + 1), dict(ld=500), dict(ldh=4), dict(k=0), dict(v=0), dict(slots=0),
                                 dict(k=A + 8), dict(v=A + 2), dict(slots=A + 4)])
def test_append_refusals(bad):
    _refused(pw.PW_EINVAL, _call(pw.pw_kv_append, APPEND, dict(APPEND_OK, c=_desc()), **bad))


ATTN = "c q ldq ldqh hq tab ldt lens B max_len scale window out lse ws wsb st".split()
ATTN_OK = dict(q=A, ldq=512, ldqh=64, hq=8, tab=A, ldt=4, lens=A, B=2, max_len=128, scale=0.1, window=0, out=A, lse=0, ws=0, wsb=0,
               st=0)


@pytest.mark.parametrize("bad", [dict(hq=0), dict(hq=3), dict(B=-1), dict(max_len=-1), dict(max_len=2 ** 31 - 100), dict(window=-1),
                                 dict(ldq=4), dict(ldqh=60), dict(scale=float("nan")), dict(scale=float("inf")), dict(ldt=3),
                                 dict(ldt=0), dict(q=0), dict(tab=0), dict(lens=0), dict(out=0), dict(q=A + 8), dict(out=A + 8),
                                 dict(tab=A + 2), dict(lens=A + 1), dict(lse=A + 2)])
def test_attention_refusals(bad):
    _refused(pw.PW_EINVAL, _call(pw.pw_attn_decode, ATTN, dict(ATTN_OK, c=_desc()), **bad))


def test_attention_workspace():
    c = _desc()
    _refused(pw.PW_EUNSUPPORTED, pw.pw_attn_workspace, c, 1 << 22, 2, 128, 0)
    _refused(pw.PW_EUNSUPPORTED, _call(pw.pw_attn_decode, ATTN, dict(ATTN_OK, c=c), B=1 << 21))
    assert pw.pw_attn_workspace(c, 0, 8, 10 ** 6, 0) == 0
    assert pw.pw_attn_workspace(c, 4, 8, 0, 0) == 0
    need = pw.pw_attn_workspace(c, 1, 8, 100000, 0)
    assert need > 0
    over = dict(B=1, max_len=100000, ldt=4000)
    _refused(pw.PW_ENOMEM, _call(pw.pw_attn_decode, ATTN, dict(ATTN_OK, c=c), **over))
    _refused(pw.PW_ENOMEM, _call(pw.pw_attn_decode, ATTN, dict(ATTN_OK, c=c), ws=A, wsb=need - 1, **over))
    _refused(pw.PW_EINVAL, _call(pw.pw_attn_decode, ATTN, dict(ATTN_OK, c=c), ws=A + 8, wsb=need, **over))
    # a window bounds what is split
    assert pw.pw_attn_workspace(c, 1, 8, 10 ** 9, 64) <= need


ROUTE = "l lt b T E K sc G tg gt rn ws ns g ids w off ss sp st".split()
ROUTE_OK = dict(l=A, lt=pw.PW_F32, b=0, T=3, E=32, K=4, sc=0, G=4, tg=2, gt=2, rn=1, ws=1.0, ns=0, g=0, ids=A, w=A, off=A, ss=A, sp=A,
                st=0)


@pytest.mark.parametrize("bad", [dict(T=-1), dict(E=0), dict(K=0), dict(K=17), dict(E=257), dict(ns=-1), dict(E=256, ns=1), dict(lt=3),
                                 dict(sc=2), dict(G=0), dict(G=3), dict(E=130, G=65), dict(tg=0), dict(tg=5), dict(gt=0), dict(gt=3),
                                 dict(E=8, G=8, tg=3), dict(ws=float("inf")), dict(ws=float("nan")), dict(T=1 << 30), dict(off=0),
                                 dict(l=0), dict(ids=0), dict(w=0), dict(ss=0), dict(sp=0)])
def test_route_refusals(bad):
    _refused(pw.PW_EINVAL, _call(pw.pw_route_grouped, ROUTE, ROUTE_OK, **bad))


def test_nothing_to_do_is_no_error():
    pw.pw_rms_norm(0, 256, 0, 0, 0, 0, 256, 1e-5, pw.PW_F16, 0, 0, 0, 0, 0)
    pw.pw_gemm_fp8(0, 256, 0, 0, 0, 0, 10, 256, 0, 10, pw.PW_F32, 0, 0, 0)
    pw.pw_kv_append(_desc(), 0, 0, 64, 64, 0, 0, 0)
    pw.pw_attn_decode(_desc(), 0, 64, 64, 2, 0, 0, 0, 0, 0, 1.0, 0, 0, 0, 0, 0, 0)


def test_tensor_level_checks():
    """Shapes, types and strides are refused before a pointer is passed on."""
    from paper_2607_16184_amd import ops
    x = torch.zeros(4, 256, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        ops.rms_norm(x)                                          # not on the device
    with pytest.raises(ValueError):
        ops.rms_norm(x.float())
    with pytest.raises(ValueError):
        ops.Linear8(x, torch.zeros(1, 2))
    with pytest.raises(ValueError):
        ops.KVCache(4, 32, 1, 64, torch.float32)
    with pytest.raises(ValueError):
        ops.route_grouped(torch.zeros(4, 8), 2)
    with pytest.raises(pw.PWError):
        ops.KVCache(4, 32, 1, 96, torch.bfloat16)


@pytest.mark.parametrize("bad", [dict(M=(1 << 30) + 1), dict(M=(1 << 31) - 1), dict(N=(1 << 30) + 1, ldy=(1 << 31) - 1),
                                 dict(N=(1 << 31) - 1, ldy=(1 << 31) - 1)])
def test_gemm_sizes_whose_tiles_pass_32_bits(bad):
    """Sizes that the tile counts would overflow at are refused, K as small as it goes."""
    _refused(pw.PW_EINVAL, _call(pw.pw_gemm_fp8, GEMM, GEMM_OK, **bad))
    _refused(pw.PW_EINVAL, pw.pw_gemm_fp8_workspace, bad.get("M", 1), bad.get("N", 1), 128)
    if "N" in bad:
        _refused(pw.PW_EINVAL, pw.pw_gemm_fp8_packed_bytes, bad["N"], 128)


def test_route_tokens_that_pass_32_bits():
    _refused(pw.PW_EINVAL, _call(pw.pw_route_grouped, ROUTE, ROUTE_OK, K=1, T=(1 << 30) + 1))


def test_lds_exchanges_inside_a_wave_are_fenced():
    """Where lanes of a wave read what others wrote to LDS, without a workgroup
    barrier, the source asks for the order: the wave barrier alone says nothing of
    memory, and a test of today's code shows nothing of the next compiler's."""
    import pathlib
    import re
    csrc = pathlib.Path(pw.LIB_PATH).parent / "csrc"
    text = {p.name: p.read_text() for p in sorted(csrc.glob("*.h*"))}
    helper = re.search(r"void wave_exchange\(\) \{(.*?)\n\}", text["pw_device.hpp"], re.S).group(1)
    lines = [x.strip() for x in helper.strip().splitlines()]
    assert lines == ['__builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");', "__builtin_amdgcn_wave_barrier();",
                     '__builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");']
    assert {n: t.count("__builtin_amdgcn_wave_barrier") for n, t in text.items() if "__builtin_amdgcn_wave_barrier" in t} == {"pw_device.hpp": 1}
    # a turn through LDS: before the reads, and before the next writes
    assert {n: t.count("wave_exchange();") for n, t in text.items() if "wave_exchange();" in t} == {
        "pw_attn.hip": 2, "pw_gemm8.hip": 2, "pw_route.hip": 3}


B = A + (1 << 16)


@pytest.mark.parametrize("bad", [dict(x=B, ldx=512, s=B), dict(r=B, ldr=264, s=B), dict(x=B, ldx=264, y=B), dict(r=B, ldr=512, y=B),
                                 dict(s=B, y=B), dict(s=B, y=B, T=1)])
def test_norm_refuses_outputs_over_rows_that_are_not_packed(bad):
    """Output rows are packed: over an input with a longer stride they would be
    written where other rows are still to be read."""
    _refused(pw.PW_EINVAL, _call(pw.pw_rms_norm, NORM, dict(NORM_OK, x=A, r=2 * A, w=3 * A, s=4 * A, y=5 * A, q=6 * A, qs=7 * A), **bad))
