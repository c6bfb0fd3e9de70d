"""Operators around the experts on the GPU against their definitions in 64 bits
(tests/ops_ref.py). Bounds are first-order error bounds: U of the output's type
for its one rounding, and for fp32 sums of n terms n 2^-23 of the terms'
magnitudes (twice the unit roundoff, whatever the order of summation)."""
import math

import numpy as np
import pytest
import torch

import ops_ref as R
from paper_2607_16184_amd import pw

pytestmark = pytest.mark.gpu
BF, FP, F32, F8 = torch.bfloat16, torch.float16, torch.float32, R.F8


def _ops():
    from paper_2607_16184_amd import ops
    return ops


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _same(a, b):
    """Equal bit for bit (a NaN equals itself)."""
    t = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[a.element_size()]
    return a.shape == b.shape and torch.equal(a.contiguous().view(t), b.contiguous().view(t))


def _within(got, want, bound, what):
    got, want = got.detach().cpu().double(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what + ": NaN in other places"
    bad = ((got - want).abs() > bound) & ~torch.isnan(want) & (got != want)
    assert not bad.any(), "%s: %d of %d out of bounds, first at %s: %r against %r" % (
        what, int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist(), got[bad][0].item(), want[bad][0].item())


# ---------------------------------------------------------------------------
# Norm
# ---------------------------------------------------------------------------

def _check_norm(out, x, r, w, eps):
    s, y, q, qs = out
    z64, y64 = R.norm(x, r, w, eps)
    H = x.shape[1]
    # the mean square is a sum of H terms, halved by the square root; the rest
    # is a handful of fp32 operations
    rel = (H / 2 + 16) * 2.0 ** -23
    if s is not None:
        _within(s, z64, R.U[x.dtype] * (1 + 2 ** -10) * z64.abs() + 2 * R.TINY[x.dtype], "sum")
    if y is not None:
        _within(y, y64, (R.U[x.dtype] * (1 + rel) + rel) * y64.abs() + 2 * R.TINY[x.dtype], "y16")
    if q is not None:
        s64 = (y64.unflatten(-1, (-1, 128)).abs().amax(-1) / 448).clamp_min(2.0 ** -126)
        _within(qs, s64, (rel + 2 ** -22) * s64, "scales")
        v = q.cpu().double().unflatten(-1, (-1, 128)) * qs.cpu().double()[..., None]
        _within(v.flatten(-2), y64, (R.U[F8] * (1 + 4 * rel) + 4 * rel) * y64.abs()
                + 1.001 * R.TINY[F8] * s64.repeat_interleave(128, -1), "y8")


@pytest.mark.parametrize("act", [BF, FP])
@pytest.mark.parametrize("H", [8, 128, 136, 512, 640, 1024, 1032, 2048, 2056, 4096, 4224, 8192, 8200, 32768])
def test_norm_widths(H, act):
    g = _gen(H)
    for T in (1, 3, 6):
        x, r, w = (torch.randn(n, H, generator=g).to(act) for n in (T, T, 1))
        w = w[0]
        y8 = H % 128 == 0
        out = _ops().rms_norm(x.cuda(), w.cuda(), r.cuda(), eps=1e-5, y16=True, y8=y8)
        _check_norm(out, x, r, w, 1e-5)
        out = _ops().rms_norm(x.cuda(), eps=0.0, y16=not y8, y8=y8)
        assert out[0] is None
        _check_norm(out, x, None, None, 0.0)


def test_norm_many_rows_strides_and_own_buffers():
    g = _gen(1)
    wide = torch.randn(1037, 1024 + 24, generator=g).to(BF)
    r, w = torch.randn(1037, 1024, generator=g).to(BF), torch.randn(1024, generator=g).to(BF)
    dev = wide.cuda()
    x = dev[:, 8:1032]
    _check_norm(_ops().rms_norm(x, w.cuda(), r.cuda(), y8=True), wide[:, 8:1032], r, w, 1e-5)
    # the sum over the residual's own buffer, the norm over x's
    xb, rb = wide[:, :1024].contiguous().cuda(), r.cuda()
    out = _ops().rms_norm(xb, w.cuda(), rb, out=(rb, xb, None, None))
    assert out[0].data_ptr() == rb.data_ptr() and out[1].data_ptr() == xb.data_ptr()
    _check_norm(out, wide[:, :1024], r, w, 1e-5)


def test_norm_extreme_rows():
    """Zero rows, rows of the smallest and largest values, rows with an infinity
    or a NaN: the others are not touched, and 8-bit codes stay defined."""
    H = 256
    x = torch.randn(8, H, generator=_gen(2)).to(BF)
    x[1] = 0
    x[2] = 1e-38                       # squares vanish: eps alone counts
    x[3, 5] = math.inf
    x[4, 7] = math.nan
    x[5] *= 1e18                       # squares near 1e36
    out = _ops().rms_norm(x.cuda(), y8=True, eps=1e-6)
    keep = [0, 1, 2, 5, 6, 7]
    _check_norm([None if t is None else t[keep] for t in out], x[keep], None, None, 1e-6)
    assert torch.isnan(out[1][4]).all()
    y = out[1][3].cpu().float()
    assert torch.isnan(y[5]) and (y[:5] == 0).all()
    assert (out[2][1].float() == 0).all() and (out[3][1] == 2.0 ** -126).all()


def test_norm_empty_batch_writes_nothing():
    out = _ops().rms_norm(torch.empty(0, 256, dtype=BF, device="cuda"), y8=True)
    assert out[1].shape == (0, 256) and out[3].shape == (0, 2)


# ---------------------------------------------------------------------------
# 8-bit product
# ---------------------------------------------------------------------------

def _gemm_case(M, N, K, seed, wide=False):
    g = _gen(seed)
    a, a_s = R.quant(torch.randn(M, K, generator=g), 128)
    w = (torch.randn(N, K, generator=g) * 100).to(F8)
    w_s = torch.rand(-(-N // 128), K // 128, generator=g) + 0.1
    if wide:                           # scales over many orders of magnitude
        a_s = a_s * 2.0 ** torch.randint(-40, 40, a_s.shape, generator=g)
        w_s = w_s * 2.0 ** torch.randint(-40, 40, w_s.shape, generator=g)
    return a, a_s.contiguous(), w, w_s.contiguous()


def _check_gemm(y, a, a_s, w, w_s):
    N, K = w.shape
    if y.shape[0] * N * K > 1 << 32:   # (the definition's products on the device)
        y, a, a_s, w, w_s = (t.cuda() for t in (y, a, a_s, w, w_s))
    af = a.double() * a_s.double().repeat_interleave(128, 1)
    wf = w.double() * w_s.double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)
    want, mass = af @ wf.T, af.abs() @ wf.abs().T
    # 128 products in one instruction, one multiply-add for each block, and the
    # joins of K's parts
    sums = (128 + K // 128 + 24) * 2.0 ** -23 * mass
    _within(y, want.cpu(), (R.U[y.dtype] * (want.abs() + sums) + sums + R.TINY[y.dtype]).cpu(), "product")


@pytest.mark.parametrize("M,N,K", [(1, 1, 128), (1, 16, 128), (2, 129, 256), (15, 500, 384), (16, 4000, 512), (17, 127, 4096),
                                   (31, 1000, 640), (33, 260, 1152), (48, 96, 2048), (64, 384, 1024), (65, 4000, 256),
                                   (100, 640, 896), (128, 256, 1024), (129, 513, 384), (200, 1030, 640), (257, 300, 2048),
                                   (300, 768, 128), (513, 2052, 1280), (777, 1100, 384)])
@pytest.mark.parametrize("out", [BF, FP, F32])
def test_gemm_sizes(M, N, K, out):
    a, a_s, w, w_s = _gemm_case(M, N, K, M * 7 + N)
    if out == FP:
        w_s = w_s * 2.0 ** -12         # stay inside fp16
    lin = _ops().Linear8(w.cuda(), w_s.cuda())
    y = lin.forward(a.cuda(), a_s.cuda(), dtype=out)
    _check_gemm(y, a, a_s, w, w_s)
    assert _same(y, lin.forward(a.cuda(), a_s.cuda(), dtype=out)), "two runs differ"


@pytest.mark.parametrize("M,N,K", [
    (3600, 3400, 1280), (2600, 5300, 2304), (4001, 3333, 8448),    # wide tiles; more than 64 blocks of K
    (2100, 2200, 1408), (1700, 2700, 4224), (900, 4800, 8320),     # pairs of small tiles
    (513, 2052, 1280), (777, 4000, 2048), (130, 700, 8448),        # small tiles, whole and in parts of K
    (1250, 4300, 10752), (1000, 4000, 14336),                      # wide tiles in parts of a long K
    (64, 6144, 4096), (40, 900, 16512), (250, 1000, 2048)])
def test_gemm_kernels(M, N, K):
    """Every kernel at sizes that it is chosen for, with odd ends."""
    a, a_s, w, w_s = _gemm_case(M, N, K, N)
    lin = _ops().Linear8(w.cuda(), w_s.cuda())
    y = lin.forward(a.cuda(), a_s.cuda(), dtype=F32)
    _check_gemm(y, a, a_s, w, w_s)
    y16 = torch.full((M, N + 5), 3.0, dtype=BF, device="cuda")
    lin.forward(a.cuda(), a_s.cuda(), out=y16[:, 1:N + 1])
    _check_gemm(y16[:, 1:N + 1], a, a_s, w, w_s)
    assert (y16[:, 0] == 3.0).all() and (y16[:, N + 1:] == 3.0).all()


@pytest.mark.parametrize("N,K", [(1, 128), (16, 256), (37, 384), (300, 1024)])
def test_packed_layout(N, K):
    """Tiles as the header lays them out; rows past N are zeros."""
    w = torch.randint(0, 256, (N, K), generator=_gen(N), dtype=torch.uint8)
    lin = _ops().Linear8(w.view(F8).cuda(), torch.ones(-(-N // 128), K // 128, device="cuda"))
    rows = np.zeros((-(-N // 16) * 16, K), np.uint8)
    rows[:N] = w.numpy()
    want = np.zeros(rows.size, np.uint8)
    n, k = np.meshgrid(np.arange(rows.shape[0]), np.arange(K), indexing="ij")
    want[(n // 16 * (K // 128) + k // 128) * 2048 + k % 128 // 64 * 1024 + 16 * (16 * (k // 16 % 4) + n % 16) + k % 16] = rows
    assert np.array_equal(lin.packed.cpu().numpy(), want)


@pytest.mark.parametrize("M,N,K", [(5, 200, 1024), (40, 130, 2048), (300, 700, 512)])
def test_gemm_wide_scales(M, N, K):
    a, a_s, w, w_s = _gemm_case(M, N, K, 3, wide=True)
    _check_gemm(_ops().Linear8(w.cuda(), w_s.cuda()).forward(a.cuda(), a_s.cuda(), dtype=F32), a, a_s, w, w_s)


@pytest.mark.parametrize("M,N,K", [(1, 30, 256), (19, 333, 512), (260, 515, 384)])
def test_gemm_strides_and_untouched_memory(M, N, K):
    a, a_s, w, w_s = _gemm_case(M, N, K, 4)
    a_wide, w_wide = (torch.full((n, K + 48), math.nan).to(F8).cuda() for n in (M, N))
    a_wide[:, 16:16 + K], w_wide[:, 32:32 + K] = a.cuda(), w.cuda()
    y = torch.full((M + 2, N + 7), 7.0, dtype=BF, device="cuda")
    _ops().Linear8(w_wide[:, 32:32 + K], w_s.cuda()).forward(a_wide[:, 16:16 + K], a_s.cuda(), out=y[1:M + 1, 3:3 + N])
    _check_gemm(y[1:M + 1, 3:3 + N], a, a_s, w, w_s)
    y[1:M + 1, 3:3 + N] = 7.0
    assert (y == 7.0).all()


@pytest.mark.parametrize("M,N,K", [(20, 144, 256), (300, 400, 256)])
def test_gemm_nan_and_infinite_scales_stay_in_their_rows(M, N, K):
    a, a_s, w, w_s = _gemm_case(M, N, K, 5)
    a[M - 3, 130] = math.nan
    w[N - 2, 7] = math.nan
    a_s[2, 1] = math.inf
    y = _ops().Linear8(w.cuda(), w_s.cuda()).forward(a.cuda(), a_s.cuda()).cpu().float()
    assert torch.isnan(y[M - 3]).all() and torch.isnan(y[:, N - 2]).all()
    assert not torch.isfinite(y[2]).any()
    rows, cols = [m for m in range(M) if m not in (2, M - 3)], [n for n in range(N) if n != N - 2]
    a[M - 3], w[N - 2], a_s[2] = 0, 0, 1.0
    clean = _ops().Linear8(w.cuda(), w_s.cuda()).forward(a.cuda(), a_s.cuda()).cpu().float()
    assert torch.equal(y[rows][:, cols], clean[rows][:, cols])


def test_gemm_long_rows():
    """K past what one pass of a small kernel holds, rows past 2^31 bytes apart."""
    a, a_s, w, w_s = _gemm_case(3, 40, 16384, 6)
    _check_gemm(_ops().Linear8(w.cuda(), w_s.cuda()).forward(a.cuda(), a_s.cuda(), dtype=F32), a, a_s, w, w_s)
    rows = torch.zeros(600, 1 << 22, dtype=torch.uint8, device="cuda").view(F8)
    a, a_s, w, w_s = _gemm_case(600, 600, 256, 7)
    rows[:, :256] = w.cuda()
    rows[:, 512:768] = a.cuda()
    _check_gemm(_ops().Linear8(rows[:, :256], w_s.cuda()).forward(rows[:, 512:768], a_s.cuda()), a, a_s, w, w_s)
    _check_gemm(_ops().Linear8(rows[:, :256], w_s.cuda()).forward(rows[:9, 512:768], a_s[:9].cuda()), a[:9], a_s[:9], w, w_s)


# ---------------------------------------------------------------------------
# Cache
# ---------------------------------------------------------------------------

def _cache(n, P, H, D, act, bits, stride=None, fill=0xFF):
    """A cache whose bytes are all 0xFF: NaN as 16-bit, 8-bit and fp32 values."""
    nb = R.block_bytes(H, P, D, bits)
    pool = torch.full(((n - 1) * (stride or nb) + nb + (nb if stride else 0),), fill, dtype=torch.uint8, device="cuda")
    return _ops().KVCache(n, P, H, D, act, fp8=bits == 8, pool=pool, block_stride=stride)


@pytest.mark.parametrize("D", [64, 128, 192, 256])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("act", [BF, FP])
@pytest.mark.parametrize("P,H,T", [(32, 1, 1), (32, 3, 70), (64, 2, 45), (128, 1, 300), (256, 2, 33)])
def test_append_writes_its_slots_alone(D, bits, act, P, H, T):
    """Random slots, padding, slots past the last block; every other byte stays."""
    n = T * 2 // P + 3
    g = _gen(D + T)
    kv = (torch.randn(T, 2, H, D, generator=g) * 3).to(act)
    kv[0] = 0
    slots = torch.randperm(n * P, generator=g)[:T]
    slots[3::7] = -1
    slots[5::11] = n * P + 5
    if T > 8:
        slots[8] = -(1 << 40)
    c = _cache(n, P, H, D, act, bits)
    assert c.block_bytes == R.block_bytes(H, P, D, bits)
    dev = kv.cuda()
    c.append(dev[:, 0], dev[:, 1], slots.cuda())
    want = np.full(c.pool.numel(), 0xFF, np.uint8)
    R.write_slots(want, c.block_bytes, kv[:, 0], kv[:, 1], slots, P, bits, n)
    assert np.array_equal(c.pool.cpu().numpy(), want)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("P,first,T", [(32, 0, 64), (32, 17, 200), (64, 1, 63), (64, 40, 41), (128, 96, 333)])
def test_append_consecutive_positions(bits, P, first, T):
    """A chunk of one sequence that starts and ends anywhere in a block, and one
    with its rows in reverse order."""
    H, D = 2, 128
    n = (first + T) // P + 2
    g = _gen(T)
    kv = torch.randn(T, 2, H, D, generator=g).to(BF)
    blocks = torch.randperm(n, generator=g)
    pos = torch.arange(first, first + T)
    slots = blocks[pos // P] * P + pos % P
    for s in (slots, slots.flip(0)):
        c = _cache(n, P, H, D, BF, bits)
        rows = torch.zeros(T, 5, H, D, dtype=BF, device="cuda")
        rows[:, 1], rows[:, 3] = kv[:, 0].cuda(), kv[:, 1].cuda()
        c.append(rows[:, 1], rows[:, 3], s.cuda())
        want = np.full(c.pool.numel(), 0xFF, np.uint8)
        R.write_slots(want, c.block_bytes, kv[:, 0], kv[:, 1], s, P, bits, n)
        assert np.array_equal(c.pool.cpu().numpy(), want)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("D", [64, 128, 192, 256])
def test_append_many_tokens_in_runs(bits, D):
    """More than 512 tokens: whole tiles, runs of every length that start and end
    anywhere in a tile, padding and lone tokens between them, a slot past the end."""
    H, P, n = 2, 64, 60
    g = _gen(D)
    slots, at = [], 0
    for length in [40, 1, 7, 8, 9, 31, 32, 33, 64, 3, 2, 100, 5, 16, 17, 65, 150]:
        at += int(torch.randint(1, 50, (1,), generator=g))
        slots += list(range(at, at + length)) + ([-1] if length % 2 else [])
        at += length
    slots += list(range(n * P - 70, n * P + 30))                  # runs past the last block
    slots += (torch.arange(40) * 3 + at).flip(0).tolist()         # lone tokens, backwards
    slots = torch.tensor(slots)
    T = slots.numel()
    assert T > 512 and at + 120 < n * P - 70
    kv = torch.randn(T, 2, H, D, generator=g).to(FP)
    c = _cache(n, P, H, D, FP, bits)
    dev = kv.cuda()
    c.append(dev[:, 0], dev[:, 1], slots.cuda())
    want = np.full(c.pool.numel(), 0xFF, np.uint8)
    R.write_slots(want, c.block_bytes, kv[:, 0], kv[:, 1], slots, P, bits, n)
    assert np.array_equal(c.pool.cpu().numpy(), want)


@pytest.mark.parametrize("bits", [16, 8])
def test_append_extreme_values(bits):
    kv = torch.randn(6, 2, 1, 64, generator=_gen(9)).to(BF)
    kv[1, 0, 0, 3] = math.nan
    kv[2, 1, 0, 9] = math.inf
    kv[3] *= 1e-38
    kv[4] *= 1e38
    c = _cache(1, 32, 1, 64, BF, bits)
    slots = torch.arange(6) * 5
    dev = kv.cuda()
    c.append(dev[:, 0], dev[:, 1], slots.cuda())
    if bits == 16:
        want = np.full(c.pool.numel(), 0xFF, np.uint8)
        R.write_slots(want, c.block_bytes, kv[:, 0], kv[:, 1], slots, 32, bits, 1)
        assert np.array_equal(c.pool.cpu().numpy(), want)
        return
    pool = c.pool.cpu()
    sc = pool[2 * 32 * 64:].view(torch.float32).view(2, 32)
    code = lambda i, t, d: pool[i * 32 * 64 + int((R.key_byte, R.value_byte)[i](t, d, 64, 8))].view(F8).float().item()
    assert math.isnan(code(0, 5, 3)) and not math.isnan(code(0, 5, 4))      # NaN stays in its place
    m = kv[1, 0, 0].float()
    assert sc[0, 5] == m[~torch.isnan(m)].abs().max() / torch.tensor(448.0)
    assert math.isinf(sc[1, 10]) and math.isnan(code(1, 10, 9)) and code(1, 10, 10) == 0
    for n in (3, 4):
        q, s = R.quant(kv[n, 0], 64)
        assert sc[0, 5 * n] == s[0, 0]
        assert [code(0, 5 * n, d) for d in range(64)] == q[0].float().tolist()


# ---------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------

def _attend_case(lens, P, H, g, D, act, bits, window=0, stride=None, seed=0, missing=None, scale=None, table_pad=0, big=1.0,
                 max_len=None, stream=None):
    """Fill a cache (NaN elsewhere) through append, attend, check every row."""
    B, L = len(lens), max(max(lens), 1) if max_len is None else max_len
    nb = -(-L // P)
    gen = _gen(seed)
    n = B * nb + 1
    perm = torch.randperm(n - 1, generator=gen) + 1       # block 0 holds NaN
    table = torch.full((B, nb + table_pad), -7, dtype=torch.int32)
    table[:, :nb] = perm.view(B, nb).int()
    unit = 1
    if stride == 256:                                     # block numbers count 256 bytes
        unit = R.block_bytes(H, P, D, bits) // 256
        table[:, :nb] *= unit
    c = _cache((n - 1) * unit + 1, P, H, D, act, bits, stride)
    kv = (torch.randn(sum(lens), 2, H, D, generator=gen) * big).to(act)
    q = (torch.randn(B, H * g + 3, D, generator=gen)).to(act)
    slots = torch.cat([table[b, torch.arange(m) // P].long() * P + torch.arange(m) % P for b, m in enumerate(lens)] or [torch.zeros(0)])
    dev = kv.cuda()
    c.append(dev[:, 0], dev[:, 1], slots.long().cuda())
    gone = [set() for _ in lens]
    if missing:
        for b, j, bad in missing:
            table[b, j] = bad
            gone[b] = gone[b] | set(range(j * P, (j + 1) * P))
    lse = torch.empty(B, H * g, device="cuda")
    tab, lens_d, q_d = table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), q.cuda()
    torch.cuda.synchronize()
    out = c.attend(q_d[:, 1:1 + H * g], tab, lens_d, L, scale=scale, window=window, lse=lse, stream=stream)
    torch.cuda.synchronize()
    sc = D ** -0.5 if scale is None else scale
    at = 0
    for b, m in enumerate(lens):
        k64, v64 = R.cached(kv[at:at + m, 0], bits), R.cached(kv[at:at + m, 1], bits)
        at += m
        o, e, mass, size = R.attend(q[b, 1:1 + H * g], k64, v64, m, sc, window, gone[b])
        # scores: D products summed in fp32 and two scalings; weights: twice the
        # score's error, an exponential, a sum of m terms; values: the second
        # 16-bit term leaves 2^-16 of a weight
        ds = (D + 8) * 2.0 ** -23 * size
        rel = 2 * ds + (m + 64) * 2.0 ** -23 + 2.0 ** -15
        _within(out[b], o, R.U[act] * (1 + 2 ** -8) * o.abs() + rel[:, None] * mass + 2 * R.TINY[act], "row %d" % b)
        _within(lse[b], e, ds + (m + 64) * 2.0 ** -23 + 2.0 ** -21 * e.abs().nan_to_num(0, 0, 0), "lse %d" % b)
    return c, out


@pytest.mark.parametrize("D", [64, 128, 192, 256])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("act", [BF, FP])
def test_attend_lengths(D, bits, act):
    _attend_case([0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300, 0], 64, 2, 3, D, act, bits, seed=D)


@pytest.mark.parametrize("P", [32, 64, 128, 256])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("g", [1, 4, 7, 16, 17, 40])
def test_attend_heads_and_blocks(P, bits, g):
    _attend_case([P - 1, 3 * P + 5, 1], P, 2, g, 64, BF, bits, seed=P + g)


@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 64, 100, 1000])
@pytest.mark.parametrize("bits", [16, 8])
def test_attend_window(window, bits):
    _attend_case([0, 1, 31, 33, 64, 99, 200, 777], 32, 1, 2, 128, FP, bits, window=window, seed=window)


@pytest.mark.parametrize("lens", [[5000], [9001, 3], [1, 4097, 0, 2050, 33]])
@pytest.mark.parametrize("bits,act,D", [(16, BF, 128), (8, FP, 64), (8, BF, 256), (16, FP, 192)])
def test_attend_split_sequences(lens, bits, act, D):
    """Long sequences beside short ones: splits and their join."""
    _attend_case(lens, 64, 2, 4, D, act, bits, seed=len(lens))
    _attend_case(lens, 64, 2, 4, D, act, bits, window=1500, seed=len(lens))


@pytest.mark.parametrize("bits", [16, 8])
def test_attend_missing_blocks(bits):
    """Blocks outside the pool are left out, also the first and all of a row."""
    _attend_case([200, 150, 64, 3000], 32, 1, 4, 128, BF, bits,
                 missing=[(0, 1, -1), (0, 6, 10 ** 6), (1, 0, -5), (2, 0, -1), (2, 1, 2 ** 31 - 1), (3, 40, -1), (3, 41, -1)])


@pytest.mark.parametrize("bits", [16, 8])
def test_attend_large_and_small_scores(bits):
    """Scores of hundreds (one key takes all), of nothing, and negative scales."""
    for scale in (30.0, 0.0, -2.0, 1e-6):
        _attend_case([77, 700], 32, 2, 2, 64, BF, bits, scale=scale, seed=5)
    _attend_case([77, 700], 32, 2, 2, 64, BF, bits, scale=1e-4, big=300.0, seed=6)


def test_attend_rising_scores():
    """Scores that rise from tile to tile: the running maximum moves every time."""
    D, n = 64, 600
    c = _cache(40, 32, 1, D, BF, 16)
    k = torch.zeros(n, 1, D)
    k[:, 0, 0] = torch.arange(n) / 4.0
    v = torch.randn(n, 1, D, generator=_gen(3))
    k, v = k.to(BF), v.to(BF)
    slots = torch.arange(n)
    c.append(k.cuda(), v.cuda(), slots.cuda())
    q = torch.zeros(1, 2, D, dtype=BF)
    q[0, 0, 0], q[0, 1, 0] = 4.0, -4.0
    out = c.attend(q.cuda(), torch.arange(40, dtype=torch.int32, device="cuda")[None], torch.tensor([n], dtype=torch.int32, device="cuda"), n, scale=1.0)
    # one product to a score, of at most 600: two roundings of it, 600 * 2^-23 in
    # an exponent
    o, _, mass, _ = R.attend(q[0], k.double(), v.double(), n, 1.0, 0)
    _within(out[0], o, R.U[BF] * 1.01 * o.abs() + 2e-3 * mass, "rising")


def test_attend_padded_tables_bounds_and_units():
    """Longer table rows, a bound beyond and below the lengths, block numbers in
    units of 256 bytes, a stride past 32 bits."""
    _attend_case([100, 5], 32, 2, 2, 64, BF, 16, table_pad=3, max_len=400)
    _attend_case([100, 5], 32, 2, 2, 64, BF, 8, stride=256)
    _attend_case([100, 5, 70], 32, 1, 2, 64, BF, 16, stride=(1 << 30) + 256)
    _attend_case([100, 5, 70], 32, 1, 2, 64, BF, 8, stride=(1 << 30) + 256)
    # a sequence longer than the bound counts as the bound
    c, _ = _attend_case([96, 200], 32, 1, 2, 64, BF, 16)
    q = torch.randn(2, 2, 64, generator=_gen(8)).to(BF).cuda()
    table = torch.tensor([[1, 2, 3], [4, 5, 6]], dtype=torch.int32, device="cuda")
    lens = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([96, 96], [10 ** 6, 97], [-4, 0])]
    a, b, z = (c.attend(q, table, n, 96) for n in lens)
    assert _same(a, b) and (z == 0).all()


@pytest.mark.parametrize("bits", [16, 8])
def test_attend_many_sequences(bits):
    _attend_case([(37 * i) % 90 for i in range(300)], 32, 1, 2, 64, BF, bits, seed=11)


@pytest.mark.parametrize("D,bits,act", [(64, 16, BF), (64, 8, FP), (128, 16, FP), (128, 8, BF), (192, 8, BF), (256, 16, BF), (256, 8, FP)])
@pytest.mark.parametrize("g", [1, 5, 20])
def test_attend_equal_shares(D, bits, act, g):
    """A large bound on the lengths: all tiles cut into equal shares, with
    workgroups that hold several short sequences and sequences over several."""
    lens = [0, 1, 33, 700, 64, 0, 0, 2, 1500, 31, 32, 5, 97, 0]
    H = 2 if g < 20 else 1
    _attend_case(lens, 64, H, g, D, act, bits, seed=g, max_len=40000)


@pytest.mark.parametrize("window", [0, 900])
def test_attend_equal_shares_of_many_sequences(window):
    """More sequences than lanes, most of them empty or short."""
    lens = [(37 * i) % 97 * (i % 3) for i in range(150)]
    lens[70], lens[149] = 4000, 2000
    _attend_case(lens, 32, 2, 2, 64, BF, 16, window=window, seed=7, max_len=5000)
    _attend_case([0] * 150, 32, 2, 2, 64, BF, 16, window=window, seed=7, max_len=5000)


@pytest.mark.parametrize("B", [256, 257])
@pytest.mark.parametrize("D,bits,act", [(64, 16, FP), (128, 8, BF), (128, 16, BF), (192, 8, FP), (256, 8, BF), (256, 16, FP)])
def test_attend_around_one_workgroup_per_cu(B, D, bits, act):
    """Lengths around the tiles of four and of eight waves, and of none."""
    _attend_case([(53 * i + 31 * (i % 4)) % 300 for i in range(B)], 32, 1, 3, D, act, bits, seed=B)


@pytest.mark.parametrize("tiles", [19, 20, 21, 39, 40, 41, 79, 80, 81])
@pytest.mark.parametrize("D,bits", [(64, 16), (128, 8), (128, 16), (256, 16)])
def test_attend_around_the_first_split(tiles, D, bits):
    _attend_case([32 * tiles, 32 * tiles - 31, 5], 64, 1, 2, D, BF, bits, seed=tiles, max_len=32 * tiles)


def test_attend_runs_twice_the_same_and_on_other_streams():
    side = torch.cuda.Stream()
    _, a = _attend_case([3000, 50], 64, 2, 4, 128, BF, 8, seed=4)
    _, b = _attend_case([3000, 50], 64, 2, 4, 128, BF, 8, seed=4, stream=side)
    assert _same(a, b)


# ---------------------------------------------------------------------------
# Routing
# ---------------------------------------------------------------------------

def _check_route(logits, K, n_shared=0, gate=None, dtype=F32, **kw):
    T, E = logits.shape
    dev = logits.to(dtype)
    ids, w, off, ss, sp = _ops().route_grouped(dev.cuda(), K, n_shared=n_shared, gate=None if gate is None else gate.cuda(),
                                               **{k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in kw.items()})
    if "bias" in kw and kw["bias"] is not None:
        kw["bias"] = kw["bias"].numpy()
    want, ww = R.route(dev.float().numpy(), K, **kw)
    ids, w = ids.cpu().numpy(), w.cpu().numpy()
    assert np.array_equal(ids[:, :K], want)
    assert np.all(np.abs(w[:, :K] - ww) <= 2.0 ** -23 * np.abs(ww))      # 64 bits, rounded once
    if n_shared:
        assert np.array_equal(ids[:, K:], np.broadcast_to(np.arange(E, E + n_shared), (T, n_shared)))
        assert np.array_equal(w[:, K:], np.ones((T, n_shared), np.float32) if gate is None else gate.numpy())
    o, order, pos = R.permute(ids, E + n_shared)
    assert np.array_equal(off.cpu().numpy(), o)
    assert np.array_equal(ss.cpu().numpy()[:order.size], order) and np.array_equal(sp.cpu().numpy()[:pos.size], pos)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("T,E,K,groups,top,gt", [(1, 1, 1, 1, 1, 1), (5, 8, 2, 1, 1, 1), (33, 60, 4, 1, 1, 1), (17, 64, 6, 8, 3, 2),
                                                 (130, 160, 6, 8, 3, 1), (50, 256, 8, 8, 4, 2), (9, 256, 16, 64, 4, 2),
                                                 (21, 63, 3, 7, 2, 2), (8, 64, 16, 64, 16, 2), (300, 72, 5, 3, 2, 2)])
def test_route_shapes(score, T, E, K, groups, top, gt):
    g = _gen(E + T)
    logits, bias = torch.randn(T, E, generator=g) * 2, torch.randn(E, generator=g) * 0.1
    _check_route(logits, K, score=score, groups=groups, top_groups=top, group_top=gt, bias=bias)
    _check_route(logits, K, score=score, groups=groups, top_groups=top, group_top=gt, renorm=False, scale=2.5)
    for dt in (BF, FP):
        _check_route(logits, K, dtype=dt, score=score, groups=groups, top_groups=top, group_top=gt, bias=bias, scale=-1.5)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("n_shared", [1, 3])
def test_route_shared_columns(score, n_shared):
    g = _gen(7)
    logits = torch.randn(70, 32, generator=g)
    _check_route(logits, 4, n_shared, torch.rand(70, n_shared, generator=g), score=score, groups=4, top_groups=2, group_top=2)
    _check_route(logits, 4, n_shared, None, score=score)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups,top,gt", [(1, 1, 1), (4, 2, 2), (4, 2, 1), (4, 4, 2)])
def test_route_masks_ties_and_extremes(score, groups, top, gt):
    """Masked experts, rows and groups, equal logits, the type's ends."""
    E = 32
    x = torch.randn(14, E, generator=_gen(5))
    x[0] = -math.inf                              # nothing is eligible
    x[1] = math.nan
    x[2, 3:] = -math.inf                          # fewer than K are
    x[3, ::2] = -math.inf
    x[4] = 1.0                                    # all tie
    x[5, 8:16] = -math.inf                        # a whole group
    x[6] = torch.finfo(F32).min
    x[7, 4] = math.inf
    x[8, 4], x[8, 9] = 3.4e38, 3.4e38
    x[9] = 0.0
    x[9, 1::2] = -0.0
    x[10, 5] = math.nan
    x[11, :31] = torch.finfo(F32).min
    x[12] = x[12].round()                         # many ties
    x[13, 24:] = -math.inf
    x[13, 24] = 50.0                              # one eligible expert in a group
    bias = torch.zeros(E)
    bias[7], bias[20] = -math.inf, 0.25
    for b in (None, bias):
        _check_route(x, 6, score=score, groups=groups, top_groups=top, group_top=gt, bias=b)
    bias = bias.clone()
    bias[3] = math.nan
    _check_route(x, 6, score=score, groups=groups, top_groups=top, group_top=gt, bias=bias, renorm=False)


def test_route_near_ties_follow_64_bits():
    """Scores that 32 bits cannot tell apart are still told apart."""
    x = 5.0 + torch.arange(64).float() * 2.0 ** -21
    x = x[torch.randperm(64, generator=_gen(1))][None].repeat(3, 1)
    _check_route(x, 8, score="sigmoid", bias=torch.full((64,), 0.3))
    _check_route(-x, 8, score="sigmoid", groups=8, top_groups=4, group_top=2)


@pytest.mark.parametrize("T,E,K,n_shared", [(2048, 64, 8, 0), (2731, 250, 5, 1), (4099, 256, 8, 0), (40000, 16, 7, 0)])
def test_route_many_slots(T, E, K, n_shared):
    """Permutations of many slots, in parts of 512 and more; the choice is checked
    by the other tests (few experts tie here)."""
    logits = torch.randn(T, E, generator=_gen(T)).cuda()
    ids, w, off, ss, sp = _ops().route_grouped(logits, K, n_shared=n_shared)
    top = torch.sort(logits.double(), dim=1, descending=True, stable=True).indices[:, :K]
    assert torch.equal(ids[:, :K].long(), top)
    o, order, pos = R.permute(ids.cpu().numpy(), E + n_shared)
    assert np.array_equal(off.cpu().numpy(), o)
    assert np.array_equal(ss.cpu().numpy(), order) and np.array_equal(sp.cpu().numpy(), pos)


def test_route_no_tokens():
    ids, w, off, _, _ = _ops().route_grouped(torch.empty(0, 16, device="cuda"), 4)
    assert ids.shape == (0, 4) and (off.cpu() == 0).all()


def test_route_matches_the_plain_router():
    """One group, softmax, no bias: ids and order of pw_route_topk."""
    from paper_2607_16184_amd.layer import PagedLayer
    logits = torch.randn(500, 64, generator=_gen(2)).cuda()
    a = _ops().route_grouped(logits, 6)
    b = PagedLayer.routing_buffers(500, 64, 6)
    pw.pw_route_topk(logits.data_ptr(), 500, 64, 6, 1, *(t.data_ptr() for t in b), torch.cuda.current_stream().cuda_stream)
    for i in (0, 2, 3, 4):
        assert torch.equal(a[i], b[i])
    assert (a[1] - b[1]).abs().max() <= 1e-6


# ---------------------------------------------------------------------------
# Together
# ---------------------------------------------------------------------------

def test_captured_calls_replay():
    """All calls of a decode step recorded into one graph, replayed with new
    inputs and eager work in between: every replay equals the eager calls."""
    ops = _ops()
    T, H, heads, D, P = 5, 512, 8, 64, 32
    g = _gen(12)
    w8, ws = (torch.randn((heads + 4) * D, H, generator=g) * 50).to(F8).cuda(), torch.full((6, 4), 1e-3, device="cuda")
    lin = ops.Linear8(w8, ws)
    x, r = torch.zeros(T, H, dtype=BF, device="cuda"), torch.zeros(T, H, dtype=BF, device="cuda")
    router = torch.randn(H, 32, generator=g).to(BF).cuda()
    cache = ops.KVCache(T * 40, P, 2, D, BF)
    cache.pool.zero_()
    table = torch.randperm(T * 40, generator=g).int().view(T, 40).cuda()
    lens, slots = torch.zeros(T, dtype=torch.int32, device="cuda"), torch.zeros(T, dtype=torch.int64, device="cuda")

    def step():
        z, _, q8, qs = ops.rms_norm(x, None, r, y16=False, y8=True)
        qkv = lin.forward(q8, qs).view(T, heads + 4, D)
        cache.append(qkv[:, heads:heads + 2], qkv[:, heads + 2:], slots)
        o = cache.attend(qkv[:, :heads], table, lens, 1200)
        y = ops.rms_norm(o.view(T, H), None, z)
        return [o, *y[:2], *ops.route_grouped((y[1] @ router).float(), 4, score="sigmoid", groups=4, top_groups=2, group_top=2)]

    def inputs(i):
        gi = _gen(100 + i)
        n = torch.randint(1, 1200, (T,), generator=gi)
        x.copy_(torch.randn(T, H, generator=gi))
        r.copy_(torch.randn(T, H, generator=gi))
        lens.copy_(n)
        slots.copy_(table.cpu()[torch.arange(T), (n - 1) // P].long() * P + (n - 1) % P)

    inputs(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(4):
        inputs(i)
        graph.replay()
        torch.cuda.synchronize()
        first = [t.clone() for t in got]
        want = step()
        torch.cuda.synchronize()
        for a, b in zip(first, want):
            assert torch.equal(a, b)


def test_outgrown_workspace_stays_with_its_graph():
    """A larger call after a capture: the graph's own buffer stays untouched by
    others, and its replays give the first result."""
    ops = _ops()
    a, a_s, w, w_s = _gemm_case(200, 4000, 4096, 31)
    lin = ops.Linear8(w.cuda(), w_s.cuda())
    x, xs = a[:65].cuda(), a_s[:65].cuda()
    want = lin.forward(x, xs).clone()
    assert 2 * pw.pw_gemm_fp8_workspace(200, 4000, 4096) > 3 * pw.pw_gemm_fp8_workspace(65, 4000, 4096) > 0
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = lin.forward(x, xs)
    held = {t.data_ptr() for t in lin._ws.kept}
    a_d, as_d = a.cuda(), a_s.cuda()
    side.wait_stream(torch.cuda.current_stream())
    big, other = lin.forward(a_d, as_d, stream=side), lin.forward(x, xs, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    fill = [torch.full((1 << 20,), 255, dtype=torch.uint8, device="cuda") for _ in range(64)]
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert _same(got, want) and _same(other, want)
    assert held <= {t.data_ptr() for t in lin._ws.kept} and len({p for p, _ in lin._ws.of.values()}) == len(lin._ws.of) >= 2
    assert sum(t.numel() for t in lin._ws.kept) <= 2 * sum(n for _, n in lin._ws.of.values())
    assert all(bool((t == 255).all()) for t in fill)
    _check_gemm(big, a, a_s, w, w_s)


def test_cache_refuses_a_pool_smaller_than_its_blocks():
    ops = _ops()
    nb = R.block_bytes(2, 32, 64, 16)
    pool = torch.zeros(4 * nb, dtype=torch.uint8, device="cuda")
    ops.KVCache(4, 32, 2, 64, BF, pool=pool)
    ops.KVCache(2, 32, 2, 64, BF, pool=pool, block_stride=3 * nb)
    for n, stride in [(5, None), (3, 2 * nb), (2, 4 * nb)]:
        with pytest.raises(ValueError):
            ops.KVCache(n, 32, 2, 64, BF, pool=pool, block_stride=stride)


@pytest.mark.parametrize("M,N,K", [(1, 1000, 3456), (4, 5236, 384), (20, 300, 2048), (60, 6000, 1024), (200, 1000, 1024), (300, 4000, 2048),
                                   (130, 6144, 4096), (1000, 4100, 640)])
def test_gemm_fp32_sums_are_fp32(M, N, K):
    """fp32 outputs hold fp32 sums. Exact products, added 32 at a time to a
    running sum, and one multiply-add per block: a random walk of K / 32 + K /
    128 roundings of 2^-24 each; four times that is allowed, in norm."""
    g = _gen(M)
    a, a_s = R.quant(torch.randn(M, K, generator=g), 128)
    w = (torch.randn(N, K, generator=g) * 100).clamp(-448, 448).to(F8)
    w_s = torch.rand(-(-N // 128), K // 128, generator=g) + 0.1
    y = _ops().Linear8(w.cuda(), w_s.cuda()).forward(a.cuda(), a_s.cuda(), dtype=F32).cpu().double()
    af = a.double() * a_s.double().repeat_interleave(128, 1)
    want = af @ (w.double() * w_s.double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)).T
    off = float((y - want).norm() / want.norm())
    assert off <= (K / 32 + K / 128) ** 0.5 * 2.0 ** -22, off


def test_route_refuses_other_buffers():
    from paper_2607_16184_amd.layer import PagedLayer
    ops, logits = _ops(), torch.randn(6, 16, device="cuda")
    good = PagedLayer.routing_buffers(6, 16, 4)
    ops.route_grouped(logits, 4, out=good)
    for i in range(5):
        short = good[i][:2] if i < 2 else good[i][:-1]
        for bad in (good[i].cpu(), good[i].double(), short):
            with pytest.raises(ValueError):
                ops.route_grouped(logits, 4, out=tuple(bad if j == i else t for j, t in enumerate(good)))


@pytest.mark.parametrize("M", [33, 48, 49, 64])
@pytest.mark.parametrize("N,K", [(2048, 256), (2049, 384), (4096, 256), (4112, 256), (5120, 384), (8192, 256), (8193, 256)])
@pytest.mark.parametrize("out", [BF, F32])
def test_gemm_decode_batches(M, N, K, out):
    """One and two workgroups for the tokens, one and two row tiles."""
    a, a_s, w, w_s = _gemm_case(M, N, K, M + N)
    _check_gemm(_ops().Linear8(w.cuda(), w_s.cuda()).forward(a.cuda(), a_s.cuda(), dtype=out), a, a_s, w, w_s)
