"""A decoder layer's operators around its paged experts, on torch tensors.

PyTorch supplies device memory and streams only; every computation is a call
into libpagedweight.so (see include/pw.h for the formulas and constraints).
Outputs are written where ``out`` points, as a serving loop that keeps its
buffers wants it, or into new tensors. Shapes, types and strides are checked
here, sizes and alignment by the library (:class:`pw.PWError`).

Work goes to the current stream, or to ``stream``: what this module allocates
then belongs to that stream; the caller orders it after whatever wrote the
inputs, and keeps them until it is done. A handle may be used on several
streams; graphs that were captured on one stream share its workspace and are
replayed one after the other. That holds for all handles together that are given
one :class:`Workspace`, as the caches of a model's layers may be. A call's tensors
and its stream belong to one device, which need not be the current one.
"""
from __future__ import annotations

from typing import Optional, Tuple

import torch

from . import pw
from .layer import PagedLayer

_TYPE = {torch.float16: pw.PW_F16, torch.bfloat16: pw.PW_BF16, torch.float32: pw.PW_F32}
_F8 = torch.float8_e4m3fn


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _int32(x: int, name: str):
    """A foreign-function call would cut a larger one down to its last 32 bits."""
    if not -(1 << 31) <= x < 1 << 31:
        raise ValueError("%s must fit 32 bits: %d" % (name, x))


def _ptr(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.data_ptr()


def _on(dev: int, stream) -> int:
    """The given stream, or the current one of the device. (Its raw handle: 0.1
    us, a Stream object 3 us, as long as a launch.)"""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(dev)
    if stream.device_index != dev:
        raise ValueError("the stream belongs to device %d, the tensors to %d" % (stream.device_index, dev))
    return stream.cuda_stream


def _call(dev: int, fn, *args):
    """fn(*args) with `dev` as the current device: a default stream's handle (0)
    means the current device's."""
    if torch._C._cuda_getDevice() == dev:
        fn(*args)
    else:
        with torch.cuda.device(dev):
            fn(*args)


def _packed(t: Optional[torch.Tensor], shape, dtype, dev: int, name: str):
    if t is not None and not (t.dtype is dtype and t.shape == shape and t.get_device() == dev and t.is_contiguous()):
        raise ValueError("%s must be a contiguous tensor of %s, %s, on device %d" % (name, tuple(shape), dtype, dev))


def _empty(shape, dtype, device, stream) -> torch.Tensor:
    """A new tensor that belongs to the stream whose kernels write it."""
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


class Workspace:
    """The device buffers of one handle, or of several that are used one after the
    other on a stream: one buffer for each stream, grown to what the calls need. A
    call is made with the buffer at hand, and where that is too small (PW_ENOMEM,
    nothing launched) again with a larger one. Sizes are powers of two and an
    outgrown buffer is kept, since a captured graph may hold its address: together
    they are smaller than the last one."""

    def __init__(self, device="cuda"):
        self.device, self.of, self.kept = torch.empty(0, device=device).device, {}, []

    def run(self, dev: int, stream, fn, args, need):
        st = _on(dev, stream)
        at = self.of.get(st, (0, 0))
        try:
            _call(dev, fn, *args, *at, st)
        except pw.PWError as e:
            if e.status != pw.PW_ENOMEM:
                raise
            t = _empty(1 << (need() - 1).bit_length(), torch.uint8, self.device, stream)
            self.kept.append(t)
            at = self.of[st] = (t.data_ptr(), t.numel())
            _call(dev, fn, *args, *at, st)


# ---------------------------------------------------------------------------
# Norm
# ---------------------------------------------------------------------------

NormOut = Tuple[Optional[torch.Tensor], Optional[torch.Tensor], Optional[torch.Tensor], Optional[torch.Tensor]]


def norm_buffers(T: int, H: int, act: torch.dtype, residual: bool = True, y16: bool = True, y8: bool = False,
                 device="cuda") -> NormOut:
    """(sum, y16, y8, y8_scale) of ``rms_norm``, None for those not wanted."""
    return (torch.empty((T, H), dtype=act, device=device) if residual else None,
            torch.empty((T, H), dtype=act, device=device) if y16 else None,
            torch.empty((T, H), dtype=_F8, device=device) if y8 else None,
            torch.empty((T, H // 128), dtype=torch.float32, device=device) if y8 else None)


def rms_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None, *,
             eps: float = 1e-5, y16: bool = True, y8: bool = False, out: NormOut = None, stream=None) -> NormOut:
    """Root-mean-square norm of x (+ residual): (sum, y16, y8, y8_scale), the
    wanted ones of them or those that ``out`` holds (pw_rms_norm)."""
    T, H = x.shape
    act, dev = x.dtype, x.get_device()
    ldx, inner = x.stride()
    _need((act is torch.bfloat16 or act is torch.float16) and dev >= 0 and inner == 1, "x must be 16-bit rows on the device")
    ldr = H
    if residual is not None:
        ldr, inner = residual.stride()
        _need(residual.shape == x.shape and residual.dtype is act and residual.get_device() == dev and inner == 1,
              "residual must have x's shape, type and device")
    if T <= 1:                         # a single row may have any stride
        ldx = ldr = H
    _packed(weight, (H,), act, dev, "weight")
    if out is None:
        with torch.cuda.stream(stream):
            out = norm_buffers(T, H, act, residual is not None, y16, y8, x.device)
    s, y, q, qs = out
    _packed(s, (T, H), act, dev, "the sum")
    _packed(y, (T, H), act, dev, "y16")
    _packed(q, (T, H), _F8, dev, "y8")
    _packed(qs, (T, H // 128), torch.float32, dev, "y8_scale")
    _call(dev, pw.pw_rms_norm, x.data_ptr(), ldx, _ptr(residual), ldr, _ptr(weight), T, H, eps, _TYPE[act], _ptr(s), _ptr(y),
          _ptr(q), _ptr(qs), _on(dev, stream))
    return out


# ---------------------------------------------------------------------------
# 8-bit product
# ---------------------------------------------------------------------------

class Linear8:
    """y = x W^T of 8-bit rows: W [N, K] e4m3 with one scale per 128 x 128
    block [ceil(N / 128), K / 128]. The weights are packed into tiles here
    (pw_gemm_fp8_pack, on the current stream or ``stream``); w8 itself is not
    kept."""

    def __init__(self, w8: torch.Tensor, w_scale: torch.Tensor, stream=None):
        self.dev = dev = w8.get_device()
        _need(w8.dtype is _F8 and w8.dim() == 2 and w8.stride(1) == 1 and dev >= 0, "w8 must be e4m3 rows on the device")
        self.N, self.K = w8.shape
        _need(self.K % 128 == 0, "K must be a multiple of 128")
        _packed(w_scale, (-(-self.N // 128), self.K // 128), torch.float32, dev, "w_scale")
        self.w_scale = w_scale
        self.packed = _empty(pw.pw_gemm_fp8_packed_bytes(self.N, self.K), torch.uint8, w8.device, stream)
        _call(dev, pw.pw_gemm_fp8_pack, w8.data_ptr(), w8.stride(0) if self.N > 1 else self.K, self.N, self.K,
              self.packed.data_ptr(), _on(dev, stream))
        if stream is not None:
            w8.record_stream(stream)       # the caller may drop it before the packing has run
        self._ws = Workspace(w8.device)

    def forward(self, x8: torch.Tensor, x_scale: torch.Tensor, out: torch.Tensor = None, dtype=torch.bfloat16,
                stream=None) -> torch.Tensor:
        """x8 [M, K] e4m3 rows with x_scale [M, K / 128] (as rms_norm gives
        them) -> [M, N] (pw_gemm_fp8)."""
        M, N, K, dev = x8.shape[0], self.N, self.K, self.dev
        _need(x8.dtype is _F8 and x8.shape == (M, K) and x8.get_device() == dev and x8.stride(1) == 1,
              "x8 must be [M, K] e4m3 rows on the weights' device")
        _packed(x_scale, (M, K // 128), torch.float32, dev, "x_scale")
        if out is None:
            out = _empty((M, N), dtype, x8.device, stream)
        _need(out.shape == (M, N) and out.dtype in _TYPE and out.get_device() == dev and (N == 1 or out.stride(1) == 1),
              "out must be [M, N] rows on the weights' device")
        args = (x8.data_ptr(), x8.stride(0) if M > 1 else K, x_scale.data_ptr(), self.packed.data_ptr(),
                self.w_scale.data_ptr(), M, N, K, out.data_ptr(), out.stride(0) if M > 1 else N, _TYPE[out.dtype])
        self._ws.run(dev, stream, pw.pw_gemm_fp8, args, lambda: pw.pw_gemm_fp8_workspace(M, N, K))
        return out


# ---------------------------------------------------------------------------
# Heads of queries and keys
# ---------------------------------------------------------------------------

class Rotation:
    """A position rotation of the first ``dims`` channels of a head (pw_rotation):
    pair i by position * inv_freq[i], by default base^(-2 i / dims); pairs (i, i +
    dims / 2), or neighbours where ``interleaved``."""

    def __init__(self, dims: int, base: float = 10000.0, inv_freq: torch.Tensor = None, amplitude: float = 1.0,
                 interleaved: bool = False, device="cuda"):
        _need(dims >= 0 and dims % 16 == 0, "dims must be a multiple of 16")
        if inv_freq is None:
            inv_freq = (base ** (-torch.arange(0, dims, 2, dtype=torch.float64) / max(dims, 1))).to(device)
        _need(inv_freq.shape == (dims // 2,), "inv_freq must be [dims / 2]")
        self.inv_freq = inv_freq.to(torch.float64).contiguous()
        self.dev = self.inv_freq.get_device()
        _need(self.dev >= 0, "inv_freq must lie on the device")
        self.dims, self.interleaved, self.amplitude = dims, interleaved, amplitude
        self.desc = pw.pw_rotation(self.inv_freq.data_ptr(), dims, int(interleaved), amplitude)


def _rows(t: Optional[torch.Tensor], T: int, D: int, act: torch.dtype, dev: int, name: str):
    """(address, heads, row stride, head stride) of heads [T, n, D]; nothing for None."""
    if t is None:
        return 0, 0, 0, 0
    rows, n, width = t.shape
    ld, ldh, inner = t.stride()
    if rows != T or width != D or t.dtype is not act or inner != 1 or t.get_device() != dev:
        raise ValueError("%s must be [%d, heads, %d], %s, on device %d, with contiguous channels" % (name, T, D, act, dev))
    return t.data_ptr(), n, ld if T > 1 else 0, ldh if n > 1 else 0   # a single row, or head, may have any stride


def _turned(rotation: Optional[Rotation], positions: Optional[torch.Tensor], T: int, dev: int):
    """The library's rotation and the positions' address."""
    if rotation is None or rotation.dims == 0:
        _packed(positions, (T,), torch.int32, dev, "positions")
        return None, 0
    _need(rotation.dev == dev, "the rotation lies on another device")
    _need(positions is not None, "a rotation needs positions")
    _packed(positions, (T,), torch.int32, dev, "positions")
    return rotation.desc, positions.data_ptr()


def norm_rotate(q: torch.Tensor, k: Optional[torch.Tensor], positions: Optional[torch.Tensor], rotation: Optional[Rotation],
                q_weight: torch.Tensor = None, k_weight: torch.Tensor = None, *, norm: bool = True, eps: float = 1e-6,
                offset: int = 0, out=None, stream=None):
    """Queries [T, heads, head_dim] and keys (or None) normed by head where
    ``norm``, then turned by positions [T] int32 + offset: (q, k) in new tensors or
    those of ``out``, which may be q and k themselves (pw_heads_norm_rotate)."""
    T, n, D = q.shape
    act, dev = q.dtype, q.get_device()
    _int32(offset, "offset")
    _need((act is torch.bfloat16 or act is torch.float16) and dev >= 0, "q must be 16-bit heads on the device")
    rot, pos = _turned(rotation, positions, T, dev)
    q_ptr, n_q, ldq, ldqh = _rows(q, T, D, act, dev, "q")
    k_ptr, n_k, ldk, ldkh = _rows(k, T, D, act, dev, "k")
    _packed(q_weight, (D,), act, dev, "q_weight")
    _packed(k_weight, (D,), act, dev, "k_weight")
    if out is None:
        out = (_empty(q.shape, act, q.device, stream), None if k is None else _empty(k.shape, act, q.device, stream))
    qo, ko = out
    _need(qo.shape == q.shape and (ko is None) == (k is None) and (k is None or ko.shape == k.shape),
          "out must have the shapes of q and k")
    qo_ptr, _, ldqo, ldqoh = _rows(qo, T, D, act, dev, "out")
    ko_ptr, _, ldko, ldkoh = _rows(ko, T, D, act, dev, "out")
    _call(dev, pw.pw_heads_norm_rotate, rot, pos, offset, q_ptr, ldq, ldqh, n_q, k_ptr, ldk, ldkh, n_k, _ptr(q_weight),
          _ptr(k_weight), int(norm), eps, T, D, _TYPE[act], qo_ptr, ldqo, ldqoh, ko_ptr, ldko, ldkoh, _on(dev, stream))
    return qo, ko


# ---------------------------------------------------------------------------
# KV cache
# ---------------------------------------------------------------------------

class KVCache:
    """Paged keys and values of one attention layer: n_blocks blocks of
    block_tokens tokens, in ``act`` or (fp8) as e4m3 codes with a scale per
    token and head. ``pool``: a uint8 device tensor to keep the blocks in (e.g.
    one that also holds weight pages), block i at byte i * block_stride.
    ``workspace``: one that other caches have, too. The parts of split sequences
    lie there, hundreds of MB for large batches of long ones (16 trees of 60
    tokens after up to 32768: 392 MB, kept as 512): a model's layers, which run
    one after the other, need them once."""

    def __init__(self, n_blocks: int, block_tokens: int, kv_heads: int, head_dim: int, act: torch.dtype, fp8: bool = False,
                 pool: torch.Tensor = None, block_stride: int = None, device="cuda", workspace: Workspace = None):
        _need(act in (torch.float16, torch.bfloat16), "act must be a 16-bit type")
        self.act, self.head_dim, self.kv_heads, self.block_tokens = act, head_dim, kv_heads, block_tokens
        self.desc = pw.pw_kv_cache(None, 0, n_blocks, block_tokens, kv_heads, head_dim, _TYPE[act], 8 if fp8 else 16)
        self.block_bytes = pw.pw_kv_block_bytes(self.desc)
        self.desc.block_stride = block_stride or self.block_bytes
        if pool is None:
            pool = torch.empty(max(n_blocks - 1, 0) * self.desc.block_stride + self.block_bytes, dtype=torch.uint8, device=device)
        self.dev = pool.get_device()
        _need(pool.dtype == torch.uint8 and pool.is_contiguous() and self.dev >= 0, "the pool must be contiguous device bytes")
        _need(pool.numel() >= (n_blocks - 1) * self.desc.block_stride + self.block_bytes, "the pool is smaller than its blocks")
        self.pool = pool
        self.desc.pool = pool.data_ptr()
        _need(workspace is None or workspace.device == pool.device, "the workspace lies on another device")
        self._ws = workspace or Workspace(pool.device)

    def append(self, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, stream=None):
        """Write k, v [T, kv_heads, head_dim] to the slots [T] int64 (block *
        block_tokens + position in it; negative: nothing) (pw_kv_append)."""
        T, dev = k.shape[0], self.dev
        _need(k.shape == (T, self.kv_heads, self.head_dim) and v.shape == k.shape, "k and v must be [T, kv_heads, head_dim]")
        ld, ldh, inner = k.stride()
        ldv, ldvh, inner_v = v.stride()
        if T <= 1:                         # a single row, or head, may have any stride
            ld = ldv = 0
        if self.kv_heads == 1:
            ldh = ldvh = 0
        _need(k.dtype is self.act and v.dtype is self.act and k.get_device() == dev and v.get_device() == dev
              and ld == ldv and ldh == ldvh and inner == 1 and inner_v == 1,
              "k and v must be of the cache's type and device, with equal strides and contiguous channels")
        _packed(slots, (T,), torch.int64, dev, "slots")
        _call(dev, pw.pw_kv_append, self.desc, k.data_ptr(), v.data_ptr(), ld, ldh, slots.data_ptr(), T, _on(dev, stream))

    def attend(self, q: torch.Tensor, block_table: torch.Tensor, lens: torch.Tensor, max_len: int, scale: float = None,
               window: int = 0, out: torch.Tensor = None, lse: torch.Tensor = None, stream=None) -> torch.Tensor:
        """Attention of one token per sequence: q [B, heads, head_dim] over the
        first lens[b] cached tokens of the blocks block_table[b] (the last
        ``window`` of them) -> [B, heads, head_dim] (pw_attn_decode)."""
        B, heads, D = q.shape
        dev = self.dev
        _int32(max_len, "max_len")
        _int32(window, "window")
        ldq, ldqh, inner = q.stride()
        if B <= 1:                         # a single sequence, or head, may have any stride
            ldq = 0
        if heads == 1:
            ldqh = 0
        _need(q.dtype is self.act and D == self.head_dim and q.get_device() == dev and inner == 1,
              "q must be [B, heads, head_dim] of the cache's type and device")
        rows, blocks = block_table.shape
        _need(block_table.dtype is torch.int32 and rows == B and block_table.get_device() == dev
              and (block_table.stride(1) == 1 or blocks <= 1), "block_table must be [B, blocks] int32 on the cache's device")
        _packed(lens, (B,), torch.int32, dev, "lens")
        _need(blocks * self.block_tokens >= max_len, "the block table is shorter than max_len")
        if out is None:
            out = _empty((B, heads, D), self.act, q.device, stream)
        _packed(out, (B, heads, D), self.act, dev, "out")
        _packed(lse, (B, heads), torch.float32, dev, "lse")
        args = (self.desc, q.data_ptr(), ldq, ldqh, heads, block_table.data_ptr(), block_table.stride(0) if B > 1 else blocks,
                lens.data_ptr(), B, max_len, D ** -0.5 if scale is None else scale, window, out.data_ptr(), _ptr(lse))
        self._ws.run(dev, stream, pw.pw_attn_decode, args,
                     lambda: pw.pw_attn_workspace(self.desc, B, heads, max_len, window))
        return out


    def append_rotated(self, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, positions: Optional[torch.Tensor],
                       rotation: Optional[Rotation], q: torch.Tensor = None, q_weight: torch.Tensor = None,
                       k_weight: torch.Tensor = None, *, norm: bool = True, eps: float = 1e-6, offset: int = 0,
                       q_out: torch.Tensor = None, stream=None) -> Optional[torch.Tensor]:
        """``norm_rotate`` of q [T, heads, head_dim] (or None) and k, with k and v
        written to the slots as ``append`` does: q in a new tensor or in ``q_out``,
        which may be q itself (pw_kv_append_rotated)."""
        T, D, dev, act = k.shape[0], self.head_dim, self.dev, self.act
        _int32(offset, "offset")
        k_ptr, n_k, ld, ldh = _rows(k, T, D, act, dev, "k")
        v_ptr, n_v, ldv, ldvh = _rows(v, T, D, act, dev, "v")
        _need(n_k == self.kv_heads and n_v == n_k and ld == ldv and ldh == ldvh,
              "k and v must be [T, kv_heads, head_dim] with equal strides")
        _packed(slots, (T,), torch.int64, dev, "slots")
        rot, pos = _turned(rotation, positions, T, dev)
        _packed(q_weight, (D,), act, dev, "q_weight")
        _packed(k_weight, (D,), act, dev, "k_weight")
        if q is not None and q_out is None:
            q_out = _empty(q.shape, act, q.device, stream)
        _need((q is None) == (q_out is None) and (q is None or q_out.shape == q.shape), "q_out must have q's shape")
        q_ptr, n_q, ldq, ldqh = _rows(q, T, D, act, dev, "q")
        qo_ptr, _, ldqo, ldqoh = _rows(q_out, T, D, act, dev, "q_out")
        _call(dev, pw.pw_kv_append_rotated, self.desc, rot, pos, offset, q_ptr, ldq, ldqh, n_q, k_ptr, v_ptr, ld, ldh,
              _ptr(q_weight), _ptr(k_weight), int(norm), eps, slots.data_ptr(), T, qo_ptr, ldqo, ldqoh, _on(dev, stream))
        return q_out

    def _table(self, block_table: torch.Tensor, B: int, max_len: int):
        """(address, row stride) of a block table."""
        rows, blocks = block_table.shape
        _int32(max_len, "max_len")
        _need(block_table.dtype is torch.int32 and rows == B and block_table.get_device() == self.dev
              and (block_table.stride(1) == 1 or blocks <= 1), "block_table must be [B, blocks] int32 on the cache's device")
        _need(blocks * self.block_tokens >= max_len, "the block table is shorter than max_len")
        return block_table.data_ptr(), block_table.stride(0) if B > 1 else blocks

    def attend_rows(self, q: torch.Tensor, starts: torch.Tensor, block_table: torch.Tensor, lens: torch.Tensor, max_len: int,
                    masks: torch.Tensor = None, scale: float = None, window: int = 0, out: torch.Tensor = None,
                    lse: torch.Tensor = None, stream=None) -> torch.Tensor:
        """Attention of several new tokens per sequence: rows starts[b] .. starts[b
        + 1] - 1 of q [T, heads, head_dim] are the last of the lens[b] cached tokens
        of the blocks block_table[b]. Each sees the tokens up to itself, or with
        ``masks`` [T, words] int64 the context and the new tokens whose bits are set
        -> [T, heads, head_dim]; rows of no sequence are not written
        (pw_attn_rows)."""
        T, heads, D = q.shape
        dev, B = self.dev, lens.shape[0]
        _int32(window, "window")
        q_ptr, _, ldq, ldqh = _rows(q, T, self.head_dim, self.act, dev, "q")
        _packed(starts, (B + 1,), torch.int32, dev, "starts")
        _packed(lens, (B,), torch.int32, dev, "lens")
        words = 0 if masks is None else masks.shape[1]
        _need(masks is None or words > 0, "masks must have at least one word")
        _packed(masks, (T, words), torch.int64, dev, "masks")
        table, ld_table = self._table(block_table, B, max_len)
        if out is None:
            out = _empty((T, heads, D), self.act, q.device, stream)
        _packed(out, (T, heads, D), self.act, dev, "out")
        _packed(lse, (T, heads), torch.float32, dev, "lse")
        args = (self.desc, q_ptr, ldq, ldqh, heads, starts.data_ptr(), T, _ptr(masks), words, table, ld_table, lens.data_ptr(), B,
                max_len, D ** -0.5 if scale is None else scale, window, out.data_ptr(), _ptr(lse))
        self._ws.run(dev, stream, pw.pw_attn_rows, args,
                     lambda: pw.pw_attn_rows_workspace(self.desc, B, T, heads, max_len, window))
        return out

    def keep(self, starts: torch.Tensor, block_table: torch.Tensor, lens: torch.Tensor, max_len: int, chosen: torch.Tensor,
             out: torch.Tensor = None, stream=None) -> torch.Tensor:
        """Of each sequence's new tokens (as in ``attend_rows``) move the chosen
        ones, by bits [B, words] int64, together behind the context -> the new
        lengths [B] int32 (pw_kv_keep)."""
        dev, B = self.dev, lens.shape[0]
        _packed(starts, (B + 1,), torch.int32, dev, "starts")
        _packed(lens, (B,), torch.int32, dev, "lens")
        words = chosen.shape[1]
        _packed(chosen, (B, words), torch.int64, dev, "chosen")
        table, ld_table = self._table(block_table, B, max_len)
        if out is None:
            out = _empty((B,), torch.int32, lens.device, stream)
        _packed(out, (B,), torch.int32, dev, "out")
        _call(dev, pw.pw_kv_keep, self.desc, starts.data_ptr(), table, ld_table, lens.data_ptr(), B, max_len, chosen.data_ptr(),
              words, out.data_ptr(), _on(dev, stream))
        return out


# ---------------------------------------------------------------------------
# Routing
# ---------------------------------------------------------------------------

_SCORE = {"softmax": pw.PW_SCORE_SOFTMAX, "sigmoid": pw.PW_SCORE_SIGMOID}


def route_grouped(logits: torch.Tensor, K: int, score: str = "softmax", bias: torch.Tensor = None, groups: int = 1,
                  top_groups: int = 1, group_top: int = 1, renorm: bool = True, scale: float = 1.0, n_shared: int = 0,
                  gate: torch.Tensor = None, out=None, stream=None):
    """Routing for PagedLayer.forward from logits [T, E]: (ids, w, offsets,
    sorted_slot, slot_pos), n_shared shared-expert columns after the K routed
    ones (pw_route_grouped)."""
    T, E = logits.shape
    dev = logits.get_device()
    _need(logits.dtype in _TYPE and dev >= 0 and logits.is_contiguous(), "logits must be packed fp32, fp16 or bf16 rows")
    _need(score in _SCORE, "score must be softmax or sigmoid")
    _packed(bias, (E,), torch.float32, dev, "bias")
    _packed(gate, (T, n_shared), torch.float32, dev, "gate")
    Kt = K + n_shared
    if out is None:
        with torch.cuda.stream(stream):
            out = PagedLayer.routing_buffers(T, E + n_shared, Kt, logits.device)
        ids, w, offsets, ss, sp = out
    else:
        ids, w, offsets, ss, sp = out
        _packed(ids, (T, Kt), torch.int32, dev, "ids")
        _packed(w, (T, Kt), torch.float32, dev, "w")
        for t, n in ((offsets, E + n_shared + 1), (ss, T * Kt), (sp, T * Kt)):
            _need(t.dtype is torch.int32 and t.get_device() == dev and t.is_contiguous() and t.numel() >= n,
                  "the routing buffers are of another kind (PagedLayer.routing_buffers)")
    _call(dev, pw.pw_route_grouped, logits.data_ptr(), _TYPE[logits.dtype], _ptr(bias), T, E, K, _SCORE[score], groups,
          top_groups, group_top, int(renorm), scale, n_shared, _ptr(gate), ids.data_ptr(), w.data_ptr(), offsets.data_ptr(),
          ss.data_ptr(), sp.data_ptr(), _on(dev, stream))
    return ids, w, offsets, ss, sp
