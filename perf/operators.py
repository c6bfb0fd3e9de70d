"""Timed calls of the operators around the paged MoE layer: what a decoder
layer runs besides its experts.

``norm``   root-mean-square norm with the residual's addition; 16-bit rows for
           the router and the experts, 8-bit rows with scales for a projection
``gemm``   8-bit floating-point product, one scale per token and 128 columns of
           the activation and one per 128 x 128 block of the weight
``append`` new keys and values written into the paged cache
``attn``   attention of one new token per sequence over the paged cache
``route``  grouped top-k routing (softmax or sigmoid scores, a balancing bias,
           groups, renormalised weights) with the expert-major permutation

The widths are those of the layers in ``paper_2607_16184_amd.synth`` (hidden
4096 and 2048, FFN 14336, 8 to 64 routed experts, up to 256 as the router
admits); batches go from one token to a prefill chunk of 4096.

With ``own`` false a pass computes the operator from elementary tensor
operations in 32 bits; with ``own`` true it calls the framework.
"""
from __future__ import annotations

import math
import random

import torch

own = False

F8_MAX = 448.0                  # largest finite e4m3 value
MIN_SCALE = 2.0 ** -126         # smallest scale (the smallest normal fp32)
_DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_F8 = torch.float8_e4m3fn


def listed():
    return [
        # one sequence, a short chat turn: latency alone
        dict(name="attn_1", kind="attn", B=1, L=300, Hkv=8, g=4, D=128, P=32, act="bf16", fp8=False, window=0, ragged=False),
        # a batch of 64 sequences of all lengths, some slots of it empty, one
        # key head per query head, sliding window, fp16
        dict(name="attn_64", kind="attn", B=64, L=4096, Hkv=16, g=1, D=64, P=64, act="f16", fp8=False, window=1500, ragged=True),
        # long contexts in 8 bits, the largest cache
        dict(name="attn_long", kind="attn", B=16, L=32768, Hkv=8, g=4, D=128, P=64, act="bf16", fp8=True, window=0, ragged=True),
        # a decode step's new tokens, one per sequence, some of them padding
        dict(name="append_64", kind="append", T=64, Hkv=8, D=128, P=32, act="bf16", fp8=False, prefill=False),
        # a prefill chunk written in 8 bits; it starts and ends inside a block
        dict(name="append_4001", kind="append", T=4001, Hkv=8, D=128, P=64, act="bf16", fp8=True, prefill=True),
        # a decode batch of the fine-grained layer: softmax, no groups
        dict(name="route_33", kind="route", T=33, E=60, K=4, score="softmax", bias=False, groups=1, top_groups=1, group_top=1,
             renorm=False, scale=1.0, n_shared=4, logits="f32"),
        # a prefill chunk of the widest layer: sigmoid scores, bias, groups
        dict(name="route_4096", kind="route", T=4096, E=256, K=8, score="sigmoid", bias=True, groups=8, top_groups=4, group_top=2,
             renorm=True, scale=2.5, n_shared=0, logits="f32"),
        # a decode batch: sum, norm and the 8-bit rows of the next projection
        dict(name="norm_64", kind="norm", T=64, H=4096, act="bf16", res=True, y16=False, y8=True),
        # a prefill chunk with an odd end, both forms of the output
        dict(name="norm_4095", kind="norm", T=4095, H=4096, act="bf16", res=True, y16=True, y8=True),
        # the query/key/value projection of a decode batch
        dict(name="gemm_16", kind="gemm", M=16, N=6144, K=4096, out="bf16"),
        # the same of a ragged chunk, with a width that ends inside a block
        dict(name="gemm_777", kind="gemm", M=777, N=4000, K=2048, out="f16"),
        # a prefill chunk through a dense gate/up projection: the largest case
        dict(name="gemm_4096", kind="gemm", M=4096, N=28672, K=4096, out="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above, of sizes that these layers have."""
    while True:
        c = _draw(rng)
        if not any(v == 3072 for v in (*c.values(), c.get("g", 0) * c.get("Hkv", 0) * c.get("D", 0))):
            return c


def _draw(rng):
    kind = rng.choice(["attn", "attn", "append", "route", "norm", "gemm", "gemm"])
    act = rng.choice(["bf16", "bf16", "f16"])
    if kind == "attn":
        c = dict(kind=kind, B=_log(rng, 1, 96), L=_log(rng, 1, 32768), Hkv=rng.choice([1, 2, 4, 8, 8, 16]),
                 g=rng.choice([1, 2, 4, 5, 7, 8, 16, 24]), D=rng.choice([64, 128, 128, 192, 256]), P=rng.choice([32, 64, 128]),
                 act=act, fp8=rng.random() < 0.4, window=0, ragged=rng.random() < 0.7)
        if rng.random() < 0.3:
            c["window"] = _log(rng, 1, 4096)
        # a cache no larger than the largest listed one, and as much work
        # besides: sequences are dropped, then shortened
        most = min(9 * 32768 * 8 * 128, 9 * 32768 * 32 * 128 // c["g"]) // (1 if c["fp8"] else 2)
        c["B"] = max(1, min(c["B"], most // (c["L"] * c["Hkv"] * c["D"])))
        c["L"] = max(1, min(c["L"], most // (c["B"] * c["Hkv"] * c["D"])))
        return c
    if kind == "append":
        return dict(kind=kind, T=_log(rng, 1, 4000), Hkv=rng.choice([1, 2, 4, 8]), D=rng.choice([64, 128, 128, 192, 256]),
                    P=rng.choice([32, 64, 128]), act=act, fp8=rng.random() < 0.5, prefill=rng.random() < 0.5)
    if kind == "route":
        groups = rng.choice([1, 1, 4, 8])
        E = groups * rng.randint(max(2, 8 // groups), 256 // groups)
        top_groups = rng.randint(1, groups)
        K = rng.randint(1, min(8, top_groups * (E // groups)))
        sig = rng.random() < 0.5
        return dict(kind=kind, T=_log(rng, 1, 4000), E=E, K=K, score="sigmoid" if sig else "softmax", bias=rng.random() < 0.6,
                    groups=groups, top_groups=top_groups, group_top=rng.choice([1, 2]), renorm=rng.random() < 0.7,
                    scale=rng.choice([1.0, 2.5]), n_shared=rng.choice([0, 0, 1]) if E < 256 else 0,
                    logits=rng.choice(["f32", "f32", act]))
    if kind == "norm":
        y8 = rng.random() < 0.6
        H = 128 * rng.randint(2, 32) if y8 else 8 * rng.randint(32, 512)
        return dict(kind=kind, T=_log(rng, 1, 4000), H=H, act=act, res=rng.random() < 0.7, y16=not y8 or rng.random() < 0.5, y8=y8)
    return dict(kind=kind, M=_log(rng, 1, 4096), N=_log(rng, 100, 14336), K=128 * _log(rng, 2, 32), out=rng.choice([act, act, "f32"]))


# ---------------------------------------------------------------------------
# The cache's layout
# ---------------------------------------------------------------------------
# A block holds P tokens of all key heads: per head its keys, then its values,
# then (8 bits) the keys' scales [Hkv][P] and the values' scales [Hkv][P] in
# fp32. Keys lie in tiles of 16 tokens, values in tiles of 32 tokens, in the
# order in which the matrix instructions take them.

def _elt(c):
    return 1 if c["fp8"] else 2


def _block_bytes(c):
    return 2 * c["Hkv"] * c["P"] * c["D"] * _elt(c) + (8 * c["Hkv"] * c["P"] if c["fp8"] else 0)


def _tiles_k(k, c):
    """[n, Hkv, P, D] in token order -> tile order, flat per head."""
    n, h, P, D = k.shape
    if c["fp8"]:
        return k.view(n, h, P // 16, 16, D // 64, 2, 4, 8).permute(0, 1, 2, 4, 6, 3, 5, 7).reshape(n, h, P * D)
    return k.view(n, h, P // 16, 16, D // 32, 4, 8).permute(0, 1, 2, 4, 5, 3, 6).reshape(n, h, P * D)


def _tiles_v(v, c):
    n, h, P, D = v.shape
    if c["fp8"]:
        return v.view(n, h, P // 32, 2, 4, 4, D // 32, 2, 16).permute(0, 1, 2, 6, 4, 8, 7, 3, 5).reshape(n, h, P * D)
    return v.view(n, h, P // 32, 2, 4, 4, D // 16, 16).permute(0, 1, 2, 6, 4, 7, 3, 5).reshape(n, h, P * D)


def _untile_k(k, c):
    n, h, P, D = k.shape[0], c["Hkv"], c["P"], c["D"]
    if c["fp8"]:
        return k.view(n, h, P // 16, D // 64, 4, 16, 2, 8).permute(0, 1, 2, 5, 3, 6, 4, 7).reshape(n, h, P, D)
    return k.view(n, h, P // 16, D // 32, 4, 16, 8).permute(0, 1, 2, 5, 3, 4, 6).reshape(n, h, P, D)


def _untile_v(v, c):
    n, h, P, D = v.shape[0], c["Hkv"], c["P"], c["D"]
    if c["fp8"]:
        return v.view(n, h, P // 32, D // 32, 4, 16, 2, 2, 4).permute(0, 1, 2, 7, 4, 8, 3, 6, 5).reshape(n, h, P, D)
    return v.view(n, h, P // 32, D // 16, 4, 16, 2, 4).permute(0, 1, 2, 6, 4, 7, 3, 5).reshape(n, h, P, D)


def _div(a, b):
    # (a division by a Python number multiplies by its reciprocal on the GPU)
    return a / torch.full_like(a, b)


def _quant(x, group):
    """8-bit codes and scales of groups of the last dimension: s = max(amax /
    448, 2^-126), code = e4m3(x / s)."""
    v = x.float().unflatten(-1, (-1, group))
    s = _div(v.abs().amax(-1), F8_MAX).clamp_min(MIN_SCALE)
    return (v / s[..., None]).to(_F8).flatten(-2), s


def _gen(seed, stream):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 100003 + stream)


def _blocks_of(c, n, seed):
    """n blocks of cached keys and values in token order: (k, v) in the
    activation's type, or 8-bit codes with their scales (k, v, ks, vs)."""
    out, scales = [], []
    for i in (0, 1):
        x = torch.randn((n, c["Hkv"], c["P"], c["D"]), generator=_gen(seed, 20 + i), device="cuda").to(_DT[c["act"]])
        if c["fp8"]:
            q, s = _quant(x, c["D"])
            out.append(q)
            scales.append(s[..., 0])
        else:
            out.append(x)
    return out + scales


def _laid_out(parts, c, n_spare):
    """The pool of the blocks in `parts`, with n_spare blocks after them."""
    n = parts[0].shape[0]
    pool = torch.zeros((n + n_spare, _block_bytes(c)), dtype=torch.uint8, device="cuda")
    half = c["P"] * c["D"] * _elt(c)
    heads = pool[:n, :2 * c["Hkv"] * half].view(n, c["Hkv"], 2 * half)
    heads[:, :, :half] = _tiles_k(parts[0], c).view(torch.uint8)
    heads[:, :, half:] = _tiles_v(parts[1], c).view(torch.uint8)
    if c["fp8"]:
        s = torch.stack([parts[2], parts[3]], 1).reshape(n, -1)
        pool[:n, 2 * c["Hkv"] * half:] = s.view(torch.uint8)
    return pool


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _lens(c):
    """Cached tokens per sequence, the new one among them (0: an empty slot of
    the batch). Ragged batches spread over the range by the golden section."""
    B, L = c["B"], c["L"]
    if not c["ragged"]:
        return [L] * B
    lens = [1 + int(L * ((0.618034 * (i + 1)) % 1.0)) for i in range(B)]
    lens[0] = L
    for i in range(7, B, 16):
        lens[i] = 0
    return [min(n, L) for n in lens]


def _attn_inputs(c, seed):
    lens = _lens(c)
    random.Random(int(seed) * 7919 + 3).shuffle(lens)
    nb = -(-c["L"] // c["P"])
    n = c["B"] * nb
    g = _gen(seed, 1)
    # queries lie in the rows of the fused query/key/value projection
    rows = torch.randn((c["B"], (c["g"] + 2) * c["Hkv"] * c["D"]), generator=g, device="cuda").to(_DT[c["act"]])
    table = torch.randperm(n, generator=g, device="cuda").to(torch.int32).view(c["B"], nb)
    return rows, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), n


def _append_inputs(c, seed):
    T, P = c["T"], c["P"]
    g = _gen(seed, 1)
    rows = torch.randn((T, 2 * c["Hkv"] * c["D"]), generator=g, device="cuda").to(_DT[c["act"]])
    rows = rows * torch.exp(torch.randn((T, 1), generator=g, device="cuda")).to(rows.dtype)
    if c["prefill"]:                   # consecutive positions of one sequence
        n = -(-(T + P // 2 + 1) // P)
        blocks = torch.randperm(n, generator=g, device="cuda")
        pos = torch.arange(T, device="cuda") + P // 2 + 1
        slots = blocks[pos // P] * P + pos % P
    else:                              # one position of each sequence
        n = 2 * T
        slots = torch.randperm(n, generator=g, device="cuda")[:T] * P + torch.randint(0, P, (T,), generator=g, device="cuda")
        slots[5::9] = -1               # padding rows write nothing
    return rows, slots, n


def _route_inputs(c, seed):
    g = _gen(seed, 1)
    logits = torch.randn((c["T"], c["E"]), generator=g, device="cuda") + torch.randn(c["E"], generator=g, device="cuda") * 0.5
    bias = torch.randint(-100, 101, (c["E"],), generator=g, device="cuda").float() * 1e-3 if c["bias"] else None
    gate = torch.rand((c["T"], c["n_shared"]), generator=g, device="cuda") if c["n_shared"] else None
    return logits.to(_DT[c["logits"]]), bias, gate


def _norm_inputs(c, seed):
    g = _gen(seed, 1)
    x = torch.randn((c["T"], c["H"]), generator=g, device="cuda").to(_DT[c["act"]])
    r = torch.randn((c["T"], c["H"]), generator=g, device="cuda").mul_(3.0).to(_DT[c["act"]]) if c["res"] else None
    w = torch.rand(c["H"], generator=g, device="cuda").add_(0.5).to(_DT[c["act"]])
    return x, r, w


def _gemm_inputs(c, seed):
    g = _gen(seed, 1)
    M, N, K = c["M"], c["N"], c["K"]
    a8, a_s = _quant(torch.randn((M, K), generator=g, device="cuda"), 128)
    w = torch.randn((N, K), generator=g, device="cuda").mul_(0.02)
    nb = -(-N // 128)
    blocks = torch.nn.functional.pad(w, (0, 0, 0, nb * 128 - N)).view(nb, 128, K // 128, 128)
    w_s = _div(blocks.abs().amax((1, 3)), F8_MAX).clamp_min(MIN_SCALE)
    w8 = (blocks / w_s[:, None, :, None]).view(nb * 128, K)[:N].to(_F8)
    return a8, a_s, w8, w_s


def prepare(case, seed):
    """The inputs, and the buffers and handles that a serving loop keeps."""
    c = dict(case)
    kind = c["kind"]
    s = dict(c=c, kind=kind)
    if own:
        from paper_2607_16184_amd import ops
        s["ops"] = ops
    if kind == "attn":
        rows, table, lens, n = _attn_inputs(c, seed)
        s.update(rows=rows, table=table, lens=lens, pool=_laid_out(_blocks_of(c, n, seed), c, 0), n=n)
        s["out"] = torch.empty((c["B"], c["g"] * c["Hkv"], c["D"]), dtype=rows.dtype, device="cuda")
    elif kind == "append":
        rows, slots, n = _append_inputs(c, seed)
        # the spare block takes what the plain form writes for padding rows
        s.update(rows=rows, slots=slots, pool=_laid_out(_blocks_of(c, n, seed), c, 1), n=n)
    elif kind == "route":
        logits, bias, gate = _route_inputs(c, seed)
        s.update(logits=logits, bias=bias, gate=gate)
        Kt, E = c["K"] + c["n_shared"], c["E"] + c["n_shared"]
        s["out"] = (torch.empty((c["T"], Kt), dtype=torch.int32, device="cuda"),
                    torch.empty((c["T"], Kt), dtype=torch.float32, device="cuda"),
                    torch.empty(E + 1, dtype=torch.int32, device="cuda"),
                    torch.empty(c["T"] * Kt, dtype=torch.int32, device="cuda"),
                    torch.empty(c["T"] * Kt, dtype=torch.int32, device="cuda"))
    elif kind == "norm":
        x, r, w = _norm_inputs(c, seed)
        T, H = c["T"], c["H"]
        s.update(x=x, r=r, w=w)
        s["out"] = (torch.empty_like(x) if c["res"] else None, torch.empty_like(x) if c["y16"] else None,
                    torch.empty((T, H), dtype=_F8, device="cuda") if c["y8"] else None,
                    torch.empty((T, H // 128), dtype=torch.float32, device="cuda") if c["y8"] else None)
    else:
        a8, a_s, w8, w_s = _gemm_inputs(c, seed)
        s.update(a8=a8, a_s=a_s, w8=w8, w_s=w_s, out=torch.empty((c["M"], c["N"]), dtype=_DT[c["out"]], device="cuda"))
    if own and kind in ("attn", "append"):
        s["cache"] = ops.KVCache(s["n"], c["P"], c["Hkv"], c["D"], _DT[c["act"]], fp8=c["fp8"], pool=s["pool"])
    if own and kind == "gemm":
        s["linear"] = ops.Linear8(s["w8"], s["w_s"])
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

EPS = 1e-5


def _cache_views(pool, c):
    """The cache's contents as values: keys and values, and the scales."""
    codes = 2 * c["Hkv"] * c["P"] * c["D"] * _elt(c)
    out = [pool[:, :codes].view(_F8 if c["fp8"] else _DT[c["act"]])]
    if c["fp8"]:
        out.append(pool[:, codes:].view(torch.float32))
    return out


def _plain_attn(s):
    c = s["c"]
    B, Hkv, P, D, g = c["B"], c["Hkv"], c["P"], c["D"], c["g"]
    n = B * s["table"].shape[1]
    blocks = s["pool"][s["table"].view(-1).long()]
    codes = 2 * Hkv * P * D * _elt(c)
    heads = blocks[:, :codes].contiguous().view(_F8 if c["fp8"] else _DT[c["act"]]).view(n, Hkv, 2, P * D)
    k = _untile_k(heads[:, :, 0].contiguous(), c).float()
    v = _untile_v(heads[:, :, 1].contiguous(), c).float()
    if c["fp8"]:
        sc = blocks[:, codes:].contiguous().view(torch.float32).view(n, 2, Hkv, P, 1)
        k, v = k * sc[:, 0], v * sc[:, 1]
    k = k.view(B, -1, Hkv, P, D).transpose(1, 2).reshape(B * Hkv, -1, D)
    v = v.view(B, -1, Hkv, P, D).transpose(1, 2).reshape(B * Hkv, -1, D)
    q = s["rows"][:, :g * Hkv * D].float().reshape(B * Hkv, g, D)
    sc = torch.bmm(q, k.transpose(1, 2).contiguous()).view(B, Hkv, g, -1) * D ** -0.5
    pos = torch.arange(k.shape[1], device="cuda")
    lens = s["lens"].long()[:, None]
    on = pos < lens
    if c["window"]:
        on = on & (pos >= lens - c["window"])
    sc = sc.masked_fill(~on[:, None, None], -math.inf)
    m = sc.amax(-1, keepdim=True).clamp_min(-3e38)       # an empty row has no maximum
    p = torch.exp(sc - m)
    den = p.sum(-1, keepdim=True)
    p = torch.where(den > 0, p / den, torch.zeros_like(p))
    o = torch.bmm(p.view(B * Hkv, g, -1), torch.where(on[:, None, :, None], v.view(B, Hkv, -1, D), 0.0).view(B * Hkv, -1, D))
    return o.view(B, Hkv * g, D).to(s["out"].dtype)


def _plain_append(s):
    c = s["c"]
    T, Hkv, P, D = c["T"], c["Hkv"], c["P"], c["D"]
    kv = s["rows"].view(T, 2, Hkv, D)
    keep = s["slots"] >= 0
    block = torch.where(keep, s["slots"] // P, s["n"])[:, None, None]    # the spare block takes padding
    t = (s["slots"] % P)[:, None, None]
    h = torch.arange(Hkv, device="cuda")[None, :, None]
    d = torch.arange(D, device="cuda")[None, None, :]
    lane = (t % 16 + 16 * (d // 8 % 4))
    e = _elt(c)
    if c["fp8"]:
        ko = (t // 16 * (D // 64) + d // 64) * 1024 + 16 * lane + d // 32 % 2 * 8 + d % 8
        vo = (t // 32 * (D // 32) + d // 32) * 1024 + 16 * (16 * (t // 4 % 4) + d % 16) + d // 16 % 2 * 8 + t // 16 % 2 * 4 + t % 4
    else:
        ko = (t // 16 * (D // 32) + d // 32) * 512 + 8 * lane + d % 8
        vo = (t // 32 * (D // 16) + d // 16) * 512 + 8 * (16 * (t // 4 % 4) + d % 16) + t // 16 % 2 * 4 + t % 4
    base = block * (_block_bytes(c) // e) + h * (2 * P * D)
    flat = s["pool"].view(-1)
    if c["fp8"]:
        codes, sc = _quant(kv, D)
        flat[base + ko] = codes[:, 0].view(torch.uint8)
        flat[base + P * D + vo] = codes[:, 1].view(torch.uint8)
        so = block[:, :, 0] * (_block_bytes(c) // 4) + 2 * Hkv * P * D // 4 + h[:, :, 0] * P + t[:, :, 0]
        flat.view(torch.float32)[so] = sc[:, 0, :, 0]
        flat.view(torch.float32)[so + Hkv * P] = sc[:, 1, :, 0]
    else:
        flat = flat.view(kv.dtype)
        flat[base + ko] = kv[:, 0]
        flat[base + P * D + vo] = kv[:, 1]
    return _cache_views(s["pool"][:s["n"]], c)


def _plain_route(s):
    c = s["c"]
    T, E, K, n_groups = c["T"], c["E"], c["K"], c["groups"]
    # The scores that decide which experts a token gets are held in 64 bits:
    # the choice then does not hang on the rounding of an exponential.
    x = s["logits"].double().clamp_max(3.0e38)
    off = torch.isnan(x) | (x == -math.inf)
    if c["score"] == "sigmoid":
        p = 1.0 / (1.0 + torch.exp(-x))
    else:
        p = torch.exp(x - x.masked_fill(off, -3.4e38).amax(1, keepdim=True)).masked_fill(off, 0.0)
        p = p / p.sum(1, keepdim=True)
    p = p.masked_fill(off, 0.0)
    choice = p if s["bias"] is None else p + s["bias"].double()
    choice = choice.masked_fill(off, -math.inf)
    if n_groups > 1:
        best = torch.sort(choice.view(T, n_groups, -1), dim=2, descending=True, stable=True).values[:, :, :c["group_top"]]
        score = torch.where(best > -math.inf, best, 0.0).sum(2).masked_fill(best[:, :, 0] == -math.inf, -math.inf)
        order = torch.sort(score, dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        inside = torch.zeros((T, n_groups), dtype=torch.bool, device="cuda").scatter_(1, order, True)
        choice = choice.masked_fill(~inside.repeat_interleave(E // n_groups, 1), -math.inf)
    top = torch.sort(choice, dim=1, descending=True, stable=True)
    ids = top.indices[:, :K]
    w = p.gather(1, ids).masked_fill(top.values[:, :K] == -math.inf, 0.0)
    if c["renorm"]:
        den = w.sum(1, keepdim=True)
        w = torch.where(den > 0, w / den, 0.0)
    w = (w * c["scale"]).float()
    if c["n_shared"]:
        ids = torch.cat([ids, torch.arange(E, E + c["n_shared"], device="cuda").expand(T, -1)], 1)
        w = torch.cat([w, s["gate"]], 1)
    flat = ids.reshape(-1)
    order = torch.sort(flat, stable=True).indices
    pos = torch.empty_like(order).scatter_(0, order, torch.arange(flat.numel(), device="cuda"))
    counts = (flat[:, None] == torch.arange(E + c["n_shared"], device="cuda")).sum(0)
    offsets = torch.nn.functional.pad(torch.cumsum(counts, 0), (1, 0))
    return [ids.int(), w, offsets.int(), order.int(), pos.int()]


def _plain_norm(s):
    c = s["c"]
    z = s["x"].float() if s["r"] is None else s["x"].float() + s["r"].float()
    y = z * torch.rsqrt(z.square().mean(1, keepdim=True) + EPS) * s["w"].float()
    out = [] if s["r"] is None else [z.to(s["x"].dtype)]
    if c["y16"]:
        out.append(y.to(s["x"].dtype))
    return out + list(_quant(y, 128)) if c["y8"] else out


def _plain_gemm(s):
    c = s["c"]
    a = (s["a8"].float().view(c["M"], -1, 128) * s["a_s"][..., None]).view(c["M"], c["K"])
    w_s = s["w_s"].repeat_interleave(128, 0)[:c["N"]]
    w = (s["w8"].float().view(c["N"], -1, 128) * w_s[..., None]).view(c["N"], c["K"])
    return (a @ w.T).to(s["out"].dtype)


def run(state):
    s, c, kind = state, state["c"], state["kind"]
    if not own:
        return {"attn": _plain_attn, "append": _plain_append, "route": _plain_route, "norm": _plain_norm, "gemm": _plain_gemm}[kind](s)
    if kind == "attn":
        n = c["g"] * c["Hkv"]
        q = s["rows"][:, :n * c["D"]].view(c["B"], n, c["D"])
        return s["cache"].attend(q, s["table"], s["lens"], c["L"], window=c["window"], out=s["out"])
    if kind == "append":
        kv = s["rows"].view(c["T"], 2, c["Hkv"], c["D"])
        s["cache"].append(kv[:, 0], kv[:, 1], s["slots"])
        return _cache_views(s["pool"][:s["n"]], c)
    if kind == "route":
        return list(s["ops"].route_grouped(s["logits"], c["K"], score=c["score"], bias=s["bias"], groups=c["groups"],
                                           top_groups=c["top_groups"], group_top=c["group_top"], renorm=c["renorm"],
                                           scale=c["scale"], n_shared=c["n_shared"], gate=s["gate"], out=s["out"]))
    if kind == "norm":
        s["ops"].rms_norm(s["x"], s["w"], s["r"], eps=EPS, out=s["out"])
        return [t for t in s["out"] if t is not None]
    return s["linear"].forward(s["a8"], s["a_s"], out=s["out"])


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    c = dict(case)
    if c["kind"] == "attn":
        keys = sum(min(n, c["window"] or n) for n in _lens(c))
        rows = c["B"] * c["g"] * c["Hkv"] * c["D"]
        token = 2 * c["Hkv"] * (c["D"] * _elt(c) + (4 if c["fp8"] else 0))
        return {"bytes": keys * token + 4 * rows + 4 * c["B"] + 4 * (keys // c["P"]), "flops": 4 * keys * c["g"] * c["Hkv"] * c["D"]}
    if c["kind"] == "append":
        row = 2 * c["Hkv"] * c["D"]
        return {"bytes": c["T"] * (row * (2 + _elt(c)) + (8 * c["Hkv"] if c["fp8"] else 0) + 8), "flops": 0}
    if c["kind"] == "route":
        Kt = c["K"] + c["n_shared"]
        return {"bytes": c["T"] * (c["E"] * (4 if c["logits"] == "f32" else 2) + 16 * Kt), "flops": 0}
    if c["kind"] == "norm":
        row = 2 + (4 if c["res"] else 0) + (2 if c["y16"] else 0) + (1 + 4 / 128 if c["y8"] else 0)
        return {"bytes": int(c["T"] * c["H"] * row) + 2 * c["H"], "flops": 0}
    M, N, K = c["M"], c["N"], c["K"]
    return {"bytes": M * K + N * K + M * N * (4 if c["out"] == "f32" else 2) + 4 * (K // 128) * (M + -(-N // 128)), "flops": 2 * M * N * K}


# ---------------------------------------------------------------------------
# The same in 64 bits
# ---------------------------------------------------------------------------

def _exact_quant(x, group):
    """Scales, and what the codes stand for before they are rounded."""
    v = x.double().unflatten(-1, (-1, group))
    s = (v.abs().amax(-1) / F8_MAX).clamp_min(MIN_SCALE)
    return (v / s[..., None]).flatten(-2), s


def exact(case, seed):
    c = dict(case)
    kind = c["kind"]
    if kind == "attn":
        rows, table, lens, n = _attn_inputs(c, seed)
        parts = _blocks_of(c, n, seed)
        H, D = c["g"] * c["Hkv"], c["D"]
        out = torch.zeros((c["B"], H, D), dtype=torch.float64, device="cuda")
        for b, length in enumerate(lens.tolist()):
            if not length:
                continue
            first = max(0, length - c["window"]) if c["window"] else 0
            idx = table[b].long()
            kv = []
            for i in (0, 1):
                t = parts[i][idx].double() * (parts[2 + i][idx].double()[..., None] if c["fp8"] else 1.0)
                kv.append(t.permute(1, 0, 2, 3).reshape(c["Hkv"], -1, D)[:, first:length])
            q = rows[b, :H * D].double().view(c["Hkv"], c["g"], D)
            for h in range(c["Hkv"]):
                out[b, h * c["g"]:(h + 1) * c["g"]] = torch.softmax(q[h] @ kv[0][h].T / math.sqrt(D), 1) @ kv[1][h]
        return out
    if kind == "append":
        rows, slots, n = _append_inputs(c, seed)
        parts = [t.double() for t in _blocks_of(c, n, seed)]
        at = (slots >= 0).nonzero()[:, 0]
        block, t = slots[at] // c["P"], slots[at] % c["P"]
        kv = rows.view(c["T"], 2, c["Hkv"], c["D"])[at].double()
        for i in (0, 1):
            if c["fp8"]:
                x, s = _exact_quant(kv[:, i], c["D"])
                parts[i][block, :, t], parts[2 + i][block, :, t] = x, s[..., 0]
            else:
                parts[i][block, :, t] = kv[:, i]
        out = [torch.cat([_tiles_k(parts[0], c), _tiles_v(parts[1], c)], 2).reshape(n, -1)]
        return out + [torch.cat([parts[2].reshape(n, -1), parts[3].reshape(n, -1)], 1)] if c["fp8"] else out
    if kind == "route":
        logits, bias, gate = _route_inputs(c, seed)
        x, G = logits.double(), c["groups"]
        p = torch.sigmoid(x) if c["score"] == "sigmoid" else torch.softmax(x, 1)
        pick = (p + bias.double() if c["bias"] else p).view(c["T"], G, -1)
        score = pick.topk(min(c["group_top"], pick.shape[2]), 2).values.sum(2)
        cut = score.topk(c["top_groups"], 1).values[:, -1:]
        pick = pick.masked_fill((score < cut)[..., None], -math.inf).view(c["T"], -1)
        w = p.gather(1, torch.sort(pick, dim=1, descending=True, stable=True).indices[:, :c["K"]])
        w = (w / w.sum(1, keepdim=True) if c["renorm"] else w) * c["scale"]
        return [None, torch.cat([w, gate.double()], 1) if c["n_shared"] else w, None, None, None]
    if kind == "norm":
        x, r, w = _norm_inputs(c, seed)
        z = x.double() + (r.double() if c["res"] else 0.0)
        y = z / torch.sqrt((z * z).sum(1, keepdim=True) / c["H"] + EPS) * w.double()
        out = ([z] if c["res"] else []) + ([y] if c["y16"] else [])
        return out + list(_exact_quant(y, 128)) if c["y8"] else out
    a8, a_s, w8, w_s = _gemm_inputs(c, seed)
    a = a8.double() * a_s.double().repeat_interleave(128, 1)
    w = w8.double() * w_s.double().repeat_interleave(128, 0)[:c["N"]].repeat_interleave(128, 1)
    return a @ w.T
