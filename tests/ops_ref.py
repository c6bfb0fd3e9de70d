"""The operators around the experts from their definitions, in 64 bits on the
host, for the tests: numpy and torch's CPU types only."""
import math

import numpy as np
import torch

F8 = torch.float8_e4m3fn
# unit roundoff of a type: half the spacing at 1
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24, F8: 2.0 ** -4}
# half the spacing of its subnormal numbers
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150, F8: 2.0 ** -10}


def quant(v, group):
    """(codes as float8, scales float32) of groups of the last axis of a float32
    CPU tensor: s = max(amax / 448, 2^-126), codes e4m3(v / s)."""
    g = v.float().unflatten(-1, (-1, group))
    s = (g.abs().amax(-1) / torch.tensor(448.0)).clamp_min(2.0 ** -126)
    return (g / s[..., None]).to(F8).flatten(-2), s


def norm(x, r, w, eps):
    z = x.double() + (0 if r is None else r.double())
    y = z / torch.sqrt((z * z).mean(-1, keepdim=True) + eps)
    return z, y if w is None else y * w.double()


def block_bytes(H, P, D, bits):
    return 2 * H * P * D * bits // 8 + (8 * H * P if bits == 8 else 0)


def key_byte(t, d, D, bits):
    lane = 16 * (d // 8 % 4) + t % 16
    if bits == 16:
        return (t // 16 * (D // 32) + d // 32) * 1024 + 16 * lane + 2 * (d % 8)
    return (t // 16 * (D // 64) + d // 64) * 1024 + 16 * lane + 8 * (d // 32 % 2) + d % 8


def value_byte(t, d, D, bits):
    lane = 16 * (t // 4 % 4) + d % 16
    if bits == 16:
        return (t // 32 * (D // 16) + d // 16) * 1024 + 16 * lane + 2 * (4 * (t // 16 % 2) + t % 4)
    return (t // 32 * (D // 32) + d // 32) * 1024 + 16 * lane + 8 * (d // 16 % 2) + 4 * (t // 16 % 2) + t % 4


def write_slots(pool, stride, k, v, slots, P, bits, n_blocks):
    """Write k, v [T, H, D] (16-bit CPU tensors) into a numpy uint8 pool, as the
    header's layout says, one token at a time."""
    T, H, D = k.shape
    d = np.arange(D)
    for n in range(T):
        s = int(slots[n])
        if s < 0 or s // P >= n_blocks:
            continue
        t, base = s % P, s // P * stride
        for h in range(H):
            for i, x in enumerate((k[n, h], v[n, h])):
                off = base + (2 * h + i) * P * D * bits // 8
                at = off + (key_byte, value_byte)[i](t, d, D, bits)
                if bits == 16:
                    b = x.contiguous().view(torch.uint8).numpy().reshape(D, 2)
                    pool[at], pool[at + 1] = b[:, 0], b[:, 1]
                else:
                    q, sc = quant(x[None], D)
                    pool[at] = q[0].view(torch.uint8).numpy()
                    so = base + 2 * H * P * D + 4 * ((i * H + h) * P + t)
                    pool[so:so + 4] = sc[0].view(torch.uint8).numpy()


def cached(x, bits):
    """What the cache holds of keys or values x [..., D] in 64 bits."""
    if bits == 16:
        return x.double()
    q, s = quant(x.float(), x.shape[-1])
    return q.double() * s.double()


def attend(q, k, v, length, scale, window, missing=()):
    """One sequence: q [Hq, D], k, v [L, H, D] in 64 bits -> (out, lse, mass,
    largest score error scale): mass = sum p |v|, the last sum |q| |k| scale."""
    Hq, D = q.shape
    H = k.shape[1]
    pos = [t for t in range(max(0, length - window) if window else 0, length) if t not in missing]
    out = torch.zeros(Hq, D, dtype=torch.float64)
    mass = torch.zeros(Hq, D, dtype=torch.float64)
    lse = torch.full((Hq,), -math.inf, dtype=torch.float64)
    big = torch.zeros(Hq, dtype=torch.float64)
    if not pos:
        return out, lse, mass, big
    idx = torch.tensor(pos)
    for h in range(Hq):
        kk, vv = k[idx, h // (Hq // H)], v[idx, h // (Hq // H)]
        s = kk @ q[h].double() * scale
        big[h] = (kk.abs() @ q[h].double().abs()).max() * abs(scale)
        p = torch.softmax(s, 0)
        out[h], mass[h], lse[h] = p @ vv, p @ vv.abs(), torch.logsumexp(s, 0)
    return out, lse, mass, big


def route(logits, K, score="softmax", bias=None, groups=1, top_groups=1, group_top=1, renorm=True, scale=1.0):
    """(ids, w) of logits [T, E] float32, by repeated search."""
    T, E = logits.shape
    ids, w = np.zeros((T, K), np.int32), np.zeros((T, K))
    for t in range(T):
        x = np.minimum(logits[t].astype(np.float64), 3.0e38)
        off = np.isnan(x) | (x == -np.inf)
        p = np.zeros(E)
        if score == "sigmoid":
            with np.errstate(over="ignore"):
                p[~off] = 1.0 / (1.0 + np.exp(-x[~off]))
        elif not off.all():
            p[~off] = np.exp(x[~off] - x[~off].max())
            p /= p.sum()
        c = p + (0.0 if bias is None else bias.astype(np.float64))
        c[off | np.isnan(c)] = -np.inf
        if top_groups < groups:
            gs = []
            for g in range(groups):
                best = sorted((v for v in c[g * (E // groups):(g + 1) * (E // groups)] if v > -np.inf), reverse=True)
                gs.append(sum(best[:group_top]) if best else -np.inf)
            kept = sorted(range(groups), key=lambda g: (-gs[g], g))[:top_groups]
            for g in range(groups):
                if g not in kept:
                    c[g * (E // groups):(g + 1) * (E // groups)] = -np.inf
        order = sorted(range(E), key=lambda e: (-c[e], e))[:K]
        pw = np.array([p[e] if c[e] > -np.inf else 0.0 for e in order])
        if renorm:
            pw = pw / pw.sum() if pw.sum() > 0 else pw * 0.0
        ids[t], w[t] = order, pw * scale
    return ids, w


def permute(ids, E):
    flat = ids.reshape(-1)
    order = np.argsort(flat, kind="stable").astype(np.int32)
    pos = np.empty_like(order)
    pos[order] = np.arange(flat.size, dtype=np.int32)
    return np.concatenate([[0], np.cumsum(np.bincount(flat, minlength=E))]).astype(np.int32), order, pos
