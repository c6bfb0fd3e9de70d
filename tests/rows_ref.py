"""Operators of several new tokens per sequence from their definitions, in 64 bits,
for the tests: head norms with the rotation, masks and attention of rows, what a
pool holds of a slot."""
import math

import numpy as np
import torch

import ops_ref as R


def heads(x, positions, inv_freq, dims, interleaved, amplitude, norm, weight, eps):
    """(y, mass) of heads x [T, n, D]: the turned values and what bounds their
    error: the magnitudes that enter each, times the amplitude."""
    y = x.double()
    if norm:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps)
        if weight is not None:
            y = y * weight.double()
    out, mass = y.clone(), y.abs().clone()
    for i in range(dims // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + dims // 2)
        angle = positions.double() * inv_freq[i].double()
        c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
        out[..., a] = amplitude * (y[..., a] * c - y[..., b] * s)
        out[..., b] = amplitude * (y[..., a] * s + y[..., b] * c)
        mass[..., a] = mass[..., b] = abs(amplitude) * (y[..., a].abs() + y[..., b].abs())
    return out, mass


def heads_rel(D, positions, inv_freq):
    """Relative error of a turned value in fp32, against its mass: the norm's as in
    the norm's tests ((D / 2 + 16) 2^-23), sine and cosine (an angle off by 2^-24 of
    half a turn, so by less than 2^-22, and functions correct to a few units: 2^-21
    together), two products and a sum (2^-22); the angle in 64 bits is off by its own
    2^-51."""
    angle = float(positions.double().abs().max() * inv_freq.double().abs().max()) if len(inv_freq) and len(positions) else 0.0
    return (D / 2 + 16) * 2.0 ** -23 + 2.0 ** -21 + 2.0 ** -22 + angle * 2.0 ** -51


def seen(n, ctx, masks=None, window=0):
    """[n, ctx + n] truth values: what each of a sequence's n rows sees."""
    t, out = torch.arange(ctx + n), torch.zeros(n, max(ctx + n, 0), dtype=torch.bool)
    for i in range(n):
        if masks is None:
            out[i] = (t <= ctx + i) & ((t > ctx + i - window) if window else True)
        else:
            bits = [bool(int(masks[i, j // 64]) >> (j % 64) & 1) if j // 64 < masks.shape[1] else False for j in range(n)]
            d = torch.tensor(bits)
            out[i, max(ctx, 0):] = d[max(-ctx, 0):]
            if ctx > 0:
                out[i, :ctx] = t[:ctx] >= ctx + int(d.sum()) - window if window else True
    return out


def attend(q, k, v, on, scale):
    """q [n, Hq, D], k, v [L, H, D], on [n, L] -> (out, lse, mass, score sizes), all in
    64 bits. Keys and values that a row does not see are not used."""
    n, Hq, D = q.shape
    H, q = k.shape[1], q.double()
    out, mass = torch.zeros(n, Hq, D, dtype=torch.float64, device=q.device), torch.zeros(n, Hq, D, dtype=torch.float64, device=q.device)
    lse = torch.full((n, Hq), -math.inf, dtype=torch.float64, device=q.device)
    big = torch.zeros(n, Hq, dtype=torch.float64, device=q.device)
    odd = ~(torch.isfinite(k).all(-1).all(-1) & torch.isfinite(v).all(-1).all(-1))
    for h in range(Hq):
        kh, vh = k[:, h // (Hq // H)].double(), v[:, h // (Hq // H)].double()
        rows = (~(on & odd).any(1)).nonzero()[:, 0]
        kf, vf = (torch.where(odd[:, None], 0.0, x) for x in (kh, vh))
        s = (q[rows, h] @ kf.T * scale).masked_fill(~on[rows], -math.inf)
        big[rows, h] = ((q[rows, h].abs() @ kf.abs().T) * on[rows]).amax(1) * abs(scale) if k.shape[0] else 0.0
        top = s.amax(1, keepdim=True).clamp_min(-1e300) if k.shape[0] else torch.zeros(len(rows), 1, dtype=torch.float64, device=q.device)
        p = torch.exp(s - top)
        den = p.sum(1, keepdim=True)
        lse[rows, h] = torch.where(den > 0, top + torch.log(den), -math.inf)[:, 0]
        p = torch.where(den > 0, p / den, 0.0)
        out[rows, h], mass[rows, h] = p @ vf, p @ vf.abs()
        for r in (on & odd).any(1).nonzero()[:, 0]:               # rows that see a value that is no number
            at = on[r].nonzero()[:, 0]
            s = kh[at] @ q[r, h] * scale
            big[r, h] = (kh[at].abs() @ q[r, h].abs()).amax() * abs(scale)
            p = torch.softmax(s, 0)
            lse[r, h] = torch.logsumexp(s, 0)
            out[r, h], mass[r, h] = (p[:, None] * vh[at]).sum(0), (p[:, None] * vh[at].abs()).sum(0)
    return out, lse, mass, big


def read_slot(pool, stride, slot, H, P, D, bits):
    """(keys, values [H, D], their scales [H]) that a numpy uint8 pool holds at a
    slot; the scales are ones in 16 bits (then keys and values are raw uint16)."""
    t, base, d = slot % P, slot // P * stride, np.arange(D)
    out, scales = [], []
    for i in (0, 1):
        rows, sc = [], []
        for h in range(H):
            at = base + (2 * h + i) * P * D * bits // 8 + (R.key_byte, R.value_byte)[i](t, d, D, bits)
            if bits == 16:
                rows.append(pool[at].astype(np.uint16) | pool[at + 1].astype(np.uint16) << 8)
            else:
                rows.append(pool[at])
                so = base + 2 * H * P * D + 4 * ((i * H + h) * P + t)
                sc.append(pool[so:so + 4].view(np.float32)[0])
        out.append(np.stack(rows))
        scales.append(np.array(sc))
    return out[0], out[1], scales[0], scales[1]


def cached(x, bits):
    """What the cache holds of keys or values x [..., D] in 64 bits; in 8 bits a NaN
    stays in its own place, it has no part in the group's scale."""
    if bits == 16:
        return x.double()
    s = (torch.where(torch.isnan(x), 0.0, x.float()).abs().amax(-1) / torch.tensor(448.0)).clamp_min(2.0 ** -126)
    return (x.float() / s[..., None]).to(R.F8).double() * s[..., None].double()
