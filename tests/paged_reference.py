"""Plain reference of the paged private store, on the CPU: byte layout of the 4-bit blocks, rotation,
quantisation, attention in 64 bits, and the error bounds that follow from the kernels' roundings."""
from __future__ import annotations

import numpy as np
import torch

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E2M1_SIGNED = np.concatenate([E2M1, -E2M1])
MAX_SCALE = np.float32(10912.0)


def to_f64(bf16_tensor):
    return bf16_tensor.detach().cpu().double().numpy()


def byte_map(D):
    """Per (token of the block, dimension): byte of the key and value code, shift of the nibble; and the
    byte of the key and value scale."""
    t, d = np.meshgrid(np.arange(16), np.arange(D), indexing="ij")
    kb = t * (D // 2) + ((d % 32) // 8) * (D // 8) + (d // 32) * 4 + (d % 8) // 2
    x = d // (D // 8)
    s = 2 * ((t // 2) % 4) if D == 128 else 4 * ((t // 4) % 2)
    vb = 8 * D + (t // 2) * D + (x ^ s) * (D // 8) + (t % 2) * (D // 16) + (d % (D // 8)) // 2
    ks = 16 * D + 2 * (t * (D // 32) + d // 32)
    vs = 17 * D + 2 * ((d // 32) * 16 + t)
    return kb, vb, ks, vs, 4 * (d % 2)


def unpack(pages4):
    """uint8 [n_pages][Hkv][blocks][18 D] -> keys, values float64 [n_pages][page_size][Hkv][D]."""
    p = pages4.detach().cpu().numpy()
    n, H, nb, bb = p.shape
    D = bb // 18
    kb, vb, ks, vs, sh = byte_map(D)

    def one(code_at, scale_at):
        code = (p[..., code_at] >> sh) & 15
        scale = (p[..., scale_at].astype(np.uint16) | (p[..., scale_at + 1].astype(np.uint16) << 8)).view(np.float16)
        with np.errstate(invalid="ignore"):
            x = E2M1_SIGNED[code] * scale.astype(np.float64)
        return x.reshape(n, H, nb * 16, D).transpose(0, 2, 1, 3)

    return one(kb, ks), one(vb, vs)


def rotate32(x, cos_sin, rot, interleaved):
    """float32 [N][H][D], [N][rot]: the operator's own rounding, every product and sum once."""
    y = x.astype(np.float32).copy()
    if rot == 0:
        return y
    h = rot // 2
    c, s = cos_sin[:, None, :h].astype(np.float32), cos_sin[:, None, h:].astype(np.float32)
    a, b = (y[..., 0:rot:2].copy(), y[..., 1:rot:2].copy()) if interleaved else (y[..., :h].copy(), y[..., h:rot].copy())
    lo, hi = a * c - b * s, b * c + a * s
    if interleaved:
        y[..., 0:rot:2], y[..., 1:rot:2] = lo, hi
    else:
        y[..., :h], y[..., h:rot] = lo, hi
    return y


def rotate64(x, cos_sin, rot, interleaved):
    """The rotation as complex products in 64 bits."""
    y = np.array(x, dtype=np.float64)
    if rot == 0:
        return y
    h = rot // 2
    z = (cos_sin[:, :h].astype(np.float64) + 1j * cos_sin[:, h:].astype(np.float64))[:, None, :]
    r = y[..., :rot]
    w = (r[..., 0::2] + 1j * r[..., 1::2] if interleaved else r[..., :h] + 1j * r[..., h:]) * z
    if interleaved:
        y[..., 0:rot:2], y[..., 1:rot:2] = w.real, w.imag
    else:
        y[..., :h], y[..., h:rot] = w.real, w.imag
    return y


def quantise32(x):
    """float32 [..., D] -> codes [..., D] 0..15, scales float16 [..., D / 32], by the operator's definition."""
    g = x.astype(np.float32).reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    with np.errstate(invalid="ignore", over="ignore"):
        amax = np.abs(g).max(-1)
        s = np.minimum(amax / np.float32(6.0), MAX_SCALE).astype(np.float16)
    s = np.where(np.isfinite(amax), s, np.float16(np.nan)).astype(np.float16)
    t = s.astype(np.float32)[..., None]
    a = np.abs(g)
    with np.errstate(invalid="ignore"):
        code = sum((a > np.float32(m) * t if even else a >= np.float32(m) * t).astype(np.uint8)
                   for m, even in ((0.25, True), (0.75, False), (1.25, True), (1.75, False), (2.5, True), (3.5, False),
                                   (5.0, True)))
    return (code | (np.signbit(g).astype(np.uint8) << 3)).reshape(x.shape), s


def held32(x):
    """The float64 values that the 4-bit format holds of float32 rows, by the operator's definition."""
    code, s = quantise32(x)
    with np.errstate(invalid="ignore"):
        return E2M1_SIGNED[code] * np.repeat(s.astype(np.float64), 32, axis=-1)


def nearest64(x):
    """What 4 bits with a scale per 32 dimensions hold of x, and half the distance to the next code: the
    nearest value by distance, ties to the even code."""
    g = np.asarray(x, dtype=np.float64).reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    s = np.minimum(np.abs(g).max(-1, keepdims=True) / 6, 10912.0).astype(np.float16).astype(np.float64)
    u = np.abs(g) / np.where(s > 0, s, 1.0)
    dist = np.abs(u[..., None] - E2M1)
    best = dist.min(-1, keepdims=True)
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])  # even codes first: argmax finds the first of the nearest
    pick = order[np.argmax(dist[..., order] == best, axis=-1)]
    return (E2M1[pick] * s * np.sign(g)).reshape(x.shape), np.broadcast_to(s, g.shape).reshape(x.shape)


def pack(pages4, page, slot, h, kc, ks, vc, vs):
    """Writes one token's codes [D] and scales [D / 32] of one KV head into a numpy pool in place."""
    D = kc.shape[0]
    kb, vb, kso, vso, sh = byte_map(D)
    blk, t = pages4[page, h, slot // 16], slot % 16
    for d in range(D):
        for at, code in ((kb[t, d], kc[d]), (vb[t, d], vc[d])):
            blk[at] = (blk[at] & (0xF0 if sh[t, d] == 0 else 0x0F)) | (int(code) << sh[t, d])
    for j in range(D // 32):
        for at, sc in ((kso[t, 32 * j], ks[j]), (vso[t, 32 * j], vs[j])):
            bits = int(np.float16(sc).view(np.uint16))
            blk[at], blk[at + 1] = bits & 255, bits >> 8


def context(k_pages, v_pages, table_row, length):
    """Keys and values [length][Hkv][D] of one context from pages [n_pages][page_size][Hkv][D]."""
    ps = k_pages.shape[1]
    t = np.arange(length)
    pg = np.asarray(table_row)[t // ps]
    return k_pages[pg, t % ps], v_pages[pg, t % ps]


def attend(q, k, v, scale, fmt):
    """q [Hq][D], k and v [T][Hkv][D], all float64 -> out [Hq][D], lse [Hq] and the bounds of both.

    Bounds.  Scores: the products are exact, the sums fp32: |ds| <= 2^-21 scale sum|q k| (accumulation in
    the MMA, the group scales and the multiplication by scale * log2 e).  p carries that relative error,
    the exponential's (2^-22) and its rounding to 16 bits: half a step, 2^-8 in bf16 and 2^-11 in f16,
    below f16's normal range 2^-25 absolute for a row whose largest p is 1 (the row sum is at least 1).
    4-bit values times their scale are rounded to f16: 2^-11.  Every output is rounded to bf16 once: 2^-8.
    The fp32 sums of n terms and the joins of warps and splits: 2^-19 of the absolute sum.
    """
    Hq, D = q.shape
    T, Hkv = k.shape[:2]
    if T == 0:
        return np.zeros((Hq, D)), np.full(Hq, -np.inf), np.zeros((Hq, D)), np.zeros(Hq)
    kk, vv = np.repeat(k, Hq // Hkv, axis=1), np.repeat(v, Hq // Hkv, axis=1)
    s = np.einsum("hd,thd->ht", q, kk) * scale
    ds = 2.0 ** -21 * scale * np.einsum("hd,thd->ht", np.abs(q), np.abs(kk)).max(-1)
    m = s.max(-1, keepdims=True)
    p = np.exp(s - m)
    l = p.sum(-1, keepdims=True)
    out = np.einsum("ht,thd->hd", p / l, vv)
    mass = np.einsum("ht,thd->hd", p / l, np.abs(vv))
    half = 2.0 ** -8 if fmt == "bf16" else 2.0 ** -11 + 2.0 ** -11
    tiny = 0.0 if fmt == "bf16" else 2.0 ** -25
    tol = (half * (1 + 2.0 ** -8) + 2 * ds[:, None] + 2.0 ** -19) * mass + tiny * np.abs(vv).sum(0) / l
    tol = tol + 2.0 ** -8 * (np.abs(out) + tol) + 1e-30
    lse = (m + np.log(l))[:, 0]
    return out, lse, tol, ds + 2.0 ** -20 + 2.0 ** -22 * np.abs(lse)


def make_bf16(shape, gen, scale=1.0):
    return (torch.randn(shape, generator=gen) * scale).to(torch.bfloat16)


def angles(n_positions, rot, base=10000.0):
    """The table [n_positions][rot] of cosines and sines, computed in 64 bits."""
    a = np.arange(n_positions)[:, None] * base ** (-np.arange(rot // 2) / max(1, rot // 2))
    return torch.from_numpy(np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32))
